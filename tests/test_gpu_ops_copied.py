"""Products from aligned copies of their operands within the error bounds of the block's other tests, in both types, and
without the gradient of the input: what is left out changes no bit of what is not."""
import pytest

torch = pytest.importorskip("torch")
import test_gpu_ops_large as large  # noqa: E402
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]
# tokens, d_in, hidden, d_out: one extent odd at a time and all, a split depth of the gate projections
BLOCKS = [(2050, 515, 1027, 261), (2048, 512, 1025, 256), (2048, 513, 1024, 256), (2051, 512, 1024, 259),
          (300, 9001, 203, 101), (4000, 510, 2044, 514)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("case", BLOCKS, ids=lambda c: "x".join(map(str, c)))
def test_gated_ff_copied(case, act, dtype):
    large.test_gated_ff_large(*case, act, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", BLOCKS + [(4100, 520, 2056, 1032), (4100, 515, 2051, 1029), (9000, 128, 1024, 128),
                                           (100, 2048, 4096, 2048), (16_384, 256, 512, 256)],
                         ids=lambda c: "x".join(map(str, c)))
def test_weights_gradients_without_the_inputs(case, dtype):
    T, D, F, O = case
    print(f"[copied] {T} {D} {F} {O} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(T + D + F)

    def rand(r, c, std=1.0):
        return (torch.randn(r, c, generator=g, device="cuda") * std).to(dtype)

    x, wg, wd, dy = rand(T, D), rand(2 * F, D, D ** -0.5), rand(O, F, F ** -0.5), rand(T, O)
    _, saved = ops.gated_ff(x, wg, wd, save=True)
    full = ops.gated_ff_backward(dy, x, wg, wd, saved)
    part = ops.gated_ff_backward(dy, x, wg, wd, saved, need_dx=False)
    assert part[0] is None and torch.equal(part[1], full[1]) and torch.equal(part[2], full[2])
