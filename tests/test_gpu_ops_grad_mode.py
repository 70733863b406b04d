"""The operators record nothing for autograd, so under grad mode they refuse tensors that require a gradient, which would
be lost; under no_grad the same calls run, and through an autograd.Function the gradients are the backward calls'."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, tabpack  # noqa: E402

pytestmark = pytest.mark.gpu


def _calls():
    """(name, call, its floating tensors) of every operator."""
    g = torch.Generator(device="cuda").manual_seed(1)

    def rand(*s):
        return torch.randn(*s, generator=g, device="cuda")

    x, r, w, dy, dv = rand(6, 16), rand(6, 16), rand(16), rand(6, 16), rand(6, 16)
    wg, wd, z, t, weight = rand(24, 16), rand(16, 12), rand(6, 9), rand(6, 3), rand(6).abs()
    idx = torch.randint(0, 9, (6, 3), generator=g, device="cuda", dtype=torch.int32)
    rstd = rand(6).abs()
    q, s = ops.quantize_rows(x)
    qw, sw = ops.quantize_rows(wg)
    b = rand(24)
    _, (gu, h) = ops.gated_ff(x, wg, wd, save=True)
    return [
        ("add_rms_norm", lambda x, w, r: ops.add_rms_norm(x, w, residual=r), (x, w, r)),
        ("add_rms_norm_q8", lambda x, w, r: ops.add_rms_norm_q8(x, w, residual=r), (x, w, r)),
        ("rms_norm_backward", lambda dy, v, w, rho, dv: ops.rms_norm_backward(dy, v, w, rho, dv=dv),
         (dy, x, w, rstd, dv)),
        ("quantize_rows", ops.quantize_rows, (x,)),
        ("distill_topk", lambda z, t, weight: ops.distill_topk(z, idx, t, row_weight=weight), (z, t, weight)),
        ("gated_ff", lambda x, wg, wd, r: ops.gated_ff(x, wg, wd, residual=r), (x, wg, wd, r)),
        ("gated_ff_backward", lambda dy, x, wg, wd, gu, h: ops.gated_ff_backward(dy, x, wg, wd, (gu, h)),
         (dy, x, wg, wd, gu, h)),
        ("q8_matmul", lambda s, sw, b: ops.q8_matmul(q, s, qw, sw, bias=b), (s, sw, b))]


def test_a_lost_gradient_is_refused():
    for name, call, tensors in _calls():
        want = call(*tensors)
        for i in range(len(tensors)):
            args = [t.detach().clone().requires_grad_(j == i) for j, t in enumerate(tensors)]
            print(f"[grad mode] {name}, tensor {i}", flush=True)
            with pytest.raises(tabpack.PackError, match="no_grad"):
                call(*args)
            for mode in (torch.no_grad, torch.inference_mode):
                with mode():
                    got = call(*args)
                got, ref = (o if isinstance(o, tuple) else (o,) for o in (got, want))
                assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_gradients_through_a_function():
    class Block(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, wg, wd):
            y, saved = ops.gated_ff(x, wg, wd, save=True)
            ctx.save_for_backward(x, wg, wd, *saved)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, wg, wd, gu, h = ctx.saved_tensors
            return ops.gated_ff_backward(dy.contiguous(), x, wg, wd, (gu, h))

    g = torch.Generator(device="cuda").manual_seed(2)
    x, wg, wd = (torch.randn(*s, generator=g, device="cuda").requires_grad_() for s in ((6, 16), (24, 16), (16, 12)))
    y = Block.apply(x, wg, wd)
    y.square().sum().backward()
    with torch.no_grad():
        _, saved = ops.gated_ff(x, wg, wd, save=True)
        want = ops.gated_ff_backward(2 * y, x, wg, wd, saved)
    assert all(torch.equal(t.grad, w) for t, w in zip((x, wg, wd), want))
