"""What layer norm, dropout, embeddings and 8-bit floating point refuse, through the C ABI and the binding: every check
runs on the host, before anything reaches a device, so none of this needs a GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, tabpack  # noqa: E402

P = 4096          # stands for a device address (aligned to 16); no refused call reads it
BF16, FP32 = 0, 1


def _refused(fn, args, part):
    lib = tabpack.load_library()
    assert getattr(lib, fn)(*args) == -1
    assert part in lib.pack_last_error().decode(), lib.pack_last_error()


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(w=None), "NULL"), (dict(o=None), "NULL"), (dict(prec=2), "precision"),
    (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"), (dict(cols=32769), "cols"),
    (dict(ldx=63), "leading"), (dict(ldr=63), "leading"), (dict(lds=63), "leading"), (dict(ldo=63), "leading"),
    (dict(ldx=1 << 31), "leading"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps")])
def test_layer_norm(kw, part):
    a = dict(x=P, ldx=64, r=P, ldr=64, w=P, b=None, prec=BF16, rows=4, cols=64, eps=1e-6, s=P, lds=64, o=P, ldo=64,
             mean=P, rstd=P)
    a.update(kw)
    _refused("pack_add_layer_norm", list(a.values()) + [None], part)


@pytest.mark.parametrize("kw,part", [
    (dict(dy=None), "NULL"), (dict(v=None), "NULL"), (dict(w=None), "NULL"), (dict(mean=None), "NULL"),
    (dict(rstd=None), "NULL"), (dict(dx=None), "NULL"), (dict(dw=None), "NULL"), (dict(work=None), "NULL"),
    (dict(nbytes=31), "workspace"), (dict(work=P + 2), "aligned"), (dict(ldy=3), "leading"), (dict(lds=3), "leading"),
    (dict(ldd=3), "leading"), (dict(ldx=3), "leading"), (dict(prec=7), "precision"), (dict(rows=-2), "rows"),
    (dict(cols=0), "cols")])
def test_layer_norm_backward(kw, part):
    a = dict(dy=P, ldy=4, v=P, lds=4, w=P, mean=P, rstd=P, ds=P, ldd=4, prec=FP32, rows=1, cols=4, dx=P, ldx=4, dw=P,
             db=P, work=P, nbytes=32)
    a.update(kw)
    _refused("pack_layer_norm_backward", list(a.values()) + [None], part)
    n = ctypes.c_size_t()
    lib = tabpack.load_library()
    assert lib.pack_layer_norm_backward_workspace_size(4, 4, None) == -1
    assert lib.pack_layer_norm_backward_workspace_size(0, 20_000, ctypes.byref(n)) == 0 and n.value >= 160_000


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(o=None), "NULL"), (dict(prec=3), "precision"), (dict(rows=-1), "rows"),
    (dict(cols=0), "cols"), (dict(p=-0.1), "p must"), (dict(p=1.5), "p must"), (dict(p=float("nan")), "p must"),
    (dict(ldx=9), "leading"), (dict(ldr=9), "leading"), (dict(ldo=9), "leading"), (dict(at=P + 4), "aligned")])
def test_dropout(kw, part):
    a = dict(x=P, ldx=10, r=P, ldr=10, prec=FP32, rows=2, cols=10, p=0.5, seed=1, step=2, at=None, site=0, o=P, ldo=10)
    a.update(kw)
    _refused("pack_dropout", list(a.values()) + [None], part)


@pytest.mark.parametrize("kw,part", [
    (dict(idx=None), "NULL"), (dict(table=None), "NULL"), (dict(o=None), "NULL"), (dict(prec=2), "precision"),
    (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"), (dict(rows=0), "rows"), (dict(rows=1 << 31), "rows"),
    (dict(cols=0), "cols"), (dict(cols=(1 << 24) + 1), "cols"), (dict(ldt=7), "leading"), (dict(ldo=7), "leading")])
def test_embed(kw, part):
    a = dict(idx=P, wide=0, table=P, ldt=8, prec=BF16, tokens=3, rows=5, cols=8, scale=1.0, o=P, ldo=8)
    a.update(kw)
    _refused("pack_embed", list(a.values()) + [None], part)


@pytest.mark.parametrize("kw,part", [
    (dict(dy=None), "NULL"), (dict(idx=None), "NULL"), (dict(o=None), "NULL"), (dict(prec=2), "precision"),
    (dict(tokens=-1), "tokens"), (dict(rows=0), "rows"), (dict(cols=0), "cols"), (dict(ldy=7), "leading"),
    (dict(work=None), "work"), (dict(nbytes=8), "workspace"), (dict(work=P + 8), "aligned"),
    (dict(tokens=(1 << 31) - 1, cols=1 << 24, ldy=1 << 24, nbytes=1 << 62), "more tiles")])
def test_embed_backward(kw, part):
    a = dict(dy=P, ldy=8, idx=P, wide=1, prec=BF16, tokens=300, rows=5, cols=8, scale=1.0, o=P, work=P, nbytes=1 << 40)
    a.update(kw)
    _refused("pack_embed_backward", list(a.values()) + [None], part)
    assert tabpack.load_library().pack_embed_backward_workspace_size(0, 1, 1, 1, None) == -1


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(q=None), "NULL"), (dict(s=None), "NULL"), (dict(prec=9), "precision"),
    (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"), (dict(cols=(1 << 24) + 1), "cols"),
    (dict(ldx=7), "leading"), (dict(ldq=7), "leading"),
    (dict(rows=(1 << 31) - 1, cols=1 << 20, ldx=1 << 20, ldq=1 << 20), "more tiles")])
def test_codes(kw, part):
    a = dict(x=P, ldx=8, prec=FP32, rows=2, cols=8, q=P, ldq=8, s=P)
    a.update(kw)
    _refused("pack_quantize_blocks", list(a.values()) + [None], part)
    tiles = list(a.values())
    _refused("pack_quantize_tiles", tiles[:4] + [1] + tiles[4:] + [None], part)


def test_tiles_of_no_parts():
    for parts in (0, -1):
        _refused("pack_quantize_tiles", [P, 8, FP32, 2, parts, 8, P, 8, P, None], "parts")
    _refused("pack_quantize_tiles", [P, 8, FP32, 1 << 30, 4, 8, P, 8, P, None], "rows")


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(xs=None), "NULL"), (dict(w=None), "NULL"), (dict(ws=None), "NULL"),
    (dict(o=None), "NULL"), (dict(prec=2), "precision"), (dict(gate=3), "gate"), (dict(gate=-2), "gate"),
    (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(n=0), "outputs"), (dict(k=0), "depth"),
    (dict(k=(1 << 24) + 1), "depth"), (dict(ldx=63), "leading"), (dict(ldw=63), "leading"), (dict(ldo=15), "leading"),
    (dict(k=1 << 20, ldx=1 << 20, ldw=1 << 20, rows=100, nbytes=16), "workspace"),
    (dict(k=1 << 20, ldx=1 << 20, ldw=1 << 20, rows=100, work=None), "work"),
    (dict(k=1 << 20, ldx=1 << 20, ldw=1 << 20, rows=100, work=P + 8), "aligned")])
def test_f8_matmul(kw, part):
    a = dict(x=P, ldx=64, xs=P, w=P, ldw=64, ws=P, b=None, gate=-1, prec=BF16, rows=4, n=16, k=64, o=P, ldo=16, work=P,
             nbytes=1 << 40)
    a.update(kw)
    _refused("pack_f8_matmul", list(a.values()) + [None], part)


def test_the_binding_refuses_host_tensors_and_wrong_ones():
    x, w, idx = torch.ones(4, 8), torch.ones(8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ops.add_layer_norm(x, w), lambda: ops.layer_norm_backward(x, x, w, w[:4], w[:4]),
                 lambda: ops.dropout(x, 0.5, 1, 1), lambda: ops.embed(idx, x), lambda: ops.embed_backward(x, idx, 3),
                 lambda: ops.quantize_blocks(x), lambda: ops.quantize_tiles(x),
                 lambda: ops.f8_matmul(x.to(torch.float8_e4m3fn), w, x.to(torch.float8_e4m3fn), w)):
        with pytest.raises(tabpack.PackError, match="device"):
            call()
    for call in (lambda: ops.add_layer_norm(x.half(), w), lambda: ops.dropout(x.double(), 0.5, 1, 1),
                 lambda: ops.embed(idx, x.half()), lambda: ops.quantize_blocks(idx)):
        with pytest.raises(tabpack.PackError, match="bfloat16 or float32"):
            call()
