"""What the student network's operators refuse, through the C ABI and the binding: every check runs on the host,
before anything reaches a device, so none of this needs a GPU."""
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


def _norm(**kw):
    a = dict(x=P, ldx=64, r=P, ldr=64, w=P, prec=BF16, rows=4, cols=64, eps=1e-6, s=P, lds=64, o=P, ldo=64, rstd=P)
    a.update(kw)
    return [a[k] for k in ("x", "ldx", "r", "ldr", "w", "prec", "rows", "cols", "eps", "s", "lds", "o", "ldo",
                           "rstd")] + [None]


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(w=None), "NULL"), (dict(o=None), "NULL"), (dict(prec=2), "precision"),
    (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"), (dict(cols=32769), "cols"),
    (dict(ldx=63), "leading"), (dict(ldr=63), "leading"), (dict(lds=63), "leading"), (dict(ldo=63), "leading"),
    (dict(ldx=1 << 31), "leading"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps")])
def test_norm_refuses(kw, part):
    _refused("pack_add_rms_norm", _norm(**kw), part)
    _refused("pack_add_rms_norm_q8", _norm(**kw), part)


def test_norm_codes_need_a_scale():
    _refused("pack_add_rms_norm_q8", _norm(rstd=None), "NULL")


@pytest.mark.parametrize("kw,part", [(dict(x=None), "NULL"), (dict(q=None), "NULL"), (dict(s=None), "NULL"),
                                     (dict(prec=-1), "precision"), (dict(cols=40_000), "cols"),
                                     (dict(ldx=7), "leading"), (dict(ldq=7), "leading")])
def test_quantize_refuses(kw, part):
    a = dict(x=P, ldx=8, prec=FP32, rows=2, cols=8, q=P, ldq=8, s=P)
    a.update(kw)
    _refused("pack_quantize_rows", [a[k] for k in ("x", "ldx", "prec", "rows", "cols", "q", "ldq", "s")] + [None], part)


@pytest.mark.parametrize("kw,part", [
    (dict(dy=None), "NULL"), (dict(v=None), "NULL"), (dict(w=None), "NULL"), (dict(rstd=None), "NULL"),
    (dict(dx=None), "NULL"), (dict(dw=None), "NULL"), (dict(work=None), "NULL"), (dict(nbytes=15), "workspace"),
    (dict(work=P + 2), "aligned"), (dict(ldy=3), "leading"), (dict(lds=3), "leading"), (dict(ldd=3), "leading"),
    (dict(ldx=3), "leading"), (dict(prec=7), "precision"), (dict(rows=-2), "rows"), (dict(cols=0), "cols")])
def test_norm_backward_refuses(kw, part):
    a = dict(dy=P, ldy=4, v=P, lds=4, w=P, rstd=P, ds=P, ldd=4, prec=FP32, rows=1, cols=4, dx=P, ldx=4, dw=P, work=P,
             nbytes=16)
    a.update(kw)
    _refused("pack_rms_norm_backward", [a[k] for k in ("dy", "ldy", "v", "lds", "w", "rstd", "ds", "ldd", "prec",
                                                       "rows", "cols", "dx", "ldx", "dw", "work", "nbytes")] + [None],
             part)
    lib = tabpack.load_library()
    assert lib.pack_rms_norm_backward_workspace_size(4, 4, None) == -1
    n = ctypes.c_size_t()
    assert lib.pack_rms_norm_backward_workspace_size(0, 4, ctypes.byref(n)) == 0 and n.value >= 16


@pytest.mark.parametrize("kw,part", [
    (dict(z=None), "NULL"), (dict(idx=None), "NULL"), (dict(t=None), "NULL"), (dict(loss=None), "NULL"),
    (dict(prec=5), "precision"), (dict(rows=-1), "rows"), (dict(V=0), "classes"), (dict(k=0), "k="),
    (dict(k=257), "k="), (dict(tau=0.0), "temperature"), (dict(tau=-1.0), "temperature"),
    (dict(tau=float("nan")), "temperature"), (dict(tau=float("inf")), "temperature"), (dict(tau=1e-40), "temperature"),
    (dict(tau=3e38), "temperature"), (dict(ldz=9), "leading"), (dict(ldg=9), "leading")])
def test_distill_refuses(kw, part):
    a = dict(z=P, ldz=10, prec=FP32, rows=2, V=10, idx=P, t=P, k=3, tau=1.0, w=P, loss=P, g=P, ldg=10)
    a.update(kw)
    _refused("pack_distill_topk", [a[k] for k in ("z", "ldz", "prec", "rows", "V", "idx", "t", "k", "tau", "w", "loss",
                                                  "g", "ldg")] + [None], part)


FF = dict(x=P, ldx=16, wg=P, ldwg=16, wd=P, ldwd=24, r=P, ldr=8, prec=BF16, act=0, T=4, D=16, F=24, O=8, gu=P, h=P,
          out=P, ldo=8, work=P, nbytes=1 << 40)


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(wg=None), "NULL"), (dict(wd=None), "NULL"), (dict(h=None), "NULL"),
    (dict(out=None), "NULL"), (dict(ldx=15), "leading"), (dict(ldwg=15), "leading"), (dict(ldwd=23), "leading"),
    (dict(ldr=7), "leading"), (dict(ldo=7), "leading"), (dict(prec=2), "precision"), (dict(act=3), "activation"),
    (dict(act=-1), "activation"), (dict(T=-1), "tokens"), (dict(T=1 << 31), "tokens"), (dict(D=0), "d_in"),
    (dict(F=0), "d_in"), (dict(O=0), "d_in"), (dict(F=(1 << 24) + 1), "d_in"),
    (dict(T=100, D=1 << 20, ldx=1 << 20, ldwg=1 << 20, work=None), "work"),
    (dict(T=100, D=1 << 20, ldx=1 << 20, ldwg=1 << 20, nbytes=16), "workspace"),
    (dict(T=100, D=1 << 20, ldx=1 << 20, ldwg=1 << 20, work=P + 8), "aligned")])
def test_gated_ff_refuses(kw, part):
    a = dict(FF, **kw)
    _refused("pack_gated_ff_forward", [a[k] for k in ("x", "ldx", "wg", "ldwg", "wd", "ldwd", "r", "ldr", "prec", "act",
                                                      "T", "D", "F", "O", "gu", "h", "out", "ldo", "work", "nbytes")]
             + [None], part)


@pytest.mark.parametrize("kw,part", [
    (dict(dy=None), "NULL"), (dict(x=None), "NULL"), (dict(gu=None), "NULL"), (dict(h=None), "NULL"),
    (dict(dgu=None), "NULL"), (dict(wd=None), "NULL"), (dict(wg=None), "NULL"), (dict(lddy=7), "leading"),
    (dict(lddx=15), "leading"), (dict(prec=9), "precision"), (dict(act=5), "activation"), (dict(T=-3), "tokens"),
    (dict(T=1 << 20, nbytes=0), "workspace"), (dict(T=1 << 20, work=P + 4), "aligned")])
def test_gated_ff_backward_refuses(kw, part):
    a = dict(FF, dy=P, lddy=8, dgu=P, dx=P, lddx=16, dwg=P, dwd=P)
    a.update(kw)
    _refused("pack_gated_ff_backward", [a[k] for k in ("dy", "lddy", "x", "ldx", "wg", "ldwg", "wd", "ldwd", "gu", "h",
                                                       "prec", "act", "T", "D", "F", "O", "dgu", "dx", "lddx", "dwg",
                                                       "dwd", "work", "nbytes")] + [None], part)


@pytest.mark.parametrize("kw,part", [
    (dict(x=None), "NULL"), (dict(xs=None), "NULL"), (dict(w=None), "NULL"), (dict(ws=None), "NULL"),
    (dict(out=None), "NULL"), (dict(gate=3), "gate"), (dict(gate=-2), "gate"), (dict(prec=3), "precision"),
    (dict(M=-1), "rows"), (dict(N=0), "outputs"), (dict(K=0), "depth"), (dict(K=131072), "depth"),
    (dict(ldx=31), "leading"), (dict(ldw=31), "leading"), (dict(ldo=7), "leading"),
    (dict(M=100, K=131071, ldx=131071, ldw=131071, work=None), "work"),
    (dict(M=100, K=131071, ldx=131071, ldw=131071, nbytes=8), "workspace")])
def test_q8_matmul_refuses(kw, part):
    a = dict(x=P, ldx=32, xs=P, w=P, ldw=32, ws=P, b=P, gate=-1, prec=BF16, M=100, N=8, K=32, out=P, ldo=8, work=P,
             nbytes=1 << 40)
    a.update(kw)
    _refused("pack_q8_matmul", [a[k] for k in ("x", "ldx", "xs", "w", "ldw", "ws", "b", "gate", "prec", "M", "N", "K",
                                               "out", "ldo", "work", "nbytes")] + [None], part)


def test_workspace_sizes():
    lib = tabpack.load_library()
    n = ctypes.c_size_t()
    for T in (0, 1, 17, 4096, (1 << 31) - 1):
        for backward in (0, 1):
            assert lib.pack_gated_ff_workspace_size(BF16, T, 24, 40, 8, backward, ctypes.byref(n)) == 0
        assert lib.pack_q8_matmul_workspace_size(T, 24, 40, -1, ctypes.byref(n)) == 0
        assert lib.pack_rms_norm_backward_workspace_size(T, 24, ctypes.byref(n)) == 0
    assert lib.pack_gated_ff_workspace_size(BF16, 1, 24, 40, 8, 0, None) == -1
    assert lib.pack_gated_ff_workspace_size(2, 1, 24, 40, 8, 0, ctypes.byref(n)) == -1
    assert lib.pack_q8_matmul_workspace_size(1, 24, 40, -1, None) == -1
    assert lib.pack_q8_matmul_workspace_size(1, 0, 40, -1, ctypes.byref(n)) == -1


def test_binding_refuses_host_tensors_and_types():
    h = torch.zeros(2, 8)
    for call in (lambda: ops.add_rms_norm(h, torch.ones(8)), lambda: ops.add_rms_norm_q8(h, torch.ones(8)),
                 lambda: ops.quantize_rows(h), lambda: ops.quantize_rows(h.double()), lambda: ops.quantize_rows([1]),
                 lambda: ops.gated_ff(h, torch.zeros(4, 8), torch.zeros(8, 2)),
                 lambda: ops.q8_matmul(h.char(), torch.ones(2), h.char(), torch.ones(2)),
                 lambda: ops.rms_norm_backward(h, h, torch.ones(8), torch.ones(2)),
                 lambda: ops.distill_topk(h, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))):
        with pytest.raises(tabpack.PackError):
            call()
