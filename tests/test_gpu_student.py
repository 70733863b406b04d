"""The distilled student (student.py) end to end: its logits and gradients against the same network in 64 bits, its
8-bit predictions against its own weights, and a short distillation of a real pack."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import configs, ops, student, synth, tabpack  # noqa: E402

pytestmark = pytest.mark.gpu


def _reference(s, x, act=torch.nn.functional.silu):
    """Logits of the network in 64 bits on the host, differentiable in the parameters."""
    params = [p.detach().double().cpu().requires_grad_() for p in s.params]
    v = x.double().cpu()

    def norm(v, w):
        return v / torch.sqrt((v ** 2).mean(1, keepdim=True) + s.eps) * w

    for b in range(s.blocks):
        w, wg, wd = params[3 * b:3 * b + 3]
        gate, up = (norm(v, w) @ wg.t()).chunk(2, 1)
        v = v + (act(gate) * up) @ wd.t()
    return norm(v, params[-2]) @ params[-1].t(), params


@pytest.mark.parametrize("rows,d_in,classes,hidden", [(70, 24, 5, 40), (33, 37, 10, 51)])
def test_student_gradients_fp32(rows, d_in, classes, hidden):
    s = student.Student(d_in, classes, blocks=2, hidden=hidden, dtype=torch.float32, seed=1)
    for p in s.params:
        if p.dim() == 1:
            p.add_(0.2 * torch.randn_like(p))
    s._copies()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, d_in, generator=g, device="cuda")
    prob = torch.softmax(2 * torch.randn(rows, classes, generator=g, device="cuda"), 1)
    idx, teacher = student.teacher_entries(prob, 3)
    weight = torch.full((rows,), 1.0 / rows, device="cuda")
    logits, kept = s.forward(x)
    loss, dz = ops.distill_topk(logits, idx, teacher, 2.0, weight)
    grads = s.backward(dz, kept)
    ref, params = _reference(s, x)
    # about ten fp32 operations deep over sums of at most 51 terms of order 1: 1e-5 of the largest value is 100 u
    # of slack on each
    assert (logits.double().cpu() - ref).abs().max() <= 1e-5 * ref.abs().max()
    p = torch.softmax(teacher.double().cpu() / 2, 1)
    lq = torch.log_softmax(ref / 2, 1).gather(1, idx.long().cpu())
    total = (4 * p * (torch.log(p) - lq)).sum() / rows
    want = float(total.detach())
    assert abs(float(loss.double().sum()) - want) <= 1e-5 * abs(want)
    for got, want in zip(grads, torch.autograd.grad(total, params)):
        assert got.shape == want.shape
        assert (got.double().cpu() - want).norm() <= 1e-4 * want.norm()


def test_student_in_8_bits_follows_its_weights():
    s = student.Student(64, 10, blocks=2, hidden=128, seed=2)
    x = torch.randn(500, 64, device="cuda")
    ref = torch.softmax(_reference(s, x)[0], 1)
    out = s.predict(x).double().cpu()
    # a code is off by half a step of 1 / 127 of its row's largest value, 5 quantised stages deep
    assert (out - ref).abs().mean() <= 5 * 0.5 / 127 and (out - ref).abs().max() <= 0.15
    assert torch.equal(s.predict(x[:1]), s.predict(x[:1]))


def test_distilled_pack():
    cfg = configs.workload("multiclass_lognormal", K=4, d_in=32, d_out=4, B=256, width_lo=64, width_hi=128, L=2)
    Xh, yh, _, _ = synth.make_data(cfg, n_train=4096, n_val=64)
    X, y = torch.from_numpy(Xh).cuda(), torch.from_numpy(yh).cuda()
    pack = tabpack.Pack(cfg).bind()
    for t in range(1, 161):
        order = synth.epoch_orders(cfg, (t - 1) // 16, 4096)
        pack.train_step(X, y, torch.from_numpy(np.ascontiguousarray(synth.batch_indices(order, (t - 1) % 16, 256))).cuda(), t)
    prob = pack.predict(X, ensemble=True)
    idx, teacher = student.teacher_entries(prob, 3)
    s = student.Student(32, 4, blocks=2, hidden=96, seed=5)
    loss = s.fit(X, idx, teacher, steps=300, batch=512)
    first, last = float(loss[:10].mean()), float(loss[-10:].mean())
    print(f"[student] distillation loss {first:.4f} -> {last:.4f}", flush=True)
    assert np.isfinite(last) and last < 0.25 * first
    agree = (s.predict(X).argmax(1) == prob.argmax(1)).float().mean().item()
    assert agree > 0.9, agree
