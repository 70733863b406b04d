"""One network distilled from an ensemble and served in 8 bits: an example of the operators of ``ops``.

An ensemble of a pack's members (``tabpack``, ``online``) answers with one forward pass per member.  The student is a
single stack of pre-normalised gated blocks over the input features,

    v_0 = x,   v_(l+1) = v_l + W_down (act(W_gate n_l) * (W_up n_l)),   n_l = rms_norm(v_l) w_l,
    logits = W_head rms_norm(v_L) w_L,

trained on the ensemble's class probabilities (the loss against its k most likely classes of each row) and served with
8-bit weights and activations.  Every product over the blocks, every norm and the loss run in the library's kernels;
PyTorch holds the fp32 master weights, applies AdamW to them and does the head's small products in training.

    python -m paper_2607_05380_amd.student            # trains a pack, distils it, serves the student in 8 bits
"""
import argparse

import torch

from . import ops, tabpack


def teacher_entries(prob, k):
    """(classes int32 [rows, k], log-probabilities fp32 [rows, k]) of the k most likely classes of prob [rows, classes]:
    a teacher's entries for ``ops.distill_topk``.  A class of probability 0 has logit -inf and is left out there."""
    top, idx = prob.float().topk(min(k, prob.shape[1]), 1)
    return idx.to(torch.int32).contiguous(), top.log().contiguous()


class Student:
    """Weights of the network: fp32 masters (``params``) and the copies that the kernels read."""

    def __init__(self, d_in, classes, blocks=2, hidden=512, act="silu", dtype=torch.bfloat16, eps=1e-6, seed=0,
                 device="cuda"):
        for name, n in (("d_in", d_in), ("classes", classes), ("blocks", blocks), ("hidden", hidden)):
            if n < 1:
                raise ops.PackError(f"{name}={n} must be positive")
        if act not in tabpack.ACTIVATIONS:
            raise ops.PackError(f"unknown activation {act!r}")
        if dtype not in (torch.bfloat16, torch.float32):
            raise ops.PackError(f"dtype must be bfloat16 or float32, not {dtype}")
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(rows, cols):
            return torch.randn(rows, cols, generator=g, device=device) * cols ** -0.5

        self.act, self.dtype, self.eps, self.classes = act, dtype, eps, classes
        self.params = []
        for _ in range(blocks):
            self.params += [torch.ones(d_in, device=device), normal(2 * hidden, d_in),
                            normal(d_in, hidden) * blocks ** -0.5]
        self.params += [torch.ones(d_in, device=device), normal(classes, d_in)]
        self.blocks = blocks
        self._copies()

    def _copies(self):
        # products read the masters rounded to the student's type; norm weights and the head stay fp32
        self.w = [p if p.dim() == 1 or i == len(self.params) - 1 else p.to(self.dtype)
                  for i, p in enumerate(self.params)]
        self.served = None

    # ------------------------------------------------------------ training
    def forward(self, x):
        """(logits fp32, what backward needs) of rows x [rows, d_in] in the student's type."""
        keep, branch, v = [], None, x
        for b in range(self.blocks):
            norm, wg, wd = self.w[3 * b:3 * b + 3]
            new, stream = (v, None) if branch is None else (branch, v)
            n, v, rstd = ops.add_rms_norm(new, norm, stream, self.eps)
            branch, saved = ops.gated_ff(n, wg, wd, act=self.act, save=True)
            keep.append((n, v, rstd, saved))
        n, v, rstd = ops.add_rms_norm(branch, self.w[-2], v, self.eps)
        return n.float() @ self.w[-1].t(), (keep, (n, v, rstd))

    def backward(self, dlogits, kept):
        """Gradients of ``params`` (fp32) from those of the logits."""
        keep, (n, v, rstd) = kept
        dn = (dlogits @ self.w[-1]).to(self.dtype)
        # the sum's gradient goes to the branch and, unchanged, to the stream it was added to
        dv, dnorm = ops.rms_norm_backward(dn, v, self.w[-2], rstd)
        grads = [dnorm, dlogits.t() @ n.float()]
        for b in reversed(range(self.blocks)):
            norm, wg, wd = self.w[3 * b:3 * b + 3]
            n, v, rstd, saved = keep[b]
            dn, dwg, dwd = ops.gated_ff_backward(dv, n, wg, wd, saved, act=self.act)
            dv, dnorm = ops.rms_norm_backward(dn, v, norm, rstd, dv=dv)
            grads = [dnorm, dwg.float(), dwd.float()] + grads
        return grads

    def fit(self, X, idx, teacher, steps, batch=1024, lr=2e-3, temperature=2.0, seed=0):
        """Distils: ``steps`` AdamW steps on batches of the rows X (fp32) with the teacher's entries; the mean loss of
        each step."""
        opt = torch.optim.AdamW(self.params, lr=lr, weight_decay=1e-4)
        g = torch.Generator(device=X.device).manual_seed(seed)
        weight = torch.full((batch,), 1.0 / batch, device=X.device)
        losses = []
        for _ in range(steps):
            rows = torch.randint(0, X.shape[0], (batch,), generator=g, device=X.device)
            logits, kept = self.forward(X[rows].to(self.dtype))
            loss, dlogits = ops.distill_topk(logits, idx[rows], teacher[rows], temperature, weight)
            for p, grad in zip(self.params, self.backward(dlogits, kept)):
                p.grad = grad
            opt.step()
            self._copies()
            losses.append(loss.sum())
        return torch.stack(losses) if losses else torch.empty(0, device=X.device)

    # ------------------------------------------------------------- serving
    def quantize(self):
        """Lays the weights out in 8 bits (once; a later fit() drops them)."""
        self.served = [p if p.dim() == 1 else ops.quantize_rows(p) for p in self.params]
        return self

    def predict(self, X):
        """Class probabilities [rows, classes] of rows X (fp32) by the 8-bit network."""
        if self.served is None:
            self.quantize()
        branch, v = None, X.to(torch.bfloat16)
        for b in range(self.blocks):
            norm, (wg, sg), (wd, sd) = self.served[3 * b:3 * b + 3]
            new, stream = (v, None) if branch is None else (branch, v)
            q, s, v = ops.add_rms_norm_q8(new, norm, stream, self.eps)
            q, s = ops.quantize_rows(ops.q8_matmul(q, s, wg, sg, gate=self.act))
            branch = ops.q8_matmul(q, s, wd, sd)
        q, s, _ = ops.add_rms_norm_q8(branch, self.served[-2], v, self.eps)
        return torch.softmax(ops.q8_matmul(q, s, *self.served[-1], dtype=torch.float32), 1)


def main(argv=None):
    from . import configs, synth
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--members", type=int, default=16)
    ap.add_argument("--rows", type=int, default=50_000)
    ap.add_argument("--epochs", type=int, default=3)
    ap.add_argument("--steps", type=int, default=600)
    ap.add_argument("--top", type=int, default=4, help="teacher classes kept of each row")
    a = ap.parse_args(argv)
    cfg = configs.workload("multiclass_lognormal", K=a.members)
    Xh, yh, Xvh, yvh = synth.make_data(cfg, n_train=a.rows, n_val=10_000)
    X, y, Xv, yv = (torch.from_numpy(t).cuda() for t in (Xh, yh, Xvh, yvh))
    pack = tabpack.Pack(cfg).bind()
    t = 0
    for e in range(a.epochs):
        order = synth.epoch_orders_device(cfg, e, a.rows, X.device)
        for s in range(a.rows // cfg["B"]):
            t += 1
            pack.train_step(X, y, order[:, s * cfg["B"]:(s + 1) * cfg["B"]].contiguous(), t)
    idx, teacher = teacher_entries(pack.predict(X, ensemble=True), a.top)
    student = Student(cfg["d_in"], cfg["d_out"])
    loss = student.fit(X, idx, teacher, a.steps).cpu()
    ens, out = pack.predict(Xv, ensemble=True), student.predict(Xv)
    right = [(p.argmax(1) == yv).float().mean().item() for p in (ens, out)]
    agree = (ens.argmax(1) == out.argmax(1)).float().mean().item()
    print(f"distillation loss {loss[:20].mean():.4f} -> {loss[-20:].mean():.4f}; accuracy on {Xv.shape[0]} rows: "
          f"ensemble of {a.members} {right[0]:.4f}, 8-bit student {right[1]:.4f}; the same class on {agree:.4f}")


if __name__ == "__main__":
    main()
