"""One network distilled from an ensemble and served in 8 bits: an example of the operators of ``ops``.

An ensemble of a pack's members (``tabpack``, ``online``) answers with one forward pass per member.  The student is a
single stack of pre-normalised gated blocks over the input features,

    v_0 = [x | embeddings of the categorical columns],
    v_(l+1) = v_l + dropout(W_down (act(W_gate n_l) * (W_up n_l))),   n_l = norm(v_l),
    logits = W_head norm(v_L),

with a root-mean-square or a layer norm, trained on the ensemble's class probabilities (the loss against its k most
likely classes of each row) and served with 8-bit weights and activations, whole numbers or floating point.  Every lookup
and its gradient, product over the blocks, norm, dropout and the loss run in the library's kernels; PyTorch holds the fp32
master weights, applies AdamW to them and does the head's small products in training.

    python -m paper_2607_05380_amd.student            # trains a pack, distils it, serves the student in 8 bits
"""
import argparse
import math

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
                 device="cuda", norm="rms", dropout=0.0, columns=(), d_column=8):
        for name, n in (("d_in", d_in), ("classes", classes), ("blocks", blocks), ("hidden", hidden),
                        ("d_column", d_column)):
            if n < 1:
                raise ops.PackError(f"{name}={n} must be positive")
        if any(n < 1 for n in columns):
            raise ops.PackError(f"columns={tuple(columns)} must be positive")
        if act not in tabpack.ACTIVATIONS:
            raise ops.PackError(f"unknown activation {act!r}")
        if norm not in ("rms", "layer"):
            raise ops.PackError(f"unknown norm {norm!r}")
        if not 0 <= dropout < 1:
            raise ops.PackError(f"dropout={dropout} must lie in [0, 1)")
        if 1 - math.floor(dropout * 65536) / 65536 > (1 + 1 / 256) * (1 - dropout):
            raise ops.PackError(f"dropout={dropout} is too near to 1 for draws of 16 bits (see ops.dropout)")
        if dtype not in (torch.bfloat16, torch.float32):
            raise ops.PackError(f"dtype must be bfloat16 or float32, not {dtype}")
        g = torch.Generator(device=device).manual_seed(seed)
        width = d_in + len(columns) * d_column

        def normal(rows, cols):
            return torch.randn(rows, cols, generator=g, device=device) * cols ** -0.5

        self.act, self.dtype, self.eps, self.classes = act, dtype, eps, classes
        self.codes = "int8"
        self.step = 0  # training steps taken, which number the dropouts' masks
        self.layer, self.p, self.seed = norm == "layer", dropout, seed & 0xFFFFFFFFFFFFFFFF
        self.params = []
        for _ in range(blocks):
            self.params += [torch.ones(width, device=device), normal(2 * hidden, width),
                            normal(width, hidden) * blocks ** -0.5]
        self.params += [torch.ones(width, device=device), normal(classes, width)]
        self.blocks, self.head = blocks, 3 * blocks + 1
        if self.layer:  # the norms' biases
            self.params += [torch.zeros(width, device=device) for _ in range(blocks + 1)]
        # all columns' classes in one table, each column's behind the ones before
        self.columns, self.d_column = tuple(columns), d_column
        self.offsets = torch.tensor([sum(columns[:i]) for i in range(len(columns))], device=device, dtype=torch.int32)
        self.sizes = torch.tensor(list(columns), device=device, dtype=torch.int32)
        if columns:
            self.params.append(torch.randn(sum(columns), d_column, generator=g, device=device))
        self._copies()

    def _copies(self):
        # products read the masters rounded to the student's type; norm weights, biases and the head stay fp32
        self.w = [p if p.dim() == 1 or i == self.head else p.to(self.dtype) for i, p in enumerate(self.params)]
        self.served = self.served_table = None

    # ------------------------------------------------------------- parts
    def _input(self, x, columns, dtype, table):
        """(v_0, indices into the table): the features, then each column's embedding; a class that its column does
        not have (negative, or too large) is missing: zeros."""
        if not self.columns:
            if columns is not None:
                raise ops.PackError("a student built without columns takes none")
            return x.to(dtype), None
        if columns is None or columns.shape != (x.shape[0], len(self.columns)):
            raise ops.PackError(f"columns must hold the classes of {len(self.columns)} columns for each row")
        there = (columns >= 0) & (columns < self.sizes)
        at = torch.where(there, columns.to(torch.int32) + self.offsets, -1).reshape(-1)
        rows = ops.embed(at, table)
        return torch.cat([x.to(dtype), rows.view(x.shape[0], -1)], 1), at

    def _norm(self, i, new, stream):
        """(n, v, statistics) of norm i: n = norm(v), v = new + stream."""
        if not self.layer:
            n, v, rstd = ops.add_rms_norm(new, self.w[3 * i], stream, self.eps)
            return n, v, (rstd,)
        n, v, mean, rstd = ops.add_layer_norm(new, self.w[3 * i], self.w[self.head + 1 + i], stream, self.eps)
        return n, v, (mean, rstd)

    def _norm_backward(self, i, dn, v, stats, dv, grads):
        """The gradient of norm i's v; the weight's and the bias's into grads."""
        if not self.layer:
            dv, grads[3 * i] = ops.rms_norm_backward(dn, v, self.w[3 * i], *stats, dv=dv)
        else:
            dv, grads[3 * i], grads[self.head + 1 + i] = ops.layer_norm_backward(dn, v, self.w[3 * i], *stats, dv=dv)
        return dv

    # ------------------------------------------------------------ training
    def forward(self, x, columns=None, step=None):
        """(logits fp32, what backward needs) of rows x [rows, d_in] and their columns' classes [rows, columns].  step:
        that of a training step, whose masks the dropout then draws (None: no dropout)."""
        p = self.p if step is not None else 0.0
        v, at = self._input(x, columns, self.dtype, self.w[-1])
        keep, branch = [], None
        for b in range(self.blocks):
            n, v, stats = self._norm(b, *((v, None) if branch is None else (branch, v)))
            branch, saved = ops.gated_ff(n, *self.w[3 * b + 1:3 * b + 3], act=self.act, save=True)
            keep.append((n, v, stats, saved))
            if p:  # (added to the stream in the same pass)
                v, branch = ops.dropout(branch, p, self.seed, step, site=b, residual=v), None
        n, v, stats = self._norm(self.blocks, *((v, None) if branch is None else (branch, v)))
        return n.float() @ self.w[self.head].t(), (keep, (n, v, stats), at, p, step)

    def backward(self, dlogits, kept):
        """Gradients of ``params`` (fp32) from those of the logits."""
        keep, (n, v, stats), at, p, step = kept
        grads = [None] * len(self.params)
        dn = (dlogits @ self.w[self.head]).to(self.dtype)
        # the sum's gradient goes to the branch and, unchanged, to the stream it was added to
        dv = self._norm_backward(self.blocks, dn, v, stats, None, grads)
        grads[self.head] = dlogits.t() @ n.float()
        for b in reversed(range(self.blocks)):
            n, v, stats, saved = keep[b]
            dbranch = ops.dropout(dv, p, self.seed, step, site=b) if p else dv
            dn, dwg, dwd = ops.gated_ff_backward(dbranch, n, *self.w[3 * b + 1:3 * b + 3], saved, act=self.act)
            dv = self._norm_backward(b, dn, v, stats, dv, grads)
            grads[3 * b + 1:3 * b + 3] = dwg.float(), dwd.float()
        if at is not None:
            rows = dv[:, dv.shape[1] - len(self.columns) * self.d_column:].reshape(-1, self.d_column)
            grads[-1] = ops.embed_backward(rows, at, self.params[-1].shape[0]).float()
        return grads

    def fit(self, X, idx, teacher, steps, batch=1024, lr=2e-3, temperature=2.0, seed=0, columns=None):
        """Distils: ``steps`` AdamW steps on batches of the rows X (fp32) and their columns' classes with the teacher's
        entries; the mean loss of each step.  Batches follow from ``seed``; the steps go on from those taken before, and with
        them the dropouts' masks."""
        opt = torch.optim.AdamW(self.params, lr=lr, weight_decay=1e-4)
        g = torch.Generator(device=X.device).manual_seed(seed)
        weight = torch.full((batch,), 1.0 / batch, device=X.device)
        losses = []
        for _ in range(steps):
            rows = torch.randint(0, X.shape[0], (batch,), generator=g, device=X.device)
            logits, kept = self.forward(X[rows], None if columns is None else columns[rows], self.step)
            loss, dlogits = ops.distill_topk(logits, idx[rows], teacher[rows], temperature, weight)
            for p, grad in zip(self.params, self.backward(dlogits, kept)):
                p.grad = grad
            opt.step()
            self.step += 1
            self._copies()
            losses.append(loss.sum())
        return torch.stack(losses) if losses else torch.empty(0, device=X.device)

    # ------------------------------------------------------------- serving
    def quantize(self, codes=None):
        """Lays the weights out in 8 bits (once; a later fit() drops them): "int8", whole numbers with a scale per
        output, or "e4m3", floating point with a scale per 128 x 128 (None: those of the last call, int8 at first)."""
        codes = self.codes if codes is None else codes
        if codes not in ("int8", "e4m3"):
            raise ops.PackError(f"unknown codes {codes!r}")
        self.codes = codes
        if codes == "int8":
            self.served = [p if p.dim() == 1 else ops.quantize_rows(p) for p in self.params[:self.head + 1]]
        else:
            self.served = [p if p.dim() == 1 else ops.quantize_tiles(p, gated=i % 3 == 1 and i < self.head)
                           for i, p in enumerate(self.params[:self.head + 1])]
        self.served_table = self.params[-1].to(torch.bfloat16) if self.columns else None
        return self

    def _codes(self, x):
        return ops.quantize_rows(x) if self.codes == "int8" else ops.quantize_blocks(x)

    def _norm_codes(self, i, new, stream):
        """Norm i's output in 8 bits, and v."""
        if self.layer or self.codes != "int8":
            n, v, _ = self._norm(i, new, stream)
            return *self._codes(n), v
        return ops.add_rms_norm_q8(new, self.w[3 * i], stream, self.eps)

    def predict(self, X, columns=None):
        """Class probabilities [rows, classes] of rows X (fp32) and their columns' classes by the 8-bit network."""
        if self.served is None:
            self.quantize()
        matmul = ops.q8_matmul if self.codes == "int8" else ops.f8_matmul
        v, _ = self._input(X, columns, torch.bfloat16, self.served_table)
        branch = None
        for b in range(self.blocks):
            (wg, sg), (wd, sd) = self.served[3 * b + 1:3 * b + 3]
            q, s, v = self._norm_codes(b, *((v, None) if branch is None else (branch, v)))
            q, s = self._codes(matmul(q, s, wg, sg, gate=self.act))
            branch = matmul(q, s, wd, sd)
        q, s, _ = self._norm_codes(self.blocks, branch, v)
        return torch.softmax(matmul(q, s, *self.served[self.head], dtype=torch.float32), 1)


def main(argv=None):
    from . import configs, synth
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--members", type=int, default=16)
    ap.add_argument("--rows", type=int, default=50_000)
    ap.add_argument("--epochs", type=int, default=3)
    ap.add_argument("--steps", type=int, default=600)
    ap.add_argument("--top", type=int, default=4, help="teacher classes kept of each row")
    ap.add_argument("--norm", choices=("rms", "layer"), default="rms")
    ap.add_argument("--dropout", type=float, default=0.0)
    ap.add_argument("--codes", choices=("int8", "e4m3"), default="int8", help="8-bit codes that serve the student")
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
    student = Student(cfg["d_in"], cfg["d_out"], norm=a.norm, dropout=a.dropout)
    loss = student.fit(X, idx, teacher, a.steps).cpu()
    student.quantize(a.codes)
    ens, out = pack.predict(Xv, ensemble=True), student.predict(Xv)
    right = [(p.argmax(1) == yv).float().mean().item() for p in (ens, out)]
    agree = (ens.argmax(1) == out.argmax(1)).float().mean().item()
    print(f"distillation loss {loss[:20].mean():.4f} -> {loss[-20:].mean():.4f}; accuracy on {Xv.shape[0]} rows: "
          f"ensemble of {a.members} {right[0]:.4f}, 8-bit student {right[1]:.4f}; the same class on {agree:.4f}")


if __name__ == "__main__":
    main()
