"""What is timed of the student's further operators: a table's categorical columns or tokens at the network's input
(``embed`` and its gradient), the norm with a mean (``add_layer_norm`` and its gradients), dropout whose mask is
never stored, and products in 8-bit floating point with a scale for each block of 128.

Where ``own`` is false ``run`` computes the same in elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
BLOCK = 128   # depth (and outputs of a weight) that share a scale
TOP = 448.0   # largest e4m3 value
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one row of a table with 16 categorical columns, answered: the launch is what counts
        dict(name="embed_row", op="embed", T=16, V=4000, D=32, spread="columns", long=False, dtype="fp32"),
        # tokens of a batch looked up in a large table
        dict(name="embed_batch", op="embed", T=65_536, V=100_003, D=512, spread="text", long=True, dtype="bf16"),
        # the table's gradient over a batch of text: few tokens are most of it, many rows have none
        dict(name="embed_grad_text", op="embed_grad", T=16_384, V=32_000, D=1024, spread="text", long=True,
             dtype="bf16"),
        # the same of 16 columns of 100 classes and 62,500 rows: each class has thousands
        dict(name="embed_grad_columns", op="embed_grad", T=1_000_000, V=1600, D=32, spread="columns", long=False,
             dtype="fp32"),
        # one row answered: the norm of a sum
        dict(name="layer_norm_row", op="ln_fwd", T=1, D=1024, dtype="bf16"),
        # a small odd table in fp32, forward and gradients
        dict(name="layer_norm_ragged", op="ln_train", T=4095, D=1023, dtype="fp32"),
        # a training step of one norm over a whole epoch's slice of rows
        dict(name="layer_norm_train", op="ln_train", T=65_536, D=1024, dtype="bf16"),
        # a small table's branch, forward and backward
        dict(name="dropout_ragged", op="dropout", T=300, D=301, p=0.1, dtype="fp32"),
        # a wide branch onto its stream, forward and backward
        dict(name="dropout_train", op="dropout", T=65_536, D=1024, p=0.15, dtype="bf16"),
        # one row through the gated projections: its codes, then the weights' bytes
        dict(name="f8_row", op="f8_linear", M=1, K=1024, N=4096, gate="silu", bias=False, dtype="bf16"),
        # a batch through a down projection, from bf16 rows
        dict(name="f8_batch", op="f8_linear", M=2048, K=2048, N=1024, gate="", bias=True, dtype="bf16"),
        # all validation rows through the gated projections, an odd number of them, from codes
        dict(name="f8_rows", op="f8", M=20_011, K=1024, N=4096, gate="silu", bias=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: as often a multiple of 64 as any number at all."""
    w = _log(rng, lo, hi)
    return max(64, (w + 32) // 64 * 64) if rng.random() < 0.5 else w


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "ln_fwd", "ln_train", "dropout", "f8", "f8_linear",
                     "f8_weights"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    e = 4 if dtype == "fp32" else 2
    if op in ("embed", "embed_grad"):
        c = dict(op=op, T=_log(rng, 1, 1_000_000), V=_log(rng, 2, 200_000), D=_width(rng, 4, 2048),
                 spread=rng.choice(["text", "columns"]), long=rng.random() < 0.5, dtype=dtype)
        c["T"] = max(1, min(c["T"], (1 << 26) // (c["D"] * e)))
        c["V"] = max(2, min(c["V"], (1 << 26) // (c["D"] * e)))
        return c
    if op in ("ln_fwd", "ln_train", "dropout"):
        c = dict(op=op, T=_log(rng, 1, 65_536), D=_width(rng, 8, 8192), dtype=dtype)
        c["T"] = max(1, min(c["T"], (1 << 27) // (c["D"] * e)))
        if op == "dropout":
            c["p"] = round(rng.choice([0.0, rng.uniform(0.01, 0.9)]), 3)
        return c
    c = dict(op=op, M=_log(rng, 1, 20_011), K=_width(rng, 8, 4096), N=_width(rng, 8, 4096),
             gate=rng.choice(["", "", "silu", "gelu"]), bias=rng.random() < 0.5, dtype=dtype)
    c["M"] = max(1, min(c["M"], int(1.6e11 // (2 * c["K"] * c["N"] * (2 if c["gate"] else 1)))))
    return c


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed((0x9E3779B97F4A7C15 * (int(seed) + 1)) % (1 << 62))


def _normal(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device=DEV) * std


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV, dtype=torch.float64)


def _bytes(case):
    return 4 if case["dtype"] == "fp32" else 2


def _tokens(case, g):
    """Indices into the table: a text's tokens by rank, or 16 columns of classes, the first ones more often; one in
    fifty is missing (-1)."""
    T, V = case["T"], case["V"]
    if case["spread"] == "text":
        rank = (torch.exp(_uniform(g, T) * math.log(V + 1)) - 1).long().clamp(0, V - 1)
        idx = torch.randperm(V, generator=g, device=DEV)[rank]
    else:
        columns = min(16, V)
        each = V // columns
        idx = (torch.arange(T, device=DEV) % columns) * each + (_uniform(g, T).square() * each).long().clamp(0, each - 1)
    idx = torch.where(_uniform(g, T) < 0.02, -1, idx)
    return idx if case["long"] else idx.to(torch.int32)


def _tiles(w, parts):
    """A weight [parts n, K] in 8 bits by tiles of 128 x 128 of each part, in 32 bits: codes and scales."""
    n, K = w.shape[0] // parts, w.shape[1]
    nb, kb = -(-n // BLOCK), -(-K // BLOCK)
    full = torch.zeros(parts, nb * BLOCK, kb * BLOCK, device=w.device)
    full[:, :n, :K] = w.float().view(parts, n, K)
    t = full.view(parts * nb, BLOCK, kb, BLOCK)
    a = t.abs().amax((1, 3), keepdim=True)
    f = torch.where(a > 0, torch.div(torch.full_like(a, TOP), a), torch.zeros_like(a))
    codes = (t * f).to(torch.float8_e4m3fn).view(torch.uint8).view(parts, nb * BLOCK, kb * BLOCK)[:, :n, :K]
    return codes.reshape(parts * n, K).view(torch.float8_e4m3fn), (a / TOP).view(parts * nb, kb)


def _blocks(x):
    """Rows in 8 bits by blocks of 128 columns, in 32 bits: codes [rows, K], scales [blocks, rows]."""
    M, K = x.shape
    kb = -(-K // BLOCK)
    full = torch.zeros(M, kb * BLOCK, device=x.device)
    full[:, :K] = x.float()
    t = full.view(M, kb, BLOCK)
    a = t.abs().amax(2, keepdim=True)
    f = torch.where(a > 0, torch.div(torch.full_like(a, TOP), a), torch.zeros_like(a))
    codes = (t * f).to(torch.float8_e4m3fn).view(torch.uint8).view(M, kb * BLOCK)[:, :K]
    return codes.contiguous().view(torch.float8_e4m3fn), (a / TOP)[:, :, 0].t().contiguous()


def prepare(case, seed):
    g = _generator(seed)
    op, dt = case["op"], DTYPES[case["dtype"]]
    s = dict(case=case)
    if op in ("embed", "embed_grad"):
        s["idx"] = _tokens(case, g)
        if op == "embed":
            s.update(table=_normal(g, case["V"], case["D"], std=case["D"] ** -0.5).to(dt), scale=case["D"] ** 0.5)
        else:
            s.update(dy=_normal(g, case["T"], case["D"], std=1e-2).to(dt), scale=case["D"] ** 0.5)
    elif op in ("ln_fwd", "ln_train"):
        # a residual stream with a mean and a few loud channels, the branch added to it, trained weights
        T, D = case["T"], case["D"]
        loud = 1 + 8 * (torch.rand(D, generator=g, device=DEV) < 0.01)
        s.update(x=_normal(g, T, D, std=0.5).to(dt), r=(_normal(g, T, D) * loud + 0.7).to(dt),
                 w=1 + _normal(g, D, std=0.1), b=_normal(g, D, std=0.1))
        if op == "ln_train":
            s.update(dy=_normal(g, T, D, std=1e-2).to(dt), dv=_normal(g, T, D, std=1e-2).to(dt))
    elif op == "dropout":
        T, D = case["T"], case["D"]
        s.update(x=_normal(g, T, D).to(dt), r=_normal(g, T, D).to(dt), dy=_normal(g, T, D, std=1e-2).to(dt),
                 seed=0x0123_4567_89AB_CDEF ^ int(seed), step=1 + int(seed) % 100_000, site=3)
    else:
        M, K, N, parts = case["M"], case["K"], case["N"], 2 if case["gate"] else 1
        w = _normal(g, parts * N, K, std=K ** -0.5)
        if op == "f8_weights":
            s.update(w=w.to(dt), parts=parts)
            return s
        # activations with a few loud channels; the weight laid out when the network was loaded
        loud = 1 + 15 * (torch.rand(K, generator=g, device=DEV) < 0.01)
        x = (_normal(g, M, K) * loud).to(dt)
        qw, sw = _tiles(w, parts)
        s.update(qw=qw, sw=sw, b=_normal(g, parts * N, std=0.1) if case["bias"] else None)
        if op == "f8":
            s["qx"], s["sx"] = _blocks(x)
        else:
            s["x"] = x
    return s


# --------------------------------------------------------------- plain form
def _act(a, g):
    if a == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))


def _words(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 of the counters c0 .. c3 (int64 tensors of 32-bit values)."""
    low = 0xFFFFFFFF
    for r in range(10):  # the generator's rounds
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32 & low) ^ c1 ^ (k0 + r * 0x9E3779B9 & low), p1 & low,
                          (p0 >> 32 & low) ^ c3 ^ (k1 + r * 0xBB67AE85 & low), p0 & low)
    return c0, c1, c2, c3


def _keep(rows, cols, p, seed, step, site):
    """Which elements dropout keeps: 16-bit draws of Philox blocks of 8 columns against floor(p 2^16)."""
    r = torch.arange(rows, device=DEV)[:, None]
    c = torch.arange(-(-cols // 8), device=DEV)[None, :]
    zero = torch.zeros_like(r + c)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF ^ 4 << 28
    w = torch.stack(_words(zero + c, zero + r, zero + site, zero + step, k0, k1), 2)
    h = torch.stack([w & 0xFFFF, w >> 16], 3).view(rows, -1)[:, :cols]
    return h >= math.floor(p * 65536)


def _plain(case, s):
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op == "embed":
        idx = s["idx"].long()
        y = s["table"][idx.clamp(min=0)].float() * s["scale"]
        return torch.where((idx >= 0)[:, None], y, torch.zeros_like(y)).to(dt)
    if op == "embed_grad":
        idx = s["idx"].long()
        total = torch.zeros(case["V"] + 1, case["D"], device=DEV)
        total.index_add_(0, torch.where(idx >= 0, idx, case["V"]), s["dy"].float())
        return (total[:-1] * s["scale"]).to(dt)
    if op in ("ln_fwd", "ln_train"):
        v = s["x"].float() + s["r"].float()
        mean = v.mean(1, keepdim=True)
        rho = 1 / torch.sqrt((v - mean).square().mean(1, keepdim=True) + EPS)
        out = dict(sum=v.to(dt), y=((v - mean) * rho * s["w"] + s["b"]).to(dt), mean=mean[:, 0], rstd=rho[:, 0])
        if op == "ln_train":
            n = (out["sum"].float() - mean) * rho
            dy = s["dy"].float()
            g = dy * s["w"]
            dx = rho * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) + s["dv"].float()
            out.update(dx=dx.to(dt), dw=(dy * n).sum(0), db=dy.sum(0))
        return out
    if op == "dropout":
        keep = _keep(case["T"], case["D"], case["p"], s["seed"], s["step"], s["site"])
        zero, f = torch.zeros((), device=DEV), 1 / (1 - case["p"])
        return dict(y=(s["r"].float() + torch.where(keep, s["x"].float() * f, zero)).to(dt),
                    dx=torch.where(keep, s["dy"].float() * f, zero).to(dt))
    if op == "f8_weights":
        q, scale = _tiles(s["w"], s["parts"])
        return _tile_values(q, scale, s["parts"])
    qx, sx = _blocks(s["x"]) if op == "f8_linear" else (s["qx"], s["sx"])
    x = qx.float() * sx.t().repeat_interleave(BLOCK, 1)[:, :case["K"]]
    out = x @ _tile_values(s["qw"], s["sw"], 2 if case["gate"] else 1).t()
    if s["b"] is not None:
        out = out + s["b"]
    if case["gate"]:
        out = _act(case["gate"], out[:, :case["N"]]) * out[:, case["N"]:]
    return out.to(dt)


def _tile_values(q, scale, parts):
    """What the codes of a weight stand for."""
    n, K = q.shape[0] // parts, q.shape[1]
    each = scale.view(parts, -1, scale.shape[1]).repeat_interleave(BLOCK, 1)[:, :n].repeat_interleave(BLOCK, 2)
    return q.float() * each[:, :, :K].reshape(parts * n, K)


# -------------------------------------------------------- the framework's own
def _own(case, s):
    from paper_2607_05380_amd import ops
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op == "embed":
        return ops.embed(s["idx"], s["table"], scale=s["scale"])
    if op == "embed_grad":
        return ops.embed_backward(s["dy"], s["idx"], case["V"], scale=s["scale"])
    if op in ("ln_fwd", "ln_train"):
        y, v, mean, rstd = ops.add_layer_norm(s["x"], s["w"], s["b"], residual=s["r"], eps=EPS)
        out = dict(sum=v, y=y, mean=mean, rstd=rstd)
        if op == "ln_train":
            dx, dw, db = ops.layer_norm_backward(s["dy"], v, s["w"], mean, rstd, dv=s["dv"])
            out.update(dx=dx, dw=dw, db=db)
        return out
    if op == "dropout":
        y = ops.dropout(s["x"], case["p"], s["seed"], s["step"], site=s["site"], residual=s["r"])
        return dict(y=y, dx=ops.dropout(s["dy"], case["p"], s["seed"], s["step"], site=s["site"]))
    if op == "f8_weights":
        q, scale = ops.quantize_tiles(s["w"], gated=s["parts"] == 2)
        return _tile_values(q, scale, s["parts"])
    qx, sx = ops.quantize_blocks(s["x"]) if op == "f8_linear" else (s["qx"], s["sx"])
    return ops.f8_matmul(qx, sx, s["qw"], s["sw"], bias=s["b"], gate=case["gate"] or None, dtype=dt)


def run(state):
    return (_own if own else _plain)(state["case"], state)


# ------------------------------------------------------------------ in 64 bits
def _philox(counters, key):
    """Philox4x32-10 on the host: counters uint64 [4, n] of 32-bit words."""
    import numpy as np
    a, b, c, d = counters
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for r in range(10):
        x, z = np.uint64(0xD2511F53) * a, np.uint64(0xCD9E8D57) * c
        a = (z >> shift) ^ b ^ np.uint64((key[0] + r * 0x9E3779B9) % 2 ** 32)
        c = (x >> shift) ^ d ^ np.uint64((key[1] + r * 0xBB67AE85) % 2 ** 32)
        b, d = z & low, x & low
    return a, b, c, d


def _mask64(rows, cols, p, seed, step, site):
    import numpy as np
    groups = (cols + 7) // 8
    at = np.arange(rows * groups, dtype=np.uint64)
    counters = (at % np.uint64(groups), at // np.uint64(groups), np.full_like(at, site), np.full_like(at, step))
    words = _philox(counters, (seed % 2 ** 32, (seed >> 32) % 2 ** 32 ^ 0x40000000))
    keep = np.empty((rows * groups, 8), dtype=bool)
    for c in range(8):  # column c of a group: half c % 2 of word c / 2
        keep[:, c] = (words[c // 2] >> np.uint64(16 * (c % 2))) % np.uint64(65536) >= int(p * 65536)
    return torch.from_numpy(keep.reshape(rows, groups * 8)[:, :cols]).to(DEV)


def _e4m3(v):
    """The nearest e4m3 value, ties to even: steps of 2^-3 of the leading bit's value, 2^-9 below 2^-6."""
    exponent = torch.frexp(v).exponent.clamp(min=-5) - 1
    step = torch.ldexp(torch.ones_like(v), exponent - 3)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _eight(x, rows):
    """Values that x's codes stand for, with a scale for each block of ``rows`` x 128."""
    nr, nc = (x.shape[0] + rows - 1) // rows, (x.shape[1] + BLOCK - 1) // BLOCK
    t = torch.nn.functional.pad(x, (0, nc * BLOCK - x.shape[1], 0, nr * rows - x.shape[0]))
    t = t.reshape(nr, rows, nc, BLOCK)
    scale = t.abs().amax(dim=(1, 3), keepdim=True) / TOP
    t = torch.where(scale > 0, _e4m3(t / scale.clamp(min=1e-300)) * scale, 0.0)
    return t.reshape(nr * rows, nc * BLOCK)[:x.shape[0], :x.shape[1]]


def exact(case, seed):
    """The operators' definitions in 64 bits, gradients by differentiating them where that is the shorter way."""
    given = prepare(case, seed)
    op = case["op"]
    if op in ("embed", "embed_grad"):
        there = given["idx"] >= 0
        if op == "embed":
            out = torch.zeros(case["T"], case["D"], dtype=torch.float64, device=DEV)
            out[there] = given["table"].double().index_select(0, given["idx"][there].long()) * given["scale"]
            return out
        order = torch.argsort(given["idx"][there].long(), stable=True)
        rows = given["idx"][there].long()[order]
        out = torch.zeros(case["V"], case["D"], dtype=torch.float64, device=DEV)
        out.index_put_((rows,), given["dy"][there][order].double() * given["scale"], accumulate=True)
        return out
    if op in ("ln_fwd", "ln_train"):
        x, r, w, b = (given[k].double() for k in "xrwb")
        v = x + r
        mean, var = v.mean(1), v.var(1, unbiased=False)
        rstd = (var + EPS).pow(-0.5)
        out = dict(sum=v, y=torch.nn.functional.layer_norm(v, (case["D"],), w, b, EPS), mean=mean, rstd=rstd)
        if op == "ln_train":
            # from the sum as it was stored, with the statistics of the forward pass: n = (v - mean) rstd is held to
            # have mean 0 and mean square 1 in the gradient
            stored, dy = v.to(DTYPES[case["dtype"]]).double(), given["dy"].double()
            n = (stored - mean[:, None]) * rstd[:, None]
            g = dy * w
            along = torch.einsum("td,td->t", g, n) / case["D"]
            dx = (g - (g.sum(1) / case["D"])[:, None] - n * along[:, None]) * rstd[:, None] + given["dv"].double()
            out.update(dx=dx, dw=torch.einsum("td,td->d", dy, n), db=dy.sum(0))
        return out
    if op == "dropout":
        keep = _mask64(case["T"], case["D"], case["p"], given["seed"], given["step"], given["site"]).double()
        return dict(y=given["r"].double() + given["x"].double() * keep / (1 - case["p"]),
                    dx=given["dy"].double() * keep / (1 - case["p"]))
    if op == "f8_weights":
        return torch.cat([_eight(w, BLOCK) for w in given["w"].double().chunk(given["parts"])])
    sx = given["sx"].double() if op == "f8" else None
    x = _eight(given["x"].double(), 1) if op == "f8_linear" else given["qx"].double() * torch.stack(
        [sx[k // BLOCK] for k in range(case["K"])], 1)
    halves = []
    for q, sw in zip(given["qw"].double().chunk(2 if case["gate"] else 1),
                     given["sw"].double().chunk(2 if case["gate"] else 1)):
        at_n = torch.arange(case["N"], device=DEV) // BLOCK
        at_k = torch.arange(case["K"], device=DEV) // BLOCK
        halves.append(torch.mm(x, (q * sw[at_n][:, at_k]).t()))
    out = torch.cat(halves, 1)
    out = out if given["b"] is None else out + given["b"].double()
    if case["gate"]:
        gate, up = out.split(case["N"], 1)
        gelu = torch.nn.functional.gelu
        return (gate * torch.sigmoid(gate) if case["gate"] == "silu" else gelu(gate)) * up
    return out


# ------------------------------------------------------------------------ work
def work(case):
    """Every input read once and every output written once; the operations of the definition."""
    op, e = case["op"], _bytes(case)
    if op in ("embed", "embed_grad"):
        T, V, D, i = case["T"], case["V"], case["D"], 8 if case["long"] else 4
        rows = min(T, V) if op == "embed" else V
        return dict(bytes=T * i + T * D * e + rows * D * e, flops=T * D)
    if op in ("ln_fwd", "ln_train"):
        T, D = case["T"], case["D"]
        if op == "ln_fwd":
            return dict(bytes=4 * T * D * e + 8 * D + 8 * T, flops=9 * T * D)
        return dict(bytes=7 * T * D * e + 16 * D + 8 * T, flops=24 * T * D)
    if op == "dropout":
        # (a generator's block, some 80 operations on 32-bit words, serves 8 elements, both ways)
        return dict(bytes=5 * case["T"] * case["D"] * e, flops=24 * case["T"] * case["D"])
    M, K, N, w = case["M"], case["K"], case["N"], 2 if case["gate"] else 1
    weights = w * N * K + 4 * (w * (-(-N // BLOCK)) * (-(-K // BLOCK)))
    if op == "f8_weights":
        return dict(bytes=w * N * K * (e + 4), flops=3 * w * N * K)
    x = M * K * (e if op == "f8_linear" else 1) + (4 * M * (-(-K // BLOCK)) if op == "f8" else 0)
    return dict(bytes=x + weights + e * M * N + (4 * w * N if case["bias"] else 0), flops=2 * w * M * N * K)
