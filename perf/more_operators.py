"""What surrounds a learned encoder's layers in training, as cases that can be
timed and checked: the embedding table (gpic_embedding) and its gradient, the
layer norm (gpic_layer_norm) and its gradients, dropout with a mask that is
never stored (gpic_dropout), and the cross entropy over a vocabulary whose
logits are never kept (gpic_cross_entropy) with its gradients.

listed() gives the cases, draw(rng) one more of the same ranges, prepare()
what a program holds before the call, run() one pass (the plain form in
elementary torch operations, or with own = True the package's entry points),
work() what a pass cannot do without, and exact() the outputs in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

DEV = "cuda"
own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
IGNORED = -100             # the target of a padded row


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the probability of one token among a vocabulary, as a service that
        # scores tokens one at a time asks for it: the weights are read once
        {"name": "loss_point_bf16", "kind": "loss", "n": 1, "k": 2048, "v": 32000,
         "dtype": "bf16", "bias": False, "padded": False, "train": False},
        # a small odd batch's training pass, where launches count
        {"name": "loss_small_f32", "kind": "loss", "n": 52, "k": 512, "v": 1013,
         "dtype": "f32", "bias": True, "padded": True, "train": True},
        # an odd float32 batch over an odd vocabulary
        {"name": "loss_train_f32", "kind": "loss", "n": 1003, "k": 700, "v": 10007,
         "dtype": "f32", "bias": True, "padded": True, "train": True},
        # a large training batch, a sixteenth of its rows padding
        {"name": "loss_train_bf16", "kind": "loss", "n": 8192, "k": 2048, "v": 50000,
         "dtype": "bf16", "bias": False, "padded": True, "train": True},
        # one point through a norm: latency
        {"name": "norm_point_f16", "kind": "norm", "n": 1, "k": 2048, "dtype": "f16",
         "train": False, "view": False},
        # an odd float32 batch inside a wider table, and back
        {"name": "norm_train_f32", "kind": "norm", "n": 10007, "k": 1000, "dtype": "f32",
         "train": True, "view": True},
        # the norm of a large batch, and back
        {"name": "norm_train_bf16", "kind": "norm", "n": 16384, "k": 2048, "dtype": "bf16",
         "train": True, "view": False},
        # a sentence's rows of a table
        {"name": "embed_few_f16", "kind": "embed", "n": 17, "k": 2048, "v": 32000,
         "dtype": "f16", "ids": "zipf", "padded": False, "train": False},
        # a small odd batch, and back
        {"name": "embed_small_f32", "kind": "embed", "n": 1003, "k": 300, "v": 777,
         "dtype": "f32", "ids": "uniform", "padded": True, "train": True},
        # a large batch whose tokens are as frequent as words are, and back
        {"name": "embed_train_bf16", "kind": "embed", "n": 32768, "k": 1024, "v": 50000,
         "dtype": "bf16", "ids": "zipf", "padded": True, "train": True},
        # dropout before a residual at odd sizes, and back
        {"name": "dropout_f32", "kind": "dropout", "n": 1003, "k": 777, "dtype": "f32",
         "p": 0.1, "residual": True, "view": True},
        # the same over a large batch's hidden values
        {"name": "dropout_bf16", "kind": "dropout", "n": 16384, "k": 4096, "dtype": "bf16",
         "p": 0.1, "residual": True, "view": False},
    ]


def _log(rng, lo, hi):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = 64 if v > 128 and rng.random() < 0.5 else 1
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["loss", "loss", "loss", "norm", "norm", "embed", "embed", "dropout"])
    while True:
        c = {"kind": kind, "n": _log(rng, 1, 32768), "k": _log(rng, 8, 4096),
             "dtype": rng.choice(["f32", "bf16", "bf16", "f16"])}
        if kind == "loss":
            c.update(v=_log(rng, 8, 65536), bias=rng.random() < 0.5, padded=rng.random() < 0.5,
                     train=rng.random() < 0.6)
        elif kind == "norm":
            c.update(train=rng.random() < 0.6, view=rng.random() < 0.3)
        elif kind == "embed":
            c.update(v=_log(rng, 8, 65536), ids=rng.choice(["zipf", "zipf", "uniform", "one"]),
                     padded=rng.random() < 0.5, train=rng.random() < 0.6)
        else:
            c.update(p=rng.choice([0.0, 0.1, 0.1, 0.3, 0.5, 0.9]), residual=rng.random() < 0.5,
                     view=rng.random() < 0.3)
        # float32 counts as three products of 16-bit parts
        w = work(c)
        if w["flops"] * (3 if c["dtype"] == "f32" else 1) <= 5e12 and w["bytes"] <= 1e9:
            return c


# ----------------------------------------------------------------- inputs
def _ids(case, n, v, gen):
    """Token numbers of a distribution: as frequent as words are (the
    frequency falls as 1 / rank), uniform, or all the same; a sixteenth of
    them padding."""
    u = torch.rand(n, device=DEV, dtype=torch.float64, generator=gen)
    how = case.get("ids", "zipf")
    if how == "zipf":
        t = torch.exp(u * math.log(v + 1.0)).long() - 1
    elif how == "uniform":
        t = (u * v).long()
    else:
        t = torch.full((n,), v // 2, device=DEV, dtype=torch.int64)
    t = t.clamp(0, v - 1)
    if case["padded"]:
        pad = torch.rand(n, device=DEV, generator=gen) < 1.0 / 16.0
        t = torch.where(pad, torch.full_like(t, IGNORED), t)
    return t


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    T = DTYPES[case["dtype"]]
    kind, n, k = case["kind"], case["n"], case["k"]

    def randn(*shape, scale=1.0):
        x = torch.randn(shape, device=DEV, dtype=torch.float32, generator=gen)
        return (x * scale).to(T)

    def table(rows, cols, scale=1.0):
        """Columns 8 .. 8 + cols of a wider table, or a table."""
        if case.get("view"):
            return randn(rows, cols + 24, scale=scale)[:, 8:8 + cols]
        return randn(rows, cols, scale=scale)

    st = {"case": case}
    if kind == "loss":
        v = case["v"]
        st["W"] = randn(v, k, scale=3.0 / math.sqrt(k))
        st["targets"] = _ids(case, n, v, gen)
        # half of the rows know their token: logits of about 18 for it, 3 around
        X = torch.randn((n, k), device=DEV, dtype=torch.float32, generator=gen)
        knows = torch.rand((n, 1), device=DEV, generator=gen) < 0.5
        w = st["W"][st["targets"].clamp(min=0)].float()
        w = w * (6.0 / w.square().sum(1, keepdim=True).sqrt().clamp(min=1e-6))
        st["X"] = (X + torch.where(knows, w, torch.zeros_like(w))).to(T)
        st["bias"] = randn(v, scale=0.5) if case["bias"] else None
        if case["train"]:
            # the mean over the rows that count; float16 with the usual scaled loss
            counts = st["targets"] >= 0
            scale = (1024.0 if case["dtype"] == "f16" else 1.0) / max(1, int(counts.sum()))
            st["dloss"] = torch.where(counts, scale, 0.0).float()
    elif kind == "norm":
        size = torch.exp(torch.randn((n, 1), device=DEV, generator=gen))
        shift = 0.5 * torch.randn((n, 1), device=DEV, generator=gen)
        st["X"] = table(n, k)
        st["X"].copy_(((st["X"].float() + shift) * size).to(T))
        st["weight"] = 1.0 + randn(k, scale=0.1)
        st["bias"] = randn(k, scale=0.1)
        if case["train"]:
            st["dY"] = randn(n, k, scale=0.01)
    elif kind == "embed":
        st["T"] = randn(case["v"], k, scale=1.0 / math.sqrt(k))
        st["ids"] = _ids(case, n, case["v"], gen)
        st["scale"] = math.sqrt(k)
        if case["train"]:
            st["dY"] = randn(n, k, scale=0.01)
    else:
        st["X"] = table(n, k)
        st["R"] = randn(n, k) if case["residual"] else None
        st["dY"] = randn(n, k, scale=0.01)
        st["seed"] = int(torch.randint(1 << 62, (1,), device=DEV, generator=gen))
        st["offset"] = int(seed) % 1000
    return st


# ------------------------------------------------------------- plain forms
def _plain_loss(st):
    c = st["case"]
    T = DTYPES[c["dtype"]]
    X, W, t = st["X"].float(), st["W"].float(), st["targets"]
    Z = X @ W.t()
    if st["bias"] is not None:
        Z = Z + st["bias"].float()
    counts = t >= 0
    row = torch.arange(c["n"], device=DEV)
    most = Z.max(1).values
    lse = most + torch.exp(Z - most[:, None]).sum(1).log()
    at = t.clamp(min=0)
    loss = torch.where(counts, lse - Z[row, at], torch.zeros_like(lse))
    if not c["train"]:
        return {"loss": loss}
    dZ = torch.exp(Z - lse[:, None])
    dZ[row, at] -= 1.0
    dZ = torch.where(counts[:, None], dZ * st["dloss"][:, None], torch.zeros_like(dZ))
    out = {"loss": loss, "lse": lse, "dX": (dZ @ W).to(T), "dW": (dZ.t() @ X).to(T)}
    if st["bias"] is not None:
        out["db"] = dZ.sum(0).to(T)
    return out


def _plain_norm(st):
    c = st["case"]
    T = DTYPES[c["dtype"]]
    X, w = st["X"].float(), st["weight"].float()
    centred = X - X.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(centred.square().mean(1, keepdim=True) + EPS)
    H = centred * r
    out = {"Y": (H * w + st["bias"].float()).to(T)}
    if c["train"]:
        dY = st["dY"].float()
        G = dY * w
        dX = r * (G - G.mean(1, keepdim=True) - H * (G * H).mean(1, keepdim=True))
        out.update(dX=dX.to(T), dW=(dY * H).sum(0).to(T), db=dY.sum(0).to(T))
    return out


def _plain_embed(st):
    c = st["case"]
    T = DTYPES[c["dtype"]]
    ids = st["ids"]
    counts = (ids >= 0)[:, None]
    at = ids.clamp(min=0)
    Y = st["T"][at].float() * st["scale"]
    out = {"Y": torch.where(counts, Y, torch.zeros_like(Y)).to(T)}
    if c["train"]:
        # a frequent token sums thousands of rows
        d = torch.where(counts, st["dY"].double(), 0.0)
        dT = torch.zeros((c["v"], c["k"]), device=DEV, dtype=torch.float64)
        dT.index_add_(0, at, d)
        out["dT"] = (dT * st["scale"]).float().to(T)
    return out


def _philox_keep(total, p, seed, offset):
    """Which of `total` values stay: the 16 bits that Philox4x32-10 (Salmon,
    Moraes, Dror and Shaw, 2011) gives a value are compared with p.  Value i
    takes half i % 8 of the block with counter (i / 8, offset) under the key
    `seed`.  32-bit words in int64."""
    blocks = (total + 7) // 8
    i = torch.arange(blocks, device=DEV, dtype=torch.int64)
    low = 0xffffffff
    c0, c1 = i & low, i >> 32
    c2 = torch.full_like(i, offset & low)
    c3 = torch.full_like(i, (offset >> 32) & low)
    k0, k1 = seed & low, (seed >> 32) & low

    def multiply(m, x):
        """(high, low) words of m x, through the halves of x."""
        a = (x & 0xffff) * m
        b = (x >> 16) * m + (a >> 16)
        return b >> 16, ((b & 0xffff) << 16) | (a & 0xffff)

    for _ in range(10):
        h0, l0 = multiply(0xD2511F53, c0)
        h1, l1 = multiply(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    halves = torch.stack([words & 0xffff, words >> 16], 2).reshape(-1)[:total]
    return halves >= _limit(p)


def _limit(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _plain_dropout(st):
    c = st["case"]
    T = DTYPES[c["dtype"]]
    n, k = c["n"], c["k"]
    keep = _philox_keep(n * k, c["p"], st["seed"], st["offset"]).reshape(n, k)
    scale = 65536.0 / (65536 - _limit(c["p"]))
    X, dY = st["X"].float(), st["dY"].float()
    Y = torch.where(keep, X * scale, torch.zeros_like(X))
    if st["R"] is not None:
        Y = Y + st["R"].float()
    return {"Y": Y.to(T), "dX": torch.where(keep, dY * scale, torch.zeros_like(dY)).to(T)}


PLAIN = {"loss": _plain_loss, "norm": _plain_norm, "embed": _plain_embed,
         "dropout": _plain_dropout}


# -------------------------------------------------------------------- run
def run(st):
    c = st["case"]
    kind = c["kind"]
    if not own:
        return PLAIN[kind](st)
    import paper_1604_02700_amd as g
    if kind == "loss":
        if not c["train"]:
            return {"loss": g.gpic_cross_entropy(st["X"], st["W"], st["targets"], st["bias"])}
        loss, lse = g.gpic_cross_entropy(st["X"], st["W"], st["targets"], st["bias"],
                                         want_lse=True)
        gr = g.gpic_cross_entropy_backward(st["dloss"], st["X"], st["W"], st["targets"], loss,
                                           lse, st["bias"], want_bias=st["bias"] is not None)
        out = {"loss": loss, "lse": lse, "dX": gr.dX, "dW": gr.dW}
        if st["bias"] is not None:
            out["db"] = gr.db
        return out
    if kind == "norm":
        if not c["train"]:
            return {"Y": g.gpic_layer_norm(st["X"], st["weight"], st["bias"], EPS)}
        Y, stats = g.gpic_layer_norm(st["X"], st["weight"], st["bias"], EPS, want_stats=True)
        gr = g.gpic_layer_norm_backward(st["dY"], st["X"], st["weight"], stats)
        return {"Y": Y, "dX": gr.dX, "dW": gr.dW, "db": gr.db}
    if kind == "embed":
        out = {"Y": g.gpic_embedding(st["ids"], st["T"], st["scale"])}
        if c["train"]:
            out["dT"] = g.gpic_embedding_backward(st["dY"], st["ids"], c["v"], st["scale"])
        return out
    return {"Y": g.gpic_dropout(st["X"], c["p"], st["seed"], st["offset"], residual=st["R"]),
            "dX": g.gpic_dropout(st["dY"], c["p"], st["seed"], st["offset"])}


# ------------------------------------------------------------------- work
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    kind, n, k = case["kind"], case["n"], case["k"]
    if kind == "loss":
        v = case["v"]
        b = v if case["bias"] else 0
        values = n * k + v * k + b                 # X, W, bias
        other = 8 * n + 4 * n                      # targets, the loss
        flops = 2.0 * n * k * v
        if case["train"]:                          # dX, dW, db; dloss and lse
            values *= 2
            other += 8 * n
            flops *= 3                             # the logits, dX, dW
        return {"bytes": float(values * size + other), "flops": flops}
    if kind == "norm":
        values, flops = 2 * n * k + 2 * k, 8.0 * n * k
        if case["train"]:                          # dY; dX and the weights' gradients
            values += 2 * n * k + 2 * k
            flops += 12.0 * n * k
        return {"bytes": float(values * size), "flops": flops}
    if kind == "embed":
        rows = 1 if case["ids"] == "one" else min(n, case["v"])
        values, flops = rows * k + n * k, 1.0 * n * k
        if case["train"]:                          # dY; dT
            values += n * k + case["v"] * k
            flops += 1.0 * n * k
        return {"bytes": float(values * size + 8 * n), "flops": flops}
    # X, the residual, Y; dY, dX; a block of 8 random halves is 10 rounds of 6
    # operations, of which the second call makes as many
    values = (5 if case["residual"] else 4) * n * k
    return {"bytes": float(values * size), "flops": 2.0 * n * k * (60 / 8 + 3)}


# ------------------------------------------------------------------ exact
def _numpy_keep(total, p, seed, offset):
    """The kept values again, in numpy's 64-bit words, a piece at a time."""
    keep = np.empty((total + 7) // 8 * 8, dtype=bool)
    word, high = np.uint64(0xffffffff), np.uint64(32)
    for first in range(0, keep.size // 8, 1 << 20):
        x = np.arange(first, min(first + (1 << 20), keep.size // 8), dtype=np.uint64)
        ctr = [x & word, x >> high, np.full_like(x, offset & 0xffffffff),
               np.full_like(x, offset >> 32)]
        key = [seed & 0xffffffff, seed >> 32]
        for _ in range(10):
            a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
            ctr = [(b >> high) ^ ctr[1] ^ np.uint64(key[0]), b & word,
                   (a >> high) ^ ctr[3] ^ np.uint64(key[1]), a & word]
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        packed = np.stack([c.astype("<u4") for c in ctr], axis=1)
        bits = packed.view("<u2").reshape(-1)
        keep[8 * first:8 * first + bits.size] = bits.astype(np.int64) >= round(p * 65536)
    return torch.from_numpy(keep[:total]).to(DEV)


def exact(case, seed):
    st = prepare(case, seed)
    kind, n, k = case["kind"], case["n"], case["k"]
    D = {x: y.double() if isinstance(y, torch.Tensor) and y.is_floating_point() else y
         for x, y in st.items()}
    del st
    if kind == "loss":
        t = D["targets"]
        real = t.ge(0)
        Z = D["X"].mm(D["W"].t())
        if D["bias"] is not None:
            Z += D["bias"]
        lse = torch.logsumexp(Z, dim=1)
        picked = Z.gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1)
        out = {"loss": (lse - picked).masked_fill(~real, 0.0)}
        if case["train"]:
            Z.sub_(lse.unsqueeze(1)).exp_()
            Z.scatter_add_(1, t.clamp(min=0).unsqueeze(1), real.double().neg().unsqueeze(1))
            Z.mul_(D["dloss"].unsqueeze(1)).masked_fill_(~real.unsqueeze(1), 0.0)
            out.update(lse=lse, dX=Z.mm(D["W"]), dW=Z.t().mm(D["X"]))
            if D["bias"] is not None:
                out["db"] = Z.sum(0)
        return out
    if kind == "norm":
        var, mean = torch.var_mean(D["X"], dim=1, unbiased=False, keepdim=True)
        sd = var.add(EPS).sqrt()
        H = D["X"].sub(mean).div(sd)
        out = {"Y": torch.addcmul(D["bias"], H, D["weight"])}
        if case["train"]:
            G = D["dY"].mul(D["weight"])
            along = G.mul(H).sum(1, keepdim=True).div(k)
            out["dX"] = G.sub(G.sum(1, keepdim=True).div(k)).sub(H.mul(along)).div(sd)
            out["dW"] = D["dY"].mul(H).sum(0)
            out["db"] = D["dY"].sum(0)
        return out
    if kind == "embed":
        ids, s = D["ids"], D["scale"]
        real = ids.ge(0)
        Y = torch.zeros((n, k), device=DEV, dtype=torch.float64)
        Y[real] = D["T"].index_select(0, ids[real]).mul(s)
        out = {"Y": Y}
        if case["train"]:
            dT = torch.zeros((case["v"], k), device=DEV, dtype=torch.float64)
            out["dT"] = dT.index_put_((ids[real],), D["dY"][real].mul(s), accumulate=True)
        return out
    keep = _numpy_keep(n * k, case["p"], D["seed"], D["offset"]).view(n, k)
    rate = 65536.0 / (65536 - round(case["p"] * 65536))
    Y = D["X"].mul(rate).mul(keep)
    if D["R"] is not None:
        Y += D["R"]
    return {"Y": Y, "dX": D["dY"].mul(rate).mul(keep)}
