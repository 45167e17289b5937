"""Workloads of the adapter, loss and gradient-norm operators, for timing and
comparison.

A case is one pass of what a program does with a compressed model besides the
products of its coded weights:

  apply   adapters of many requests beside a shared projection: for the tokens
          of a batch, each with its own adapter (or none), y = y0 + s B (A x)
          on the outputs y0 of one or more projections that share x;
  back    its gradients: of every adapter's A and B, and of x;
  loss    softmax cross entropy of a large vocabulary from hidden states and
          head weights: per token the loss and the log of the sum;
  dloss   its gradient: of the hidden states, and of the head where it trains;
  clip    the global norm of many gradients and their clipping.

The plain forms work on whole dense arrays in 32 bits: every adapter is applied
to every token and masked, the logits are formed whole, the gradients lie in
flat buffers.
"""
import math
from types import SimpleNamespace

import torch

own = False  # False: the plain forms; True: this package's operators

DEV = "cuda"
NEG = -100  # the target of a token without a loss
BLOCK_8B = [([4096, 1024, 1024], 4096), ([4096], 4096), ([12288, 12288], 4096), ([4096], 12288)]


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one sequence decodes a token: q/k/v of a 4096-wide block; all latency
        dict(name="apply-one-token", op="apply", M=1, rows="4096+1024+1024", d_in=4096, rank=16, n=8, ids="mixed",
             none=0.0, ranks=False, y="bf16", keep=False),
        # a serving batch of 64 sequences, each with one of 32 adapters or none: gate and up
        dict(name="apply-64-requests", op="apply", M=64, rows="12288+12288", d_in=4096, rank=16, n=32, ids="mixed",
             none=0.1, ranks=False, y="bf16", keep=False),
        # a ragged prefill chunk of 2000 tokens from a few requests, adapters of mixed rank, 32-bit outputs
        dict(name="apply-prefill-2000", op="apply", M=2000, rows="5120", d_in=25600, rank=64, n=12, ids="segments",
             none=0.1, ranks=True, y="fp32", keep=False),
        # adapter training, four adapters in one batch of 8192 tokens, the rank-space activations kept
        dict(name="apply-train-8192", op="apply", M=8192, rows="4096+1024+1024", d_in=4096, rank=16, n=4,
             ids="segments", none=0.0, ranks=False, y="bf16", keep=True),
        # and the backward pass of that
        dict(name="back-train-8192", op="back", M=8192, rows="4096+1024+1024", d_in=4096, rank=16, n=4,
             ids="segments", none=0.0, ranks=False, y="bf16", dx=True),
        # a small odd-sized layer, mixed tokens, odd rank
        dict(name="back-ragged-333", op="back", M=333, rows="333", d_in=296, rank=5, n=7, ids="mixed", none=0.2,
             ranks=True, y="bf16", dx=True),
        # scoring the next token of one sequence over a 151,936-word vocabulary: the head is read once
        dict(name="loss-one-token", op="loss", T=1, N=151936, D=4096, ignore=0.0),
        # perplexity of a text of 2000 tokens
        dict(name="loss-2000", op="loss", T=2000, N=151936, D=4096, ignore=0.0),
        # adapter training through a frozen head: a short odd batch over a 32,003-word vocabulary, prompts ignored
        dict(name="dloss-301-frozen", op="dloss", T=301, N=32003, D=1000, ignore=0.4, head=False),
        # a training step's loss gradient of 4096 tokens, head and hidden states
        dict(name="dloss-4096", op="dloss", T=4096, N=151936, D=4096, ignore=0.0, head=True),
        # clipping the adapter gradients of 36 blocks, 504 tensors in 32 bits
        dict(name="clip-adapters", op="clip", kind="adapters", layers=36, rank=16, dtype="fp32", max_norm=1.0),
        # clipping the gradients of an embedding, a head and what lies between, ragged, mostly bf16
        dict(name="clip-ragged-1e9", op="clip", kind="ragged", count=61, total=1_000_000_007, dtype="mixed",
             max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["apply", "apply", "apply", "back", "back", "loss", "dloss", "dloss", "clip"])
    if op in ("apply", "back"):
        d_in = _log_int(rng, 64, 12288)
        if rng.random() < 0.7:
            d_in = max(64, d_in // 8 * 8)
        rows = [_log_int(rng, 64, 12288) for _ in range(rng.choice([1, 1, 2, 3]))]
        c = dict(op=op, M=_log_int(rng, 1 if op == "apply" else 16, 8192), rows="+".join(map(str, rows)), d_in=d_in,
                 rank=rng.choice([1, 4, 5, 8, 16, 16, 16, 32, 48, 64, 128]), n=_log_int(rng, 1, 48),
                 ids=rng.choice(["mixed", "segments"]), none=rng.choice([0.0, 0.0, 0.1, 0.5]),
                 ranks=rng.random() < 0.3, y="bf16")
        if op == "apply":
            c.update(y=rng.choice(["bf16", "bf16", "fp32"]), keep=rng.random() < 0.3)
        else:
            c.update(dx=rng.random() < 0.8)
        # the dense plain form's products, kept below those of the largest loss
        while c["M"] * c["n"] * c["rank"] * (d_in + sum(rows)) > 3e11:
            c["n"] = max(1, c["n"] // 2) if c["n"] > 1 else 1
            c["M"] = max(1, c["M"] * 3 // 4)
        return c
    if op in ("loss", "dloss"):
        T, N, D = _log_int(rng, 1, 4096), _log_int(rng, 1000, 151936), max(64, _log_int(rng, 64, 5120) // 8 * 8)
        c = dict(op=op, T=T, N=min(N, int(622e6 / D)), D=D, ignore=rng.choice([0.0, 0.0, 0.3, 0.9]))
        if op == "dloss":
            c.update(head=rng.random() < 0.6)
        return c
    return dict(op="clip", kind="ragged", count=_log_int(rng, 1, 500), total=_log_int(rng, 5000, 1_000_000_000),
                dtype=rng.choice(["fp32", "bf16", "mixed"]), max_norm=rng.choice([1.0, 1.0, 100.0]))


# ---------------------------------------------------------------- inputs
def _gen(seed, *more):
    s = int(seed) & 0xFFFFFFFF
    for m in more:
        s = (s * 1000003 + int(m) + 1) & 0x7FFFFFFFFFFF
    return torch.Generator(device=DEV).manual_seed(s)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _rows(c):
    return [int(r) for r in c["rows"].split("+")]


def _ids(c, g):
    """The adapter of every token: each token its own draw, or runs of ragged lengths; -1 for none."""
    M, n = c["M"], c["n"]
    if c["ids"] == "mixed":
        ids = torch.randint(0, n, (M,), generator=g, device=DEV)
        none = torch.rand(M, generator=g, device=DEV) < c["none"]
    else:
        runs = max(1, min(M, n))
        cuts = torch.rand(runs, generator=g, device=DEV).add_(0.2).cumsum(0)
        run = torch.bucketize(torch.arange(M, device=DEV) / M, (cuts / cuts[-1])[:-1], right=True)
        ids = torch.randperm(n, generator=g, device=DEV)[run % n]
        none = (torch.rand(runs, generator=g, device=DEV) < c["none"])[run]
    return torch.where(none, -1, ids).int()


def _adapters(c, g):
    """Per projection: A [n, rank, d_in], B [n, d_out, rank] in bf16, the scales; the ranks of the adapters. What lies
    past an adapter's rank is no part of it."""
    n, R, d_in = c["n"], c["rank"], c["d_in"]
    ranks = torch.randint(1, R + 1, (n,), generator=g, device=DEV).int() if c["ranks"] else None
    pools = []
    for d_out in _rows(c):
        A = (_randn(g, n, R, d_in) * (1 / math.sqrt(d_in))).bfloat16()
        B = (_randn(g, n, d_out, R) * 0.05).bfloat16()
        scale = torch.rand(n, generator=g, device=DEV) + 0.5
        pools.append((A, B, scale))
    return pools, ranks


def _clip_sizes(c):
    if c["kind"] == "adapters":
        return [c["rank"] * d for _ in range(c["layers"]) for rows, d_in in BLOCK_8B for r in rows for d in (d_in, r)]
    # ragged: each weight 1.7 times the one seven places before it, in turn large and small
    w = [1.7 ** ((i * 5) % 13) for i in range(c["count"])]
    return [max(1, int(c["total"] * x / sum(w))) for x in w]


def _clip_bf16(c, i):
    return c["dtype"] == "bf16" or (c["dtype"] == "mixed" and i % 4 != 3)


def prepare(case, seed):
    c, st = case, SimpleNamespace(c=case)
    if c["op"] in ("apply", "back"):
        g = _gen(seed, 3)
        st.ids = _ids(c, g)
        pools, st.ranks = _adapters(c, g)
        st.A, st.B, st.scale = ([p[i] for p in pools] for i in range(3))
        st.X = _randn(g, c["M"], c["d_in"]).bfloat16()
        if c["op"] == "apply":
            dt = torch.float32 if c["y"] == "fp32" else torch.bfloat16
            st.Y0 = [_randn(g, c["M"], r).to(dt) for r in _rows(c)]
        else:
            st.T = [_down(st.X, A, st.ids, st.ranks)[1] for A in st.A]  # kept from the forward pass
            st.dY = [(_randn(g, c["M"], r) * 1e-3).bfloat16() for r in _rows(c)]
            # what the shared projections pass back to x
            st.dX0 = (_randn(g, c["M"], c["d_in"]) * 1e-3).bfloat16() if c["dx"] else None
        return st
    if c["op"] in ("loss", "dloss"):
        g = _gen(seed, 5)
        T, N, D = c["T"], c["N"], c["D"]
        st.V = _randn(g, N, D).mul_(0.02 * math.sqrt(4096 / D)).bfloat16()
        t = torch.randint(0, N, (T,), generator=g, device=DEV)
        # tokens the model is sure of, and others it is not
        lift = torch.rand((T, 1), generator=g, device=DEV) * 6
        st.H = (_randn(g, T, D) + lift * st.V[t].float()).bfloat16()
        # ignored: the prompts of sequences of 512 tokens; one token always counts
        place = torch.arange(T, device=DEV)
        st.target = torch.where((place % 512 < c["ignore"] * min(T, 512)) & (place < T - 1), NEG, t)
        if c["op"] == "dloss":
            st.lse = _plain_loss(st)["lse"]
            live = st.target >= 0
            w = torch.rand(T, generator=g, device=DEV) + 0.5  # per-token weights of a mean
            st.g = torch.where(live, w, 0.0) / torch.where(live, w, 0.0).sum()
        return st
    g = _gen(seed, 7)
    sizes = _clip_sizes(c)
    want = {"fp32": torch.float32, "bf16": torch.bfloat16}
    at, place = {"fp32": 0, "bf16": 0}, []
    for i, size in enumerate(sizes):
        k = "bf16" if _clip_bf16(c, i) else "fp32"
        place.append((k, at[k], size))
        at[k] += (size + 63) // 64 * 64  # tensors on 64-element boundaries of their flat buffer
    st.flat, st.out = {}, {}
    for k, total in at.items():
        if total:
            st.flat[k] = torch.empty(total, dtype=want[k], device=DEV)
            for a in range(0, total, 1 << 26):
                st.flat[k][a:a + (1 << 26)] = _randn(g, min(1 << 26, total - a))
            st.flat[k] *= 3.0 / math.sqrt(sum(sizes))
            st.out[k] = torch.zeros(total, dtype=want[k], device=DEV)
    # the gaps belong to no tensor
    for k, a, size in place:
        st.flat[k][a + size:a + (size + 63) // 64 * 64] = 0
    if own:  # the handle that a training program makes once for its gradients
        import paper_2607_08643_amd as bsq
        st.plan = bsq.GradPlan([st.flat[k][a:a + s] for k, a, s in place], [st.out[k][a:a + s] for k, a, s in place])
    return st


# ---------------------------------------------------------------- plain forms
def _up_to_rank(W, ranks, dim):
    """The entries of W within each adapter's rank, in 32 bits; 0 past it."""
    W = W.float()
    if ranks is None:
        return W
    shape = [W.shape[0], 1, 1]
    shape[dim] = W.shape[dim]
    inside = torch.arange(W.shape[dim], device=DEV) < ranks[:, None]
    return torch.where(inside.view(shape), W, 0.0)


def _down(X, A, ids, ranks):
    """A x of every adapter, masked to each token's own: [M, n, rank], and its own alone [M, rank]."""
    n, R, d_in = A.shape
    t = (X.float() @ _up_to_rank(A, ranks, 1).reshape(n * R, d_in).T).view(-1, n, R)
    mine = ids[:, None] == torch.arange(n, device=DEV)
    t = torch.where(mine[:, :, None], t, 0.0)
    return t, t.sum(1)


def _plain_apply(st):
    out, kept = [], []
    for A, B, scale, Y0 in zip(st.A, st.B, st.scale, st.Y0):
        n, R, _ = A.shape
        t, own_t = _down(st.X, A, st.ids, st.ranks)
        up = _up_to_rank(B, st.ranks, 2).transpose(1, 2).reshape(n * R, -1)
        delta = (t * scale[:, None]).view(-1, n * R) @ up
        out.append((Y0.float() + delta).to(Y0.dtype))
        kept.append(own_t)
    return {"y": out, "t": kept} if st.c["keep"] else {"y": out}


def _plain_back(st):
    dX = st.dX0.float() if st.c["dx"] else None
    dA, dB = [], []
    for A, B, scale, t, dY in zip(st.A, st.B, st.scale, st.T, st.dY):
        n, R, d_in = A.shape
        mine = (st.ids[:, None] == torch.arange(n, device=DEV))[:, :, None]
        dY = dY.float()
        u = (dY @ _up_to_rank(B, st.ranks, 2).transpose(1, 2).reshape(n * R, -1).T).view(-1, n, R)
        u = torch.where(mine, u * scale[:, None], 0.0).view(-1, n * R)
        ts = torch.where(mine, t[:, None, :] * scale[:, None], 0.0).view(-1, n * R)
        dA.append((u.T @ st.X.float()).view(n, R, d_in))
        dB.append((dY.T @ ts).view(-1, n, R).transpose(0, 1).contiguous())
        if dX is not None:
            dX = dX + u @ _up_to_rank(A, st.ranks, 1).reshape(n * R, d_in)
    out = {"dA": dA, "dB": dB}
    return out if dX is None else {"dX": dX.bfloat16(), **out}


def _plain_loss(st):
    logits = st.H.float() @ st.V.float().T
    top = logits.amax(1)
    lse = top + (logits - top[:, None]).exp_().sum(1).log()
    live = st.target >= 0
    own_logit = logits.gather(1, st.target.clamp_min(0)[:, None])[:, 0]
    return {"loss": torch.where(live, lse - own_logit, 0.0), "lse": torch.where(live, lse, 0.0)}


def _plain_dloss(st):
    H, V = st.H.float(), st.V.float()
    live = (st.target >= 0)[:, None]
    d = (H @ V.T).sub_(st.lse[:, None]).exp_().mul_(st.g[:, None])
    d.scatter_add_(1, st.target.clamp_min(0)[:, None], -st.g[:, None])
    d.mul_(live)
    out = {"dH": (d @ V).bfloat16()}
    return {**out, "dV": (d.T @ H).bfloat16()} if st.c["head"] else out


def _plain_clip(st):
    total = sum(f.float().square().sum() for f in st.flat.values())
    norm = total.sqrt()
    coef = (st.c["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    return {"norm": torch.stack([norm, coef]),
            **{k: torch.mul(f.float(), coef).to(f.dtype) for k, f in st.flat.items()}}


PLAIN = {"apply": _plain_apply, "back": _plain_back, "loss": _plain_loss, "dloss": _plain_dloss, "clip": _plain_clip}


def run(st):
    c = st.c
    if not own:
        return PLAIN[c["op"]](st)
    import paper_2607_08643_amd as bsq
    if c["op"] in ("apply", "back"):
        pools = [bsq.AdapterPool(A, B, scale, st.ranks) for A, B, scale in zip(st.A, st.B, st.scale)]
        plan = bsq.bsq_adapters_plan(st.ids, c["n"])
        if c["op"] == "apply":
            y, t = bsq.bsq_adapters_apply(plan, pools, st.X, st.Y0, keep=c["keep"])
            return {"y": y, "t": t} if c["keep"] else {"y": y}
        dX, dA, dB = bsq.bsq_adapters_grad(plan, pools, st.X, st.T, st.dY, base=st.dX0, want_dx=c["dx"])
        return {"dX": dX, "dA": dA, "dB": dB} if c["dx"] else {"dA": dA, "dB": dB}
    if c["op"] == "loss":
        loss, lse = bsq.bsq_xent_loss(st.H, st.V, st.target)
        return {"loss": loss, "lse": lse}
    if c["op"] == "dloss":
        dH, dV = bsq.bsq_xent_grad(st.H, st.V, st.target, st.lse, st.g, head=c["head"])
        return {"dH": dH, "dV": dV} if c["head"] else {"dH": dH}
    norm = bsq.bsq_grad_clip(st.plan, c["max_norm"])
    return {"norm": norm, **st.out}


# ---------------------------------------------------------------- work, 64-bit results
def work(case):
    c = case
    if c["op"] in ("apply", "back"):
        M, d_in, R, rows = c["M"], c["d_in"], c["rank"], _rows(c)
        live = M * (1 - c["none"])
        used = min(c["n"], math.ceil(live))  # adapters that a batch can touch
        weights = used * R * (len(rows) * d_in + sum(rows))
        es = 4 if c["y"] == "fp32" else 2
        if c["op"] == "apply":
            kept = len(rows) * M * R * 4 if c["keep"] else 0
            return {"bytes": 2 * weights + 2 * M * d_in + 2 * M * sum(rows) * es + 4 * M + kept,
                    "flops": 2 * live * R * (len(rows) * d_in + sum(rows))}
        dx = 1 if c["dx"] else 0
        grads = 4 * c["n"] * R * (len(rows) * d_in + sum(rows))
        return {"bytes": 2 * weights + grads + 2 * M * d_in * (1 + 2 * dx) + 2 * M * sum(rows) + 4 * M * R * len(rows),
                "flops": 2 * live * R * (len(rows) * d_in * (1 + dx) + 2 * sum(rows))}
    if c["op"] in ("loss", "dloss"):
        T, N, D = c["T"], c["N"], c["D"]
        live = T * (1 - c["ignore"])
        if c["op"] == "loss":
            return {"bytes": 2 * (N * D + live * D) + 16 * T, "flops": 2 * live * N * D}
        head = 1 if c["head"] else 0
        return {"bytes": 2 * (N * D * (1 + head) + live * D + T * D) + 16 * T, "flops": 2 * live * N * D * (2 + head)}
    n = sum(s * (2 if _clip_bf16(c, i) else 4) for i, s in enumerate(_clip_sizes(c)))
    return {"bytes": 2 * n, "flops": 3 * sum(_clip_sizes(c))}


def _each(ids, n, ranks, R):
    """Per adapter: its tokens and its rank."""
    for a in range(n):
        yield a, (ids == a).nonzero()[:, 0], R if ranks is None else int(ranks[a])


def _exact_adapters(st):
    c = st.c
    n, R = c["n"], c["rank"]
    X = st.X.double()
    res = {"y": [], "t": [], "dA": [], "dB": []}
    dX = st.dX0.double() if c["op"] == "back" and c["dx"] else None
    for p, (A, B, scale) in enumerate(zip(st.A, st.B, st.scale)):
        if c["op"] == "apply":
            y, t = st.Y0[p].double(), torch.zeros((c["M"], R), dtype=torch.float64, device=DEV)
        else:
            dA, dB = torch.zeros_like(A, dtype=torch.float64), torch.zeros_like(B, dtype=torch.float64)
        for a, tok, r in _each(st.ids, n, st.ranks, R):
            Aa, Ba, s, x = A[a, :r].double(), B[a, :, :r].double(), float(scale[a]), X[tok]
            if c["op"] == "apply":
                t[tok, :r] = x @ Aa.T
                y[tok] += s * (t[tok, :r] @ Ba.T)
                continue
            dy = st.dY[p][tok].double()
            u = s * (dy @ Ba)
            dA[a, :r] = u.T @ x
            dB[a, :, :r] = s * (dy.T @ st.T[p][tok, :r].double())
            if dX is not None:
                dX[tok] += u @ Aa
        for k, v in (("y", y), ("t", t)) if c["op"] == "apply" else (("dA", dA), ("dB", dB)):
            res[k].append(v)
    if c["op"] == "apply":
        return {"y": res["y"], "t": res["t"]} if c["keep"] else {"y": res["y"]}
    out = {"dA": res["dA"], "dB": res["dB"]}
    return out if dX is None else {"dX": dX, **out}


def _exact_loss(st):
    """In blocks of tokens: the loss by the definition, its gradient from the probabilities."""
    c = st.c
    T, V = c["T"], st.V.double()
    loss, lse = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(2))
    dH = torch.zeros((T, c["D"]), dtype=torch.float64, device=DEV)
    dV = torch.zeros_like(V) if c.get("head") else None
    live = (st.target >= 0).nonzero()[:, 0]
    for tok in live.split(1024):
        h, t = st.H[tok].double(), st.target[tok]
        z = h @ V.T
        if c["op"] == "loss":
            logp = torch.log_softmax(z, 1)
            lse[tok] = (z - logp)[:, 0]
            loss[tok] = -logp[torch.arange(len(tok), device=DEV), t]
            continue
        p = (z - st.lse[tok, None].double()).exp_()
        p[torch.arange(len(tok), device=DEV), t] -= 1
        p *= st.g[tok, None].double()
        dH[tok] = p @ V
        if dV is not None:
            dV += p.T @ h
    if c["op"] == "loss":
        return {"loss": loss, "lse": lse}
    return {"dH": dH} if dV is None else {"dH": dH, "dV": dV}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("apply", "back"):
        return _exact_adapters(st)
    if case["op"] in ("loss", "dloss"):
        return _exact_loss(st)
    flat = {k: f.double() for k, f in st.flat.items()}
    norm = math.sqrt(sum(float(torch.dot(f, f)) for f in flat.values()))
    coef = min(1.0, case["max_norm"] / (norm + 1e-6))
    return {"norm": torch.tensor([norm, coef], dtype=torch.float64, device=DEV),
            **{k: f * coef for k, f in flat.items()}}
