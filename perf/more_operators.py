"""Workloads of the operators between a compressed model and the model it was
made from, for timing and comparison.

A case is one pass of what a program does with the two besides the products of
the coded weights:

  top     the teacher's top logits: of every token's logits the K largest with
          their words, and the log of the sum over the whole vocabulary;
  loss    distillation: per token the divergence of the student, given by its
          hidden states and head weights, from the teacher's top logits;
  step    the same with its gradient: of the hidden states, and of the head
          where it trains;
  verify  drafted tokens of many sequences, accepted or refused by the
          teacher's probabilities and given random numbers, and the token that
          follows them.

The plain forms work on whole dense arrays: the logits of the student are formed
whole in 32 bits, the probabilities of drafts in 64, since a draw compares a
random number with a sum over the vocabulary.
"""
import math
from types import SimpleNamespace

import torch

own = False  # False: the plain forms; True: this package's operators

DEV = "cuda"
INF = float("inf")
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # the teacher has scored the last tokens of eight sequences: all latency
        dict(name="top-8-tokens", op="top", T=8, N=151936, K=64, z="bf16", scale=1.0, masked=0.0),
        # a chunk of the teacher's forward pass over a training text
        dict(name="top-512", op="top", T=512, N=151936, K=64, z="bf16", scale=0.5, masked=0.0),
        # 32-bit logits of an odd vocabulary with words that are masked out, a long list
        dict(name="top-ragged-301", op="top", T=301, N=32003, K=200, z="fp32", scale=1.0, masked=0.3),
        # a short validation text, a narrow student
        dict(name="loss-37", op="loss", T=37, N=32003, D=1000, K=16, scale=1.0, norm=False, ignore=0.0),
        # validation on a text of 2000 tokens; the teacher's probabilities are of its whole vocabulary
        dict(name="loss-2000", op="loss", T=2000, N=151936, D=4096, K=64, scale=0.5, norm=True, ignore=0.0),
        # adapter training through a frozen head: a short odd batch, prompts ignored
        dict(name="step-301-frozen", op="step", T=301, N=32003, D=1000, K=50, scale=1.0, norm=False, ignore=0.4,
             head=False),
        # a training step of 4096 tokens through a frozen head: what recovers a compressed model with adapters alone
        dict(name="step-4096-frozen", op="step", T=4096, N=151936, D=4096, K=64, scale=0.5, norm=True, ignore=0.0,
             head=False),
        # the same with a head that trains
        dict(name="step-4096-head", op="step", T=4096, N=151936, D=4096, K=64, scale=0.5, norm=False, ignore=0.0,
             head=True),
        # one sequence, four drafted tokens: all latency
        dict(name="verify-one", op="verify", B=1, L=4, N=151936, z="bf16", draft=True, ragged=False, greedy=False,
             masked=0.0),
        # a serving batch of 64 sequences, four drafted tokens each
        dict(name="verify-64", op="verify", B=64, L=4, N=151936, z="bf16", draft=True, ragged=False, greedy=False,
             masked=0.0),
        # drafts of ragged lengths looked up in the text, with no probabilities of their own; a third of the sequences
        # greedy, most of the vocabulary cut off by the sampler
        dict(name="verify-ragged-33", op="verify", B=33, L=7, N=32003, z="fp32", draft=False, ragged=True, greedy=True,
             masked=0.9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["top", "top", "loss", "step", "step", "verify", "verify"])
    if op == "top":
        return dict(op=op, T=_log_int(rng, 1, 600), N=_log_int(rng, 1000, 151936), K=_log_int(rng, 1, 256),
                    z=rng.choice(["bf16", "bf16", "fp32"]), scale=rng.choice([1.0, 0.5, 0.7]),
                    masked=rng.choice([0.0, 0.0, 0.3, 0.99]))
    if op in ("loss", "step"):
        T, N, D = _log_int(rng, 1, 4096), _log_int(rng, 1000, 151936), max(64, _log_int(rng, 64, 5120) // 8 * 8)
        c = dict(op=op, T=T, N=min(N, int(622e6 / D)), D=D, K=_log_int(rng, 1, 256), scale=rng.choice([1.0, 0.5, 0.7]),
                 norm=rng.random() < 0.5, ignore=rng.choice([0.0, 0.0, 0.3, 0.9]))
        if op == "step":
            c.update(head=rng.random() < 0.5)
        return c
    return dict(op=op, B=_log_int(rng, 1, 64), L=rng.choice([0, 1, 2, 3, 4, 5, 7, 8]), N=_log_int(rng, 1000, 151936),
                z=rng.choice(["bf16", "bf16", "fp32"]), draft=rng.random() < 0.7, ragged=rng.random() < 0.5,
                greedy=rng.random() < 0.3, masked=rng.choice([0.0, 0.0, 0.9]))


# ---------------------------------------------------------------- inputs
def _gen(seed, *more):
    s = int(seed) & 0xFFFFFFFF
    for m in more:
        s = (s * 1000003 + int(m) + 1) & 0x7FFFFFFFFFFF
    return torch.Generator(device=DEV).manual_seed(s)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _lens(c):
    """Drafted tokens of each sequence."""
    return [(5 * b + 3) % (c["L"] + 1) if c["ragged"] else c["L"] for b in range(c["B"])]


def _greedy(c):
    return [c["greedy"] and b % 3 == 0 for b in range(c["B"])]


def _teacher(c, g):
    """A teacher's top logits: per token K words of its own, frequent ones more often, with falling logits; the log of
    the sum over the whole vocabulary, of which they hold most."""
    T, N, K = c["T"], c["N"], min(c["K"], c["N"])
    j = torch.arange(K, device=DEV)
    ids = j + ((N - K) * ((j + _rand(g, T, K)) / K) ** 3).long().clamp_max(N - K)
    ids = ids.gather(1, _rand(g, T, K).argsort(1))
    fall = -(_rand(g, T, K).clamp_min(1e-6).log()) * (4.0 / (1 + j.float()))
    fall[:, 0] = 0
    top = 14 + 2 * _randn(g, T, 1) - fall.cumsum(1)
    held = (top * c["scale"]).exp().sum(1).log()
    norm = held - (0.85 + 0.149 * _rand(g, T)).log()
    if K < c["K"]:
        ids = torch.nn.functional.pad(ids, (0, c["K"] - K), value=-1)
        top = torch.nn.functional.pad(top, (0, c["K"] - K), value=-INF)
    return ids.int(), top, norm


def prepare(case, seed):
    c, st = case, SimpleNamespace(c=case)
    if c["op"] == "top":
        g = _gen(seed, 11)
        st.Z = torch.empty((c["T"], c["N"]), dtype=TYPES[c["z"]], device=DEV)
        for rows in st.Z.split(128):
            z = _randn(g, *rows.shape) * 2.5
            # a few words that the teacher is sure of
            z.scatter_add_(1, torch.randint(0, c["N"], (len(rows), 12), generator=g, device=DEV),
                           6 + 6 * _rand(g, len(rows), 12))
            if c["masked"]:
                z[_rand(g, *rows.shape) < c["masked"]] = -INF
                z[:, 0].clamp_min_(0.0)  # one word always stays
            rows.copy_(z)
        return st
    if c["op"] in ("loss", "step"):
        g = _gen(seed, 13)
        T, N, D = c["T"], c["N"], c["D"]
        st.V = _randn(g, N, D).mul_(0.02 * math.sqrt(4096 / D)).bfloat16()
        st.ids, st.top, norm = _teacher(c, g)
        st.norm = norm if c["norm"] else None
        # tokens where the student is as sure as the teacher, and others where it is not
        st.H = (_randn(g, T, D) + 6 * _rand(g, T, 1) * st.V[st.ids[:, 0].long()].float()).bfloat16()
        # ignored: the prompts of sequences of 512 tokens; one token always counts
        place = torch.arange(T, device=DEV)
        prompt = (place % 512 < c["ignore"] * min(T, 512)) & (place < T - 1)
        st.ids[prompt] = -1
        if c["op"] == "step":
            w = torch.where(prompt, 0.0, _rand(g, T) + 0.5)  # per-token weights of a mean
            st.g = w / w.sum()
        return st
    g = _gen(seed, 17)
    B, L, N = c["B"], c["L"], c["N"]
    dt = TYPES[c["z"]]
    st.target = torch.empty((B, L + 1, N), dtype=dt, device=DEV)
    st.draft = torch.empty((B, L, N), dtype=dt, device=DEV) if c["draft"] else None
    st.tokens = torch.empty((B, L), dtype=torch.int32, device=DEV)
    temp = 0.6 + 0.6 * _rand(g, B)
    for b in range(B):
        z = _randn(g, L + 1, N) * 2
        z.scatter_add_(1, torch.randint(0, N, (L + 1, 8), generator=g, device=DEV), 8 + 4 * _rand(g, L + 1, 8))
        if c["masked"]:
            z[_rand(g, L + 1, N) < c["masked"]] = -INF
        z[:, 0].clamp_min_(0.0)  # one word always stays
        st.target[b] = z
        # the draft is near the teacher, and its tokens are drawn from it
        y = (z[:L] + 0.6 * _randn(g, L, N)).to(dt)
        if c["draft"]:
            st.draft[b] = y
        noise = -(-_rand(g, L, N).clamp(1e-7, 1 - 1e-7).log()).log()
        if L:
            st.tokens[b] = (y.float() / temp[b] + noise).argmax(1).int()
    st.u, st.r = _rand(g, B, L), _rand(g, B)
    st.lens = torch.tensor(_lens(c), dtype=torch.int32, device=DEV) if c["ragged"] else None
    st.temp = torch.where(torch.tensor(_greedy(c), device=DEV), 0.0, temp)
    return st


# ---------------------------------------------------------------- plain forms
def _plain_top(st):
    c = st.c
    K = min(c["K"], c["N"])
    z = st.Z.float()
    top, ids = z.sort(dim=1, descending=True, stable=True)
    top, ids = top[:, :K].clone(), ids[:, :K]
    ids = torch.where(top > -INF, ids, -1).int()
    if K < c["K"]:
        ids = torch.nn.functional.pad(ids, (0, c["K"] - K), value=-1)
        top = torch.nn.functional.pad(top, (0, c["K"] - K), value=-INF)
    z = z * c["scale"]
    peak = z.amax(1)
    return {"ids": ids, "top": top, "lse": peak + (z - peak[:, None]).exp_().sum(1).log()}


def _probabilities(st):
    """The teacher's probabilities of its words (0 where there is none), and their logarithms."""
    there = st.ids >= 0
    a = torch.where(there, st.top * st.c["scale"], -INF)
    if st.norm is None:
        peak = a.amax(1, keepdim=True).clamp_min(-1e30)
        a = a - (peak + (a - peak).exp().sum(1, keepdim=True).log())
    else:
        a = a - st.norm[:, None]
    return torch.where(there, a.exp(), 0.0), a


def _plain_distill(st):
    c = st.c
    p, logp = _probabilities(st)
    live = (st.ids >= 0).any(1)
    H, V = st.H.float(), st.V.float()
    z = (H @ V.T).mul_(c["scale"])
    peak = z.amax(1)
    lse = peak + (z - peak[:, None]).exp_().sum(1).log()
    at = st.ids.clamp_min(0).long()
    terms = torch.where(p > 0, p * (logp - (z.gather(1, at) - lse[:, None])), 0.0)
    out = {"loss": torch.where(live, terms.sum(1), 0.0), "lse": torch.where(live, lse, 0.0)}
    if c["op"] == "loss":
        return out
    gs = torch.where(live, st.g * c["scale"], 0.0)[:, None]
    total = torch.where(live, p.sum(1), 0.0)[:, None]
    d = z.sub_(lse[:, None]).exp_().mul_(gs * total)
    d.scatter_add_(1, at, torch.where(p > 0, -gs * p, 0.0))
    out["dH"] = (d @ V).bfloat16()
    if c["head"]:
        out["dV"] = (d.T @ H).bfloat16()
    return out


def _plain_verify(st):
    c = st.c
    B, L, N = c["B"], c["L"], c["N"]
    rows = torch.arange(B, device=DEV)
    lens = torch.full((B,), L, device=DEV) if st.lens is None else st.lens.long()
    greedy = st.temp == 0

    def softmax(z):
        z = z.double() / torch.where(greedy, 1.0, st.temp).double()[:, None, None]
        e = (z - z.amax(2, keepdim=True)).exp_()
        return e / e.sum(2, keepdim=True)

    p = softmax(st.target)
    best = st.target.float()
    best = (best == best.amax(2, keepdim=True)).to(torch.uint8).argmax(2)  # the lowest index of the largest
    x = st.tokens.long()
    px = p[:, :L].gather(2, x[:, :, None])[:, :, 0]
    if st.draft is None:
        q, qx = None, torch.ones_like(px)
    else:
        q = softmax(st.draft)
        qx = q.gather(2, x[:, :, None])[:, :, 0]
    ok = torch.where(greedy[:, None], x == best[:, :L], st.u.double() * qx < px)
    ok &= torch.arange(L, device=DEV) < lens[:, None]
    count = ok.long().cumprod(1).sum(1)
    w = p[rows, count]
    refused = count < lens
    if L:
        at = count.clamp_max(L - 1)
        if q is None:
            rest = w.scatter(1, x[rows, at][:, None], 0.0)
        else:
            rest = (w - q[rows, at]).clamp_min_(0.0)
        w = torch.where((refused & (rest.sum(1) > 0))[:, None], rest, w)
    sums = w.cumsum(1)
    drawn = (sums <= st.r.double()[:, None] * sums[:, -1:]).sum(1)
    drawn = torch.where(greedy, best[rows, count], drawn)
    place = torch.arange(L + 1, device=DEV)
    out = torch.nn.functional.pad(st.tokens, (0, 1), value=-1)
    out = torch.where(place < count[:, None], out, -1)
    out = torch.where(place == count[:, None], drawn[:, None].int(), out)
    return {"count": count.int(), "out": out}


PLAIN = {"top": _plain_top, "loss": _plain_distill, "step": _plain_distill, "verify": _plain_verify}


def run(st):
    c = st.c
    if not own:
        return PLAIN[c["op"]](st)
    import paper_2607_08643_amd as bsq
    if c["op"] == "top":
        ids, top, lse = bsq.bsq_top_logits(st.Z, c["K"], scale=c["scale"])
        return {"ids": ids, "top": top, "lse": lse}
    if c["op"] == "loss":
        loss, lse = bsq.bsq_distill_loss(st.H, st.V, st.ids, st.top, norm=st.norm, scale=c["scale"])
        return {"loss": loss, "lse": lse}
    if c["op"] == "step":
        loss, lse, kept = bsq.bsq_distill_loss(st.H, st.V, st.ids, st.top, norm=st.norm, scale=c["scale"], keep=True)
        dH, dV = bsq.bsq_distill_grad(st.H, st.V, st.ids, st.top, lse, st.g, norm=st.norm, scale=c["scale"], kept=kept,
                                      head=c["head"])
        out = {"loss": loss, "lse": lse, "dH": dH}
        return {**out, "dV": dV} if c["head"] else out
    count, out = bsq.bsq_draft_verify(st.target, st.tokens, st.u, st.r, draft=st.draft, lens=st.lens,
                                      temperature=st.temp)
    return {"count": count, "out": out}


# ---------------------------------------------------------------- work, 64-bit results
def work(case):
    c = case
    if c["op"] == "top":
        es = 2 if c["z"] == "bf16" else 4
        return {"bytes": c["T"] * (c["N"] * es + 8 * c["K"] + 4), "flops": 3 * c["T"] * c["N"]}
    if c["op"] in ("loss", "step"):
        T, N, D = c["T"], c["N"], c["D"]
        live = T * (1 - c["ignore"])
        small = T * (8 * c["K"] + 16)
        if c["op"] == "loss":
            return {"bytes": 2 * (N * D + live * D) + small, "flops": 2 * live * N * D}
        head = 1 if c["head"] else 0
        return {"bytes": 2 * (N * D * (1 + head) + live * D + T * D) + small, "flops": 2 * live * N * D * (2 + head)}
    es = 2 if c["z"] == "bf16" else 4
    rows = sum(n + 1 + (n if c["draft"] and not greedy else 0) for n, greedy in zip(_lens(c), _greedy(c)))
    return {"bytes": rows * c["N"] * es + c["B"] * (12 * c["L"] + 20), "flops": 3 * rows * c["N"]}


def _exact_top(st):
    """By whole-number keys: the bits of the value in order, then the lower index."""
    c = st.c
    K = min(c["K"], c["N"])
    z = st.Z.float()
    bits = z.view(torch.int32).long()
    keys = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 32) - torch.arange(c["N"], device=DEV)
    ids = keys.topk(K, dim=1).indices
    top = z.gather(1, ids).double()
    ids = torch.where(top == -INF, -1, ids).int()
    full = torch.full((c["T"], c["K"]), -1, dtype=torch.int32, device=DEV)
    vals = torch.full((c["T"], c["K"]), -INF, dtype=torch.float64, device=DEV)
    full[:, :K], vals[:, :K] = ids, top
    return {"ids": full, "top": vals, "lse": torch.logsumexp(z.double() * c["scale"], 1)}


def _exact_distill(st):
    """In blocks of tokens, by the definition: the divergence from log q, its gradient from the probabilities."""
    c = st.c
    T, s, V = c["T"], c["scale"], st.V.double()
    loss, lse = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(2))
    dH = torch.zeros((T, c["D"]), dtype=torch.float64, device=DEV)
    dV = torch.zeros_like(V) if c.get("head") else None
    for tok in (st.ids >= 0).any(1).nonzero()[:, 0].split(1024):
        h, ids, a = st.H[tok].double(), st.ids[tok], st.top[tok].double() * s
        a = a.masked_fill(ids < 0, -INF)
        logp = torch.log_softmax(a, 1) if st.norm is None else a - st.norm[tok, None].double()
        p, at = logp.exp(), ids.clamp_min(0).long()
        z = (h @ V.T) * s
        logq = torch.log_softmax(z, 1)
        lse[tok] = torch.logsumexp(z, 1)
        loss[tok] = (torch.xlogy(p, p) - p * logq.gather(1, at)).sum(1)
        if c["op"] == "loss":
            continue
        d = logq.exp() * p.sum(1, keepdim=True)
        d.scatter_add_(1, at, -p)
        d *= st.g[tok, None].double() * s
        dH[tok] = d @ V
        if dV is not None:
            dV += d.T @ h
    out = {"loss": loss, "lse": lse}
    if c["op"] == "loss":
        return out
    return {**out, "dH": dH} if dV is None else {**out, "dH": dH, "dV": dV}


def _exact_verify(st):
    """One sequence after another, one drafted token after another."""
    c = st.c
    N, count, out = c["N"], [], []
    for b, n in enumerate(_lens(c)):
        tau = float(st.temp[b])
        tokens, said = st.tokens[b, :n].tolist(), []

        def law(z):
            return torch.softmax(z.double() / tau, 0)

        w = None
        for i, x in enumerate(tokens):
            if tau == 0:
                z = st.target[b, i].float()
                if int((z == z.max()).nonzero()[0]) != x:
                    break
            else:
                p = law(st.target[b, i])
                q = law(st.draft[b, i]) if st.draft is not None else \
                    torch.zeros(N, dtype=torch.float64, device=DEV).index_fill_(0, torch.tensor([x], device=DEV), 1.0)
                if not float(st.u[b, i]) * float(q[x]) < float(p[x]):
                    w = p - q
                    w = w * (w > 0)
                    if float(w.sum()) <= 0:
                        w = p
                    break
            said.append(x)
        if tau == 0:
            z = st.target[b, len(said)].float()
            nxt = int((z == z.max()).nonzero()[0])
        else:
            sums = (law(st.target[b, len(said)]) if w is None else w).cumsum(0)
            nxt = int(torch.searchsorted(sums, sums[-1:] * float(st.r[b]), right=True))
        count.append(len(said))
        out.append(said + [nxt] + [-1] * (c["L"] - len(said)))
    return {"count": torch.tensor(count, dtype=torch.int32, device=DEV),
            "out": torch.tensor(out, dtype=torch.int32, device=DEV)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "top":
        return _exact_top(st)
    if case["op"] in ("loss", "step"):
        return _exact_distill(st)
    return _exact_verify(st)
