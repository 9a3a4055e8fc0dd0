"""The timed cases of the logit operators: top logits, distillation from them, beam search.

A worker of a data-parallel run may send what its model answers instead of what it learned: of every row of logits the k largest
with their indices and the mass of the rest, the Top-k message of a row.  A student reads such messages in its loss and
gradient; a beam search picks its next tokens from them and moves the beams' states along.  `run` makes one such call, or
computes the same with elementary torch operations.
"""
import math

import torch

own = False

MOST_LOGITS = 2048 * 131_072       # logits of the largest listed case
MOST_STATE = 6 * 128 * 12 * 1000 * 128  # state bytes of the largest listed reordering
EOS = 0


def _case(kind, N=0, V=0, k=0, dtype="bf16", T=1.0, rest=True, pad=0, B=0, W=0, K=0, states=0, heads=0, room=0, length=0, row=0):
    return {"kind": kind, "N": N, "V": V, "k": k, "dtype": dtype, "T": T, "rest": rest, "pad": pad, "B": B, "W": W, "K": K,
            "states": states, "heads": heads, "room": room, "length": length, "row": row}


def listed():
    cases = {
        # the teacher answers one token: latency counts
        "top_1x50257_bf16": _case("top", 1, 50_257, 64),
        # a batch of short sequences, rows of odd length
        "top_999x50257_bf16": _case("top", 999, 50_257, 50),
        # a large vocabulary in full precision, softened
        "top_1024x131072_f32": _case("top", 1024, 131_072, 128, "f32", 2.0),
        # evaluation of a few tokens: the loss alone
        "loss_16x32000_f32": _case("loss", 16, 32_000, 32, "f32"),
        # evaluation of a batch, the teacher's probabilities renormalised over what was sent
        "loss_4096x32000_bf16": _case("loss", 4096, 32_000, 16, rest=False),
        # a training step that learns the loss's weight between its forward and its backward pass
        "train_2048x50257_f32": _case("train", 2048, 50_257, 64, "f32", 2.0, pad=200),
        # loss and gradient in one call: a micro-batch with padding, and a large batch
        "fused_511x50257_bf16": _case("fused", 511, 50_257, 64, pad=37),
        "fused_2048x131072_bf16": _case("fused", 2048, 131_072, 100, T=2.0),
        # a step of beam search: one sentence, and a batch in which one beam of each sentence has ended
        "beams_1x4x50257_bf16": _case("beams", V=50_257, B=1, W=4, K=4),
        "beams_32x8x128000_f32": _case("beams", V=128_000, dtype="f32", B=32, W=8, K=8),
        # the key and value caches of 12 layers follow the beams: a sentence's first tokens, a batch far on
        "reorder_1x4_24x12x17": _case("reorder", B=1, W=4, states=24, heads=12, room=64, length=17, row=128),
        "reorder_16x8_6x12x1000": _case("reorder", B=16, W=8, states=6, heads=12, room=1024, length=1000, row=128),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _spread(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """Rows of 300 to 160 thousand logits, one to 4096 of them; 1 to 64 sentences of 2 to 16 beams; caches of one to 1000 tokens."""
    kind = rng.choice(["top", "top", "loss", "train", "fused", "fused", "beams", "beams", "reorder"])
    dtype = rng.choice(["bf16", "f32"])
    if kind == "reorder":
        B, W = _spread(rng, 1, 32), rng.choice([2, 3, 4, 5, 8, 12, 16])
        states, heads, row = rng.choice([2, 4, 7, 24]), rng.choice([1, 2, 8, 12]), rng.choice([2, 12, 64, 128, 160, 256])
        most = max(1, MOST_STATE // (B * W * states * heads * row))
        length = min(_spread(rng, 1, 1000), most)
        return _case(kind, B=B, W=W, states=states, heads=heads, room=length + rng.choice([0, 1, 24]), length=length, row=row)
    V = _spread(rng, 300, 160_000)
    if kind == "beams":
        W = rng.choice([2, 3, 4, 5, 8, 12, 16])
        B = min(_spread(rng, 1, 64), max(1, MOST_LOGITS // 8 // (V * W)))
        return _case(kind, V=V, dtype=dtype, B=B, W=W, K=rng.choice([W, W, 2 * W]))
    N = min(_spread(rng, 1, 4096), MOST_LOGITS // (2 * V))
    pad = rng.choice([0, N // 8]) if kind in ("train", "fused") else 0
    return _case(kind, N, V, min(rng.choice([1, 8, 20, 50, 64, 100, 256]), V // 4), dtype, rng.choice([1.0, 1.0, 2.0, 0.7]),
                 rng.random() < 0.7, pad)


def _logits(rows, V, dtype, g):
    """Peaked rows, as trained models have them: a spread of 2 to 3.5 around an offset of the row's own."""
    scale = 2.0 + 1.5 * torch.rand((rows, 1), generator=g, device="cuda")
    z = torch.randn((rows, V), generator=g, device="cuda") * scale + torch.randn((rows, 1), generator=g, device="cuda")
    return z.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _message(t, k, T):
    """A teacher's message, in torch: the k largest logits, their indices, how many, and ln of the rest's mass next to the largest."""
    val, idx = torch.topk(t, k, dim=1)
    e = torch.exp((t.double() - val[:, :1].double()) / T).scatter_(1, idx, 0.0)
    return {"idx": idx.int(), "val": val.float(), "rest": e.sum(1).log().float(),
            "count": torch.full((t.shape[0],), k, dtype=torch.int32, device="cuda")}


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, N, V, k = case["kind"], case["N"], case["V"], case["k"]
    if kind == "reorder":
        B, W = case["B"], case["W"]
        shape = (B * W, case["heads"], case["room"], case["row"])
        s.src = [torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8) for _ in range(case["states"])]
        s.dst = [torch.zeros_like(x) for x in s.src]
        # the parents of a step: D of the W beams go on, each at least once
        D = _parents(W)
        keep = torch.rand((B, W), generator=g, device="cuda").argsort(1)[:, :D]
        more = torch.randint(0, D, (B, W - D), generator=g, device="cuda")
        s.parent = torch.cat([keep, keep.gather(1, more)], 1)
        s.parent = s.parent.gather(1, torch.rand((B, W), generator=g, device="cuda").argsort(1)).int().contiguous()
    elif kind == "beams":
        B, W = case["B"], case["W"]
        s.logits = _logits(B * W, V, case["dtype"], g)
        s.score = (-20.0 * torch.rand((B, 1), generator=g, device="cuda") - 3.0 * torch.rand((B, W), generator=g, device="cuda"))
        s.score = s.score.sort(1, descending=True).values.contiguous()
        s.done = torch.zeros((B, W), dtype=torch.uint8, device="cuda")
        n = _ended(W)
        if n:
            s.done.scatter_(1, torch.rand((B, W), generator=g, device="cuda").argsort(1)[:, :n], 1)
    else:
        s.logits = _logits(N, V, case["dtype"], g)
        if kind != "top":
            t = 0.8 * s.logits.float() + torch.randn((N, V), generator=g, device="cuda")
            s.msg = _message(t, k, case["T"])
            if case["pad"]:  # padding: rows without a message
                s.msg["count"][N - case["pad"]:] = 0
            s.weight = torch.rand(N, generator=g, device="cuda") / max(1, N)
    if own:
        _keep(s)
    return s


def _parents(W):
    return max(1, W * 5 // 8)


def _ended(W):
    return W // 8


_ctx = None


def _keep(s):
    """What a program keeps from call to call: the context and its output buffers."""
    global _ctx
    from paper_2507_05508_b200 import binding as B

    if _ctx is None:
        _ctx = B.mlmc_create(torch.cuda.current_device(), 1, 1, 1)
    case = s.case
    kind, N, V = case["kind"], case["N"], case["V"]
    if kind == "top":
        s.out = B.LogitBuffers(N, case["k"])
    elif kind == "beams":
        s.rows = B.LogitBuffers(case["B"] * case["W"], min(case["K"], V))
        s.out = B.BeamBuffers(case["B"], case["K"])
    elif kind == "reorder":
        s.states = B.BeamStates(list(zip(s.src, s.dst)), case["W"], tokens=2)  # of the whole caches; how far they are filled is the call's
    else:
        s.rows = B.LogitBuffers.of(s.msg["idx"], s.msg["val"], s.msg["count"], s.msg["rest"])
        s.out = B.DistillBuffers(N)
        if kind != "loss":
            s.grad = torch.empty_like(s.logits)


def run(s):
    case = s.case
    kind, T, rest = case["kind"], case["T"], case["rest"]
    if own:
        from paper_2507_05508_b200 import binding as B

        if kind == "top":
            B.mlmc_top_logits(_ctx, s.logits, None, T, s.out)
            return {"idx": s.out.idx, "val": s.out.val, "rest": s.out.rest, "count": s.out.count}
        if kind == "loss":
            B.mlmc_distill(_ctx, s.logits, s.rows, T, rest, None, s.out, None)
            return {"loss": s.out.loss}
        if kind == "train":
            B.mlmc_distill(_ctx, s.logits, s.rows, T, rest, None, s.out, None)
            B.mlmc_distill_grad(_ctx, s.logits, s.rows, T, rest, s.weight, s.out, s.grad)
            return {"loss": s.out.loss, "grad": s.grad}
        if kind == "fused":
            B.mlmc_distill(_ctx, s.logits, s.rows, T, rest, s.weight, s.out, s.grad)
            return {"loss": s.out.loss, "grad": s.grad}
        if kind == "beams":
            B.mlmc_top_logits(_ctx, s.logits, s.done, T, s.rows)
            B.mlmc_beam_select(_ctx, s.rows, V=case["V"], W=case["W"], T=T, score=s.score, done=s.done, eos=EOS, out=s.out)
            return {"token": s.out.token, "parent": s.out.parent, "score": s.out.score, "done": s.out.done}
        B.mlmc_beam_reorder(_ctx, s.parent, s.states.first(case["length"]))
        return s.dst
    if kind == "top":
        return _top(s.logits, case["k"], T)
    if kind == "beams":
        return _beams(s)
    if kind == "reorder":
        W, n = case["W"], case["length"]
        first = torch.arange(case["B"], device="cuda")[:, None] * W
        at = (first + s.parent).reshape(-1)
        return [b.__setitem__((slice(None), slice(None), slice(0, n)), a[:, :, :n].index_select(0, at)) or b
                for a, b in zip(s.src, s.dst)]
    return _distill(s, kind != "loss")


# ------------------------------------------------------------------------------------------ plain forms
def _order(z):
    """A 64-bit number per logit: larger for larger logits, and among equal ones for lower indices."""
    bits = (z + 0.0).view(torch.int32)
    up = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    return up.long() * 2**32 + (2**32 - 1 - torch.arange(z.shape[1], device=z.device))


def _top(logits, k, T):
    z = logits.float()
    idx = torch.topk(_order(z), k, dim=1).indices
    val = z.gather(1, idx)
    e = torch.exp((z - val[:, :1]) / T).scatter_(1, idx, 0.0)
    return {"idx": idx.int(), "val": val, "rest": e.double().sum(1).log().float(),
            "count": torch.full((z.shape[0],), k, dtype=torch.int32, device=z.device)}


def _distill(s, grad):
    """T^2 KL(q || p) of every row and T w (p - q), p and q over the sent logits and, with `rest`, the rest as one more."""
    case, m = s.case, s.msg
    T, rest = case["T"], case["rest"]
    z = s.logits.float()
    idx = m["idx"].long()
    live = m["count"] > 0
    e = torch.exp((z - z.max(1, keepdim=True).values) / T)
    p = e / e.double().sum(1, keepdim=True).float()
    p_sent = p.gather(1, idx)
    u = torch.exp((m["val"].double() - m["val"][:, :1].double()) / T)
    u_rest = torch.exp(m["rest"].double())[:, None] if rest else torch.zeros_like(u[:, :1])
    total = u.sum(1, keepdim=True) + u_rest
    q, q_rest = u / total, u_rest / total
    zd = s.logits.double()
    log_p = (z.gather(1, idx).double() / T) - torch.logsumexp(zd / T, 1, keepdim=True)
    loss = (q * (q.log() - log_p)).sum(1)
    others = e.scatter(1, idx, 0.0).double().sum(1, keepdim=True)
    p_rest = others / e.double().sum(1, keepdim=True)
    if rest:
        loss = loss + (q_rest * (q_rest.log() - p_rest.log()))[:, 0]
    loss = torch.where(live, T * T * loss, 0.0).float()
    if not grad:
        return {"loss": loss}
    q = q.float()
    d = p * (1.0 - q_rest / p_rest).float() if rest else p.clone()
    d.scatter_(1, idx, p_sent - q)
    d = torch.where(live[:, None], d * (T * s.weight)[:, None], 0.0)
    return {"loss": loss, "grad": d.to(s.logits.dtype)}


def _beams(s):
    """The K best continuations: every beam's K largest logits are enough, and their scores are compared in 64 bits."""
    case = s.case
    B, W, V, K = case["B"], case["W"], case["V"], case["K"]
    z = s.logits.float()
    idx = torch.topk(_order(z), min(K, V), dim=1).indices
    lse = torch.logsumexp(z.double(), 1, keepdim=True)
    score = (s.score.double().reshape(-1, 1) + (z.gather(1, idx).double() - lse)).reshape(B, W, -1)
    token = idx.reshape(B, W, -1)
    ended = s.done.bool()[:, :, None]
    first = (torch.arange(score.shape[2], device="cuda") == 0)[None, None]
    kept = torch.where(first, s.score.double()[:, :, None], -math.inf)
    score = torch.where(ended, kept, score).reshape(B, -1)
    token = torch.where(ended, EOS, token).reshape(B, -1)
    best, at = torch.sort(score, dim=1, descending=True, stable=True)
    at = at[:, :K]
    parent = at // min(K, V)
    token = token.gather(1, at)
    done = s.done.gather(1, parent).bool() | (token == EOS)
    return {"token": token.int(), "parent": parent.int(), "score": best[:, :K].float(), "done": done.to(torch.uint8)}


# ------------------------------------------------------------------------------------------ what has to be read, written, computed
def work(case):
    kind, N, V, k = case["kind"], case["N"], case["V"], case["k"]
    size = 2 if case["dtype"] == "bf16" else 4
    if kind == "reorder":
        one = case["B"] * case["W"] * case["states"] * case["heads"] * case["length"] * case["row"]
        return {"bytes": float(one * (1 + _parents(case["W"]) / case["W"]) + 4 * case["B"] * case["W"]), "flops": 0.0}
    if kind == "beams":  # rows of beams that have ended need not be read
        rows = case["B"] * (case["W"] - _ended(case["W"]))
        return {"bytes": float(rows * V * size + case["B"] * (case["W"] * 5 + case["K"] * 13)), "flops": 4.0 * rows * V}
    if kind == "top":
        return {"bytes": float(N * (V * size + 8 * k + 8)), "flops": 4.0 * N * V}
    live = N - case["pad"]
    read = live * (V * size + 8 * k + 8)
    if kind == "loss":
        return {"bytes": float(read + 4 * N), "flops": 4.0 * live * V}
    return {"bytes": float(read + N * (V * size + 8)), "flops": 7.0 * live * V}


# ------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    s = _plain_state(case, seed)
    kind, T = case["kind"], case["T"]
    if kind == "reorder":
        return None  # bytes are moved, nothing is computed
    if kind == "top":
        parts = [_exact_top(z.double(), case["k"], T) for z in s.logits.split(256)]
        return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    if kind == "beams":
        W, K = case["W"], case["K"]
        parts = [_exact_beams(s.logits[b * W:(b + 1) * W].double(), s.score[b].double(), s.done[b].bool(), K) for b in range(case["B"])]
        return {key: torch.stack([p[key] for p in parts]) for key in parts[0]}
    parts = [_exact_distill(s, slice(a, min(a + 128, case["N"]))) for a in range(0, case["N"], 128)]
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}


def _plain_state(case, seed):
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_top(z, k, T):
    val, idx = torch.sort(z, dim=1, descending=True, stable=True)
    behind = torch.logsumexp(val[:, k:] / T, 1) - val[:, 0] / T
    return {"idx": idx[:, :k].int(), "val": val[:, :k], "rest": behind,
            "count": torch.full((z.shape[0],), k, dtype=torch.int32, device=z.device)}


def _exact_beams(z, score, done, K):
    W, V = z.shape
    total = score[:, None] + torch.log_softmax(z, 1)
    total[done] = -math.inf
    total[done, EOS] = score[done]
    best, at = torch.sort(total.reshape(-1), descending=True, stable=True)
    parent, token = at[:K] // V, at[:K] % V
    return {"token": token.int(), "parent": parent.int(), "score": best[:K],
            "done": (done[parent] | (token == EOS)).to(torch.uint8)}


def _exact_distill(s, rows):
    """The loss as a sum over buckets of q ln(q / p), the gradient as its derivative by every logit."""
    case = s.case
    T, V = case["T"], case["V"]
    z = s.logits[rows].double() / T
    idx, live = s.msg["idx"][rows].long(), (s.msg["count"][rows] > 0)[:, None]
    n = z.shape[0]
    log_p = torch.log_softmax(z, 1)
    sent = torch.zeros((n, V), dtype=torch.bool, device="cuda").scatter_(1, idx, True)
    t = s.msg["val"][rows].double()
    buckets = t / T
    if case["rest"]:
        buckets = torch.cat([buckets, t[:, :1] / T + s.msg["rest"][rows].double()[:, None]], 1)
    log_q = torch.log_softmax(buckets, 1)
    log_p_buckets = log_p.gather(1, idx)
    rest = log_p.masked_fill(sent, -math.inf).logsumexp(1, keepdim=True)
    if case["rest"]:
        log_p_buckets = torch.cat([log_p_buckets, rest], 1)
    loss = torch.where(live, T * T * (log_q.exp() * (log_q - log_p_buckets)).sum(1, keepdim=True), 0.0)[:, 0]
    if case["kind"] == "loss":
        return {"loss": loss}
    # -sum_b q_b ln p_b: by a logit of the row p, less what its bucket has of q times its share of the bucket
    k = idx.shape[1]
    mine = torch.zeros((n, V), dtype=torch.float64, device="cuda")
    if case["rest"]:
        mine = (log_q[:, k:] + log_p - rest).exp()
    mine = mine.scatter(1, idx, log_q[:, :k].exp())
    grad = T * s.weight[rows].double()[:, None] * (log_p.exp() - mine)
    return {"loss": loss, "grad": torch.where(live, grad, 0.0)}
