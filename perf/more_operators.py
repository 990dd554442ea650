"""Timed cases of the calls around a student's rows of logits: token embeddings and
their gradient, low-rank adapters of many requests and their gradients, the
selection of beams and the reordering of their states; with their plain forms.

  op     "embed" (embed_tokens), "embed_grad" (embed_grads), "adapt" (add_adapters),
         "adapt_grad" (adapter_grads), "beam" (beam_select), "reorder" (reorder_beams)
  embed, embed_grad
    N, V, H     tokens, vocabulary and hidden size; dtype of the table, of the gradient's rows
    out         dtype of what is returned
    skew        tokens are drawn in proportion to 1 / rank^skew (0: evenly)
    padded      a tenth of the tokens are -1 (past the end of their sequence)
  adapt, adapt_grad
    N, H, O     tokens, width of the input and of the projection; dtype of input and adapters
    G, r        adapters and their rank; y: dtype of the projection's rows
    packed      the tokens of a request lie together (else each token has any adapter)
    base        tokens without an adapter, of ten
    low         adapt_grad: the forward pass kept its r numbers per token
  beam
    B, W, V     groups, beams each and vocabulary; k: beams wanted; dtype of the logits
    finished    some beams have ended
  reorder
    B, W, S     groups, beams each and elements (bf16) of a beam's state; place: in place

Where `own` is true the library's calls are made, else the same operators in
elementary torch operations.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
# a drawn case costs no more than the largest listed one of its operator
MOST_TABLE = 151936 * 4096
MOST_EMBED = 32768 * 4096
MOST_ADAPT = 8192 * 8192            # elements of the input and the projection
MOST_PLAIN = 8192 * 8192 * 256      # products of the plain form, which takes every adapter
MOST_BEAM = 512 * 151936
MOST_STATES = 1 << 28


def _embed(name, N, V, H, dtype, out, skew, padded):
    return dict(name=name, op="embed", N=N, V=V, H=H, dtype=dtype, out=out, skew=skew,
                padded=padded)


def _embed_grad(name, N, V, H, dtype, out, skew, padded):
    return dict(name=name, op="embed_grad", N=N, V=V, H=H, dtype=dtype, out=out, skew=skew,
                padded=padded)


def _adapt(name, N, H, O, G, r, dtype, y, packed, base):
    return dict(name=name, op="adapt", N=N, H=H, O=O, G=G, r=r, dtype=dtype, y=y, packed=packed,
                base=base)


def _adapt_grad(name, N, H, O, G, r, dtype, y, packed, base, low):
    return dict(name=name, op="adapt_grad", N=N, H=H, O=O, G=G, r=r, dtype=dtype, y=y,
                packed=packed, base=base, low=low)


def _beam(name, B, W, V, k, dtype, finished):
    return dict(name=name, op="beam", B=B, W=W, V=V, k=k, dtype=dtype, finished=finished)


def _reorder(name, B, W, S, place):
    return dict(name=name, op="reorder", B=B, W=W, S=S, place=place)


def listed():
    return [
        # the new tokens of a decoding step, an odd width: latency alone
        _embed("embed_step", 7, 32000, 1000, "f32", "f32", 0.0, False),
        # the tokens of a learner's batch
        _embed("embed_batch", 32768, 151936, 4096, "bf16", "bf16", 1.0, False),
        # the embedding's gradient in a learner's step: text has few words often
        _embed_grad("embed_grad_batch", 16384, 151936, 4096, "bf16", "f32", 1.0, False),
        # the ragged end of a batch, a small model
        _embed_grad("embed_grad_ragged", 1111, 50257, 1000, "f32", "bf16", 0.5, True),
        # a decoding step of requests with adapters of their own, on the head
        _adapt("adapt_step", 64, 4096, 151936, 32, 16, "bf16", "bf16", False, 1),
        # prompts of such requests, packed, at a square projection
        _adapt("adapt_prompts", 8192, 4096, 4096, 8, 32, "bf16", "bf16", True, 0),
        # the learner's step on four adapters
        _adapt_grad("adapt_grad_batch", 8192, 4096, 4096, 4, 16, "bf16", "bf16", True, 0, True),
        # fp32 training of one small adapter, odd sizes, some tokens without
        _adapt_grad("adapt_grad_odd", 777, 1000, 2001, 3, 8, "f32", "f32", False, 2, False),
        # one prompt's beams, fp32 logits
        _beam("beam_one", 1, 4, 32000, 4, "f32", False),
        # a batch of prompts, some beams ended
        _beam("beam_batch", 64, 8, 151936, 8, "bf16", True),
        # one prompt's states after a step
        _reorder("reorder_one", 1, 4, 100003, False),
        # the states of a batch
        _reorder("reorder_batch", 16, 8, 1 << 21, True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "adapt", "adapt_grad", "beam", "reorder"))
    kind = rng.choice(("bf16", "bf16", "f32"))
    if op in ("embed", "embed_grad"):
        H = _spread(rng, 64, 8192)
        V = _spread(rng, 2000, min(151936, MOST_TABLE // H))
        out = rng.choice(("bf16", "f32"))
        most = MOST_EMBED * 4 // (H * (BYTES[kind] + BYTES[out]))
        N = _spread(rng, 1, min(32768 if op == "embed" else 16384, most))
        make = _embed if op == "embed" else _embed_grad
        c = make("", N, V, H, kind, out,
                 rng.choice((0.0, 0.5, 1.0)), rng.random() < 0.3)
    elif op in ("adapt", "adapt_grad"):
        H = _spread(rng, 128, 8192)
        r = rng.choice((4, 8, 16, 16, 32, 64, rng.randint(1, 64)))
        G = _spread(rng, 1, 64)
        O = _spread(rng, 128, 151936 if op == "adapt" else 8192)
        y = rng.choice((kind, "f32"))
        most = min(8192, MOST_ADAPT * 2 // (H * BYTES[kind] + O * BYTES[y]),
                   MOST_PLAIN // (G * r * (H + O)))
        N = _spread(rng, 1, max(1, most))
        packed, base = rng.random() < 0.5, rng.choice((0, 1, 3))
        if op == "adapt":
            c = _adapt("", N, H, O, G, r, kind, y, packed, base)
        else:
            c = _adapt_grad("", N, H, O, G, r, kind, y, packed, base, rng.random() < 0.5)
    elif op == "beam":
        V = _spread(rng, 2000, 151936)
        W = rng.choice((1, 2, 4, 5, 8, 16))
        B = _spread(rng, 1, max(1, MOST_BEAM * 2 // (W * V * BYTES[kind])))
        c = _beam("", min(B, 256), W, V, rng.choice((W, 2 * W)), kind, rng.random() < 0.5)
    else:
        W = rng.choice((2, 3, 4, 8, 16))
        S = _spread(rng, 1000, 1 << 22)
        B = _spread(rng, 1, max(1, min(64, MOST_STATES // (W * S))))
        c = _reorder("", B, W, S, rng.random() < 0.5)
    del c["name"]
    return c


def work(case):
    c = case
    op = c["op"]
    if op == "embed":
        n = c["N"] * c["H"]
        rows = int(_distinct(c)) * c["H"]
        return {"bytes": rows * BYTES[c["dtype"]] + n * BYTES[c["out"]] + 4 * c["N"], "flops": n}
    if op == "embed_grad":
        n = c["N"] * c["H"]
        kept = int(n * 0.9) if c["padded"] else n
        return {"bytes": kept * BYTES[c["dtype"]] + c["V"] * c["H"] * BYTES[c["out"]] +
                4 * c["N"], "flops": 2 * kept}
    if op in ("adapt", "adapt_grad"):
        N, H, O, r, e, ey = c["N"], c["H"], c["O"], c["r"], BYTES[c["dtype"]], BYTES[c["y"]]
        used = N * (10 - c["base"]) / 10
        adapters = c["G"] * (1.0 - (1.0 - 1.0 / c["G"]) ** (used if not c["packed"] else 4 * c["G"]))
        ab = int(adapters * r * (H + O)) * e
        if op == "adapt":
            return {"bytes": int(used) * H * e + 2 * N * O * ey + ab + 4 * N,
                    "flops": int(2 * used * r * (H + O))}
        times = 2 * H + 2 * O + (0 if c["low"] else H)
        return {"bytes": int(used) * (H * e + O * ey) + N * H * e + ab + 4 * c["G"] * r * (H + O) +
                (4 * N * r if c["low"] else 0) + 4 * N, "flops": int(2 * used * r * times)}
    if op == "beam":
        n = int(c["B"] * c["W"] * c["V"] * (0.875 if c["finished"] else 1.0))
        return {"bytes": n * BYTES[c["dtype"]] + 12 * c["B"] * (c["W"] + c["k"]), "flops": 3 * n}
    # a state that is its own parent stays in place; each parent is read once
    B, W = c["B"], c["W"]
    read = B * W * (1.0 - (1.0 - 1.0 / W) ** W)
    moved = B * (W - 1) if c["place"] else B * W
    return {"bytes": int((read + moved) * c["S"]) * 2, "flops": int(moved)}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _pad(n, to):
    return (n + to - 1) // to * to


def _buffer(*shape, dtype):
    """Rows of shape[-1] elements whose stride is a multiple of 8."""
    buf = torch.zeros(*shape[:-1], _pad(shape[-1], 8), dtype=DTYPES[dtype], device="cuda")
    return buf[..., :shape[-1]]


def _normal(g, *shape, dtype, size=1.0):
    t = _buffer(*shape, dtype=dtype)
    t.copy_(torch.randn(*shape, device="cuda", generator=g) * size)
    return t


def _weights_of_ranks(c):
    return torch.arange(1, c["V"] + 1, device="cuda", dtype=torch.float64) ** -c["skew"]


def _distinct(c):
    """Expected distinct tokens among N."""
    n = c["N"] * (0.9 if c["padded"] else 1.0)
    V, skew = c["V"], c["skew"]
    if skew == 0.0:
        return V * -math.expm1(n * math.log1p(-1.0 / V))
    total = sum(i ** -skew for i in range(1, V + 1))
    return sum(-math.expm1(-n * i ** -skew / total) for i in range(1, V + 1))


def _tokens(c, g):
    """Ids as a text has them: in proportion to 1 / rank^skew, over a shuffled vocabulary."""
    below = torch.cumsum(_weights_of_ranks(c), 0)
    u = torch.rand(c["N"], device="cuda", generator=g, dtype=torch.float64) * below[-1]
    rank = torch.searchsorted(below, u).clamp(max=c["V"] - 1)
    ids = torch.randperm(c["V"], device="cuda", generator=g)[rank].int()
    if c["padded"]:
        ids[torch.rand(c["N"], device="cuda", generator=g) < 0.1] = -1
    return ids


def _requests(c, g):
    """The adapter of each token, -1 without."""
    N, G = c["N"], c["G"]
    if c["packed"]:
        # about four requests to an adapter, of unequal lengths
        cuts = torch.rand(4 * G, device="cuda", generator=g).sort().values
        at = torch.searchsorted(cuts, (torch.arange(N, device="cuda") + 0.5) / N)
    else:
        at = torch.arange(N, device="cuda")
    count = N + 4 * G + 1
    ids = torch.randint(0, G, (count,), device="cuda", generator=g, dtype=torch.int32)
    ids[torch.rand(count, device="cuda", generator=g) < c["base"] / 10] = -1
    return ids[at]


def prepare(case, seed):
    c, g = case, _generator(seed)
    op = c["op"]
    s = {"c": c}
    if op == "embed":
        s.update(ids=_tokens(c, g), table=_normal(g, c["V"], c["H"], dtype=c["dtype"], size=0.02))
    elif op == "embed_grad":
        s.update(ids=_tokens(c, g), dy=_normal(g, c["N"], c["H"], dtype=c["dtype"], size=1e-3))
    elif op in ("adapt", "adapt_grad"):
        N, H, O, G, r = c["N"], c["H"], c["O"], c["G"], c["r"]
        s.update(ids=_requests(c, g), x=_normal(g, N, H, dtype=c["dtype"]),
                 a=_normal(g, G, r, H, dtype=c["dtype"], size=H ** -0.5),
                 b=_normal(g, G, r, O, dtype=c["dtype"], size=r ** -0.5),
                 scales=torch.rand(G, device="cuda", generator=g) + 0.5)
        if op == "adapt":
            s["y"] = _normal(g, N, O, dtype=c["y"], size=2.0)
        else:
            s["dy"] = _normal(g, N, O, dtype=c["y"], size=1e-2)
            s["low"] = _low(s) if c["low"] else None
    elif op == "beam":
        B, W, V = c["B"], c["W"], c["V"]
        z = _normal(g, B * W, V, dtype=c["dtype"], size=2.0)
        # a few tokens that the model holds likely
        at = torch.randint(0, V, (B * W, 6), device="cuda", generator=g)
        z[torch.arange(B * W, device="cuda")[:, None], at] = (
            8.0 + 4.0 * torch.frac(at * 0.6180339887)).to(z.dtype)
        done = None
        if c["finished"]:
            done = (torch.rand(B, W, device="cuda", generator=g) < 0.125).to(torch.uint8)
        s.update(z=z, scores=-20.0 * torch.rand(B, W, device="cuda", generator=g), finished=done)
    else:
        B, W, S = c["B"], c["W"], c["S"]
        s.update(states=_normal(g, B * W, S, dtype="bf16"),
                 parents=torch.randint(0, W, (B, W), device="cuda", generator=g,
                                       dtype=torch.int32))
    return s


# ---------------------------------------------------------------- plain forms

def _of(ids, count):
    """[N, count]: 1 where a token has that adapter."""
    return (ids[:, None] == torch.arange(count, device=ids.device)).float()


def _low(s):
    """t = x a_g^T: every adapter's, of which a token keeps its own."""
    G, r, H = s["a"].shape
    t = (s["x"].float() @ s["a"].float().reshape(G * r, H).T).view(-1, G, r)
    return (t * _of(s["ids"], G)[:, :, None]).sum(1)


def _spread_low(t, ids, scales):
    """[N, G * r]: s_g t in the columns of a token's adapter."""
    w = _of(ids, scales.numel()) * scales
    return (w[:, :, None] * t[:, None, :]).reshape(t.shape[0], -1)


def _plain_embed(s):
    c, ids = s["c"], s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * _scale(c)
    return {"hidden": torch.where(ids[:, None] >= 0, rows, 0.0).to(DTYPES[c["out"]])}


def _plain_embed_grad(s):
    c, ids = s["c"], s["ids"].long()
    rows = torch.where(ids[:, None] >= 0, s["dy"].float(), 0.0) * _scale(c)
    d = torch.zeros(c["V"], c["H"], device=ids.device)
    d.index_add_(0, ids.clamp(min=0), rows)
    return {"dtable": d.to(DTYPES[c["out"]])}


def _scale(c):
    return math.sqrt(c["H"])


def _plain_adapt(s):
    c = s["c"]
    G, r, O = s["b"].shape
    wide = _spread_low(_low(s), s["ids"], s["scales"])
    out = s["y"].float() + wide @ s["b"].float().reshape(G * r, O)
    return {"out": out.to(DTYPES[c["y"]])}


def _plain_adapt_grad(s):
    c = s["c"]
    G, r, O = s["b"].shape
    H = c["H"]
    x, dy = s["x"].float(), s["dy"].float()
    t = s["low"] if s["low"] is not None else _low(s)
    u = (dy @ s["b"].float().reshape(G * r, O).T).view(-1, G, r)
    u = (u * (_of(s["ids"], G) * s["scales"])[:, :, None]).reshape(-1, G * r)
    return {"da": (u.T @ x).view(G, r, H),
            "db": (_spread_low(t, s["ids"], s["scales"]).T @ dy).view(G, r, O),
            "dx": (u @ s["a"].float().reshape(G * r, H)).to(DTYPES[c["dtype"]])}


def _plain_beam(z, scores, finished, k):
    B, W = scores.shape
    V = z.shape[1]
    # (scores in 64 bits: beams that are nearly as good change places in 32)
    wide = z.float()
    lse = torch.logsumexp(wide.double(), 1)
    # a row's best k, ties to the lower token: the value's order and the token in one number
    n = min(k, V)
    bits = wide.view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    key = key * 2 ** 31 + (V - 1 - torch.arange(V, device=z.device))
    at = V - 1 - (torch.topk(key, n, 1).values & (2 ** 31 - 1))
    total = scores.double().view(B * W, 1) + (wide.gather(1, at).double() - lse[:, None])
    ids = at
    if finished is not None:
        done = finished.view(B * W, 1) != 0
        first = torch.arange(n, device=z.device) == 0
        total = torch.where(done, torch.where(first, scores.double().view(B * W, 1), -math.inf),
                            total)
        ids = torch.where(done, -1, ids)
    total, ids = total.view(B, W * n), ids.view(B, W * n)
    best = torch.sort(total, dim=1, descending=True, stable=True)
    pick = best.indices[:, :k]
    some = best.values[:, :k] > -math.inf
    return {"scores": best.values[:, :k].float(),
            "parents": torch.where(some, pick // n, -1).int(),
            "ids": torch.where(some, ids.gather(1, pick), -1).int()}


def _plain_reorder(states, parents):
    B, W = parents.shape
    at = torch.arange(B, device=parents.device)[:, None] * W + parents
    return states[at.reshape(-1)]


# ---------------------------------------------------------------- one pass

def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if own:
        import paper_2606_24143_amd as opd

        if op == "embed":
            return opd.embed_tokens(s["table"], s["ids"], scale=_scale(c), dtype=DTYPES[c["out"]])
        if op == "embed_grad":
            return opd.embed_grads(s["dy"], s["ids"], c["V"], scale=_scale(c),
                                   dtype=DTYPES[c["out"]])
        if op == "adapt":
            return opd.add_adapters(s["y"], s["x"], s["a"], s["b"], s["ids"], scales=s["scales"])
        if op == "adapt_grad":
            return opd.adapter_grads(s["dy"], s["x"], s["a"], s["b"], s["ids"],
                                     scales=s["scales"], low=s["low"])
        if op == "beam":
            return opd.beam_select(s["z"], s["scores"], k=c["k"], finished=s["finished"])
        return opd.reorder_beams(s["states"], s["parents"],
                                 out=s["states"] if c["place"] else None)
    if op == "embed":
        return _plain_embed(s)
    if op == "embed_grad":
        return _plain_embed_grad(s)
    if op == "adapt":
        return _plain_adapt(s)
    if op == "adapt_grad":
        return _plain_adapt_grad(s)
    if op == "beam":
        return _plain_beam(s["z"], s["scores"], s["finished"], c["k"])
    moved = _plain_reorder(s["states"], s["parents"])
    if c["place"]:
        s["states"].copy_(moved)
        moved = s["states"]
    return {"states": moved}


# ---------------------------------------------------------------- in 64 bits

def _exact_adapters(s):
    c = s["c"]
    x, a, b = s["x"].double(), s["a"].double(), s["b"].double()
    N, H, O, G, r = c["N"], c["H"], c["O"], c["G"], c["r"]
    forward = c["op"] == "adapt"
    rows = s["y"].double() if forward else s["dy"].double()
    dx = torch.zeros(N, H, dtype=torch.float64, device=x.device)
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for g in range(G):
        at = (s["ids"] == g).nonzero()[:, 0]
        if not at.numel():
            continue
        scale = float(s["scales"][g])
        if forward:
            rows[at] += scale * (x[at] @ a[g].T @ b[g])
            continue
        t = s["low"][at].double() if s["low"] is not None else x[at] @ a[g].T
        u = scale * (rows[at] @ b[g].T)
        dx[at] = u @ a[g]
        da[g] = u.T @ x[at]
        db[g] = scale * (t.T @ rows[at])
    return {"out": rows} if forward else {"da": da, "db": db, "dx": dx}


def _exact_beam(s):
    c = s["c"]
    B, W, V, k = c["B"], c["W"], c["V"], c["k"]
    scores = torch.full((B, k), -math.inf, dtype=torch.float64)
    parents = torch.full((B, k), -1, dtype=torch.int32)
    ids = torch.full((B, k), -1, dtype=torch.int32)
    done = s["finished"].cpu() if s["finished"] is not None else torch.zeros(B, W)
    for b in range(B):
        total = s["scores"][b].double()[:, None] + torch.log_softmax(
            s["z"][b * W:(b + 1) * W].double(), 1)
        for w in range(W):
            if done[b, w]:
                total[w] = -math.inf
                total[w, 0] = s["scores"][b, w].double()
        # a tie goes to the lower parent, then to the lower token
        flat = total.view(-1)
        least = torch.topk(flat, min(k, flat.numel())).values[-1]
        at = (flat >= least).nonzero()[:, 0]
        value, order = torch.sort(flat[at], descending=True, stable=True)
        for j, (v, i) in enumerate(zip(value[:k].tolist(), at[order][:k].tolist())):
            if v == -math.inf:
                break
            scores[b, j], parents[b, j] = v, i // V
            ids[b, j] = -1 if done[b, i // V] else i % V
    return {"scores": scores, "parents": parents, "ids": ids}


def exact(case, seed):
    s = prepare(case, seed)
    c, op = case, case["op"]
    if op == "embed":
        wide = torch.cat([s["table"].double() * _scale(c),
                          torch.zeros(1, c["H"], dtype=torch.float64, device="cuda")])
        return {"hidden": wide[s["ids"].long()]}
    if op == "embed_grad":
        d = torch.zeros(c["V"] + 1, c["H"], dtype=torch.float64, device="cuda")
        d.index_add_(0, torch.where(s["ids"] < 0, c["V"], s["ids"]).long(), s["dy"].double())
        return {"dtable": d[:c["V"]] * _scale(c)}
    if op in ("adapt", "adapt_grad"):
        return _exact_adapters(s)
    if op == "beam":
        return _exact_beam(s)
    moved = torch.empty_like(s["states"], dtype=torch.float64)
    W = c["W"]
    for i, p in enumerate(s["parents"].reshape(-1).tolist()):
        moved[i] = s["states"][i // W * W + p].double()
    return {"states": moved}
