"""Timed cases of the calls around a rollout's rows of logits: blockwise 8-bit
quantisation, the output head's product, and the verification of drafted
tokens; with their plain forms.

  op     "quantize" (quantize_blocks), "head" (head_logits), "verify" (verify_drafts)
  quantize
    N, H        rows and columns; dtype of the rows
    rows        rows per block: 1 (hidden states) or 128 (head weights); a block is 128 columns wide
    scale       "f32" or "e8m0" (powers of two)
  head
    N, V, H     tokens, vocabulary and hidden size
    scale       of both operands' scales; out: dtype of the logits
  verify
    B, D, V     sequences, drafted tokens per sequence (at most) and vocabulary; dtype of the logits
    draft       the drafter's logits are given (else its tokens are certain: q is 1 at them)
    ragged      sequences have between none and D drafted tokens
    accept      about the chance that a drafted token is kept

Where `own` is true the library's calls are made, else the same operators in
elementary torch operations.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 128
TOP = 448.0  # the largest e4m3 value
# a drawn case costs no more than the largest listed one of its operator
MOST_QUANTIZE = 151936 * 4096
MOST_HEAD = 4096 * 151936 * 4096
MOST_VERIFY = 512 * 17 * 151936


def _quantize(name, N, H, dtype, rows, scale):
    return dict(name=name, op="quantize", N=N, H=H, dtype=dtype, rows=rows, scale=scale)


def _head(name, N, V, H, scale, out):
    return dict(name=name, op="head", N=N, V=V, H=H, scale=scale, out=out)


def _verify(name, B, D, V, dtype, draft, ragged, accept):
    return dict(name=name, op="verify", B=B, D=D, V=V, dtype=dtype, draft=draft, ragged=ragged,
                accept=accept)


def listed():
    return [
        # the last few tokens of a step, an odd width: latency alone
        _quantize("quantize_few", 7, 1000, "f32", 1, "f32"),
        # the hidden states of one learner or scoring batch
        _quantize("quantize_hidden", 8192, 4096, "bf16", 1, "e8m0"),
        # the output head after a weight update
        _quantize("quantize_weights", 151936, 4096, "bf16", 128, "f32"),
        # one rollout token of a small drafter
        _head("head_token", 1, 32000, 2048, "e8m0", "f32"),
        # a decoding step of a rollout batch
        _head("head_decode", 64, 151936, 4096, "f32", "bf16"),
        # the ragged end of a scoring batch, fp32 logits
        _head("head_ragged", 1111, 50257, 2000, "f32", "f32"),
        # teacher scoring, and verification of a large batch
        _head("head_scoring", 4096, 151936, 4096, "f32", "bf16"),
        _head("head_scoring_e8m0", 4096, 151936, 4096, "e8m0", "bf16"),
        # one rollout with a drafter
        _verify("verify_one", 1, 3, 32000, "bf16", True, False, 0.8),
        # a rollout batch
        _verify("verify_batch", 64, 5, 151936, "bf16", True, False, 0.7),
        # the largest rollout batch, drafts of unequal length
        _verify("verify_large", 512, 8, 151936, "bf16", True, True, 0.8),
        # drafts copied from the prompt, fp32 logits
        _verify("verify_copied", 256, 8, 50257, "f32", False, False, 0.6),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("quantize", "head", "head", "verify", "verify"))
    if op == "quantize":
        rows = rng.choice((1, 1, 128))
        H = _spread(rng, 64, 8192)
        N = _spread(rng, 1, min(151936, MOST_QUANTIZE // H))
        c = _quantize("", N, H, rng.choice(("bf16", "f32")), rows, rng.choice(("f32", "e8m0")))
    elif op == "head":
        V = _spread(rng, 2000, 151936)
        H = rng.choice((_spread(rng, 128, 8192), BLOCK * rng.randint(4, 64)))
        N = _spread(rng, 1, max(1, min(4096, MOST_HEAD // (V * H))))
        c = _head("", N, V, H, rng.choice(("f32", "e8m0")), rng.choice(("bf16", "f32")))
    else:
        V = _spread(rng, 2000, 151936)
        dtype = rng.choice(("bf16", "bf16", "f32"))
        D = rng.randint(1, 12)
        most = MOST_VERIFY * 2 // ((2 * D + 1) * V * BYTES[dtype])
        c = _verify("", _spread(rng, 1, max(1, min(512, most))), D, V, dtype,
                    rng.random() < 0.7, rng.random() < 0.5, round(rng.uniform(0.4, 0.95), 2))
    del c["name"]
    return c


def _blocks(n, size):
    return (n + size - 1) // size


def _rows_read(c):
    """Expected (target, draft) rows up to the first rejection of a sequence."""
    lens = range(c["D"] + 1) if c["ragged"] else (c["D"],)
    a = c["accept"]
    target = sum(sum(a ** i for i in range(n + 1)) for n in lens) / len(lens)
    draft = sum(sum(a ** i for i in range(n)) for n in lens) / len(lens) if c["draft"] else 0.0
    return target, draft


def work(case):
    c = case
    if c["op"] == "quantize":
        n = c["N"] * c["H"]
        scales = _blocks(c["N"], c["rows"]) * _blocks(c["H"], BLOCK)
        return {"bytes": n * (BYTES[c["dtype"]] + 1) + scales * (4 if c["scale"] == "f32" else 1),
                "flops": 3 * n}
    if c["op"] == "head":
        nb, s = _blocks(c["H"], BLOCK), 4 if c["scale"] == "f32" else 1
        return {"bytes": (c["N"] + c["V"]) * c["H"] + s * nb * (c["N"] + _blocks(c["V"], BLOCK)) +
                c["N"] * c["V"] * BYTES[c["out"]],
                "flops": 2 * c["N"] * c["V"] * c["H"]}
    # the rows up to the first rejection, once; drafts, uniforms and outputs
    elements = sum(_rows_read(c)) * c["B"] * c["V"]
    return {"bytes": int(elements * BYTES[c["dtype"]]) + c["B"] * (16 * c["D"] + 16),
            "flops": int(4 * elements)}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _pad(n, to):
    return (n + to - 1) // to * to


def _hidden(g, N, H):
    """Hidden states: tokens of unequal size, and a few channels far larger."""
    x = torch.randn(N, H, device="cuda", generator=g)
    x *= torch.exp(0.3 * torch.randn(N, 1, device="cuda", generator=g))
    x *= torch.exp(torch.randn(1, H, device="cuda", generator=g).clamp(min=1.5) - 1.5)
    return x


def _weights(g, V, H):
    return torch.randn(V, H, device="cuda", generator=g) * 0.02


def _quantized(x, rows, scale):
    """(q, scales) as a program that made them once keeps them: rows of q a
    multiple of 16 bytes apart."""
    q, s = _plain_quantize(x, rows, scale)
    N, H = x.shape
    buf = torch.zeros(N, _pad(H, 16), dtype=torch.uint8, device=x.device)
    buf[:, :H] = q.view(torch.uint8)
    return buf.view(torch.float8_e4m3fn)[:, :H], s


def _rows(x, dtype):
    """x as rows of a logit buffer whose stride is a multiple of 8 elements."""
    n, V = x.shape
    buf = torch.zeros(n, _pad(V, 8), dtype=DTYPES[dtype], device=x.device)
    buf[:, :V] = x
    return buf[:, :V]


def prepare(case, seed):
    c, g = case, _generator(seed)
    if c["op"] == "quantize":
        make = _hidden if c["rows"] == 1 else _weights
        return {"c": c, "x": _rows(make(g, c["N"], c["H"]), c["dtype"])}
    if c["op"] == "head":
        x, sx = _quantized(_hidden(g, c["N"], c["H"]), 1, c["scale"])
        w, sw = _quantized(_weights(g, c["V"], c["H"]), BLOCK, c["scale"])
        return {"c": c, "x": x, "sx": sx, "w": w, "sw": sw}
    B, D, V = c["B"], c["D"], c["V"]
    z = torch.randn(B * (D + 1), V, device="cuda", generator=g) * 2.0
    ids = None
    if c["draft"]:
        # drafts drawn from a drafter near the target
        near = z.view(B, D + 1, V)[:, :D].reshape(B * D, V)
        y = _rows(near + torch.randn(B * D, V, device="cuda", generator=g) *
                  ((1.0 - c["accept"]) / 0.4), c["dtype"])
        u = torch.rand(B * D, V, device="cuda", generator=g).clamp_(min=1e-30)
        ids = torch.argmax(y.float() - torch.log(-torch.log(u)), 1).view(B, D).int()
        del near, u
    else:
        # drafts that the target holds likely
        y = None
        ids = torch.randint(0, V, (B, D), device="cuda", generator=g, dtype=torch.int32)
        rows = (torch.arange(B * (D + 1), device="cuda").view(B, D + 1)[:, :D]).reshape(-1)
        likely = math.log(c["accept"] / (1.0 - c["accept"]))
        z[rows, ids.reshape(-1).long()] = torch.logsumexp(z[rows], 1) + likely
    lens = (torch.randint(0, D + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
            if c["ragged"] else None)
    return {"c": c, "z": _rows(z, c["dtype"]), "y": y, "ids": ids.contiguous(), "lens": lens,
            "u": torch.rand(B, D + 1, device="cuda", generator=g)}


# ---------------------------------------------------------------- plain forms

def _plain_quantize(x, rows, scale):
    N, H = x.shape
    nr, nh = _blocks(N, rows), _blocks(H, BLOCK)
    xp = torch.zeros(nr * rows, nh * BLOCK, dtype=torch.float32, device=x.device)
    xp[:N, :H] = x
    xp = xp.view(nr, rows, nh, BLOCK)
    top = xp.abs().amax((1, 3))
    if scale == "f32":
        # (divided in 64 bits: a tensor divided by a number is multiplied by its inverse,
        # and the last bit of a scale decides the ties of its block)
        s = stored = torch.clamp((top.double() / TOP).float(), min=2.0 ** -126)
    else:
        # 448 is 0.875 times 2^9: the least power of two that is top / 448 or more
        m, e = torch.frexp(top)
        e = torch.where(top > 0, e - 9 + (m > 0.875), -127).clamp(-127, 127)
        s = torch.ldexp(torch.ones_like(top, dtype=torch.float64), e)
        stored = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    q = (xp / s[:, None, :, None].to(torch.float32)).to(torch.float8_e4m3fn)
    return q.view(nr * rows, nh * BLOCK)[:N, :H].contiguous(), stored


def _wide(q, s, rows):
    """The values that q and its scales stand for, in 32 bits."""
    N, H = q.shape
    s = s.to(torch.float32).repeat_interleave(rows, 0)[:N].repeat_interleave(BLOCK, 1)[:, :H]
    return q.to(torch.float32) * s


def _plain_head(x, sx, w, sw, out):
    return (_wide(x, sx, 1) @ _wide(w, sw, BLOCK).T).to(out)


def _plain_verify(z, ids, u, y, lens):
    B, D = ids.shape
    V = z.shape[1]
    seq, pos = torch.arange(B, device=z.device), torch.arange(D, device=z.device)
    logp = torch.log_softmax(z.double(), 1).view(B, D + 1, V)
    at = ids.long()[..., None]
    p_at = logp[:, :D].gather(2, at)[..., 0]
    if y is not None:
        logq = torch.log_softmax(y.double(), 1).view(B, D, V)
        q_at = logq.gather(2, at)[..., 0].exp()
    else:
        logq, q_at = None, torch.ones_like(p_at)
    n = torch.full_like(ids[:, 0], D) if lens is None else lens
    keep = (u[:, :D].double() * q_at < p_at.exp()) & (pos < n[:, None])
    accepted = keep.int().cumprod(1).sum(1)
    refused = accepted < n
    # the draw, from the residual at the first rejection or the row past the drafts
    mass = logp[seq, accepted].exp()
    tested = accepted.clamp(max=D - 1)
    if logq is not None:
        q = logq[seq, tested].exp()
    else:
        q = torch.zeros_like(mass)
        q[seq, ids[seq, tested].long()] = 2.0
    mass = torch.where(refused[:, None], (mass - q).clamp(min=0.0), mass)
    cdf = mass.cumsum(1)
    drawn = (cdf <= u[:, D:].double() * cdf[:, -1:]).sum(1).clamp(max=V - 1)
    slot = torch.arange(D + 1, device=z.device)
    padded = torch.cat([ids, ids[:, :1]], 1)
    out = torch.where(slot == accepted[:, None], drawn[:, None].int(), padded)
    used = slot <= accepted[:, None]
    lp = logp.gather(2, out.long()[..., None])[..., 0]
    return {"accepted": accepted.int(), "ids": torch.where(used, out, -1),
            "logp": torch.where(used, lp, 0.0).float()}


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["c"]
    if own:
        import paper_2606_24143_amd as opd

        kinds = {"f32": torch.float32, "e8m0": torch.float8_e8m0fnu}
        if c["op"] == "quantize":
            return opd.quantize_blocks(state["x"], block_rows=c["rows"],
                                       scale_dtype=kinds[c["scale"]])
        if c["op"] == "head":
            return opd.head_logits(state["x"], state["sx"], state["w"], state["sw"],
                                   dtype=DTYPES[c["out"]])
        return opd.verify_drafts(state["z"], state["ids"], state["u"], draft_logits=state["y"],
                                 draft_lens=state["lens"])
    if c["op"] == "quantize":
        q, s = _plain_quantize(state["x"], c["rows"], c["scale"])
        return {"q": q, "scales": s}
    if c["op"] == "head":
        return {"logits": _plain_head(state["x"], state["sx"], state["w"], state["sw"],
                                      DTYPES[c["out"]])}
    return _plain_verify(state["z"], state["ids"], state["u"], state["y"], state["lens"])


# ---------------------------------------------------------------- in 64 bits

def _nearest_e4m3(v):
    """The e4m3 value nearest to v (64 bits): 3 bits after the leading one,
    exponents from -6, ties to the even one."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _exact_quantize(x, rows, scale):
    N, H = x.shape
    q = torch.empty(N, H, dtype=torch.float64, device=x.device)
    scales = torch.empty(_blocks(N, rows), _blocks(H, BLOCK), dtype=torch.float64,
                         device=x.device)
    for j in range(scales.shape[1]):
        cols = slice(j * BLOCK, min(j * BLOCK + BLOCK, H))
        part = x[:, cols].double()
        top = part.abs().amax(1)
        top = torch.nn.functional.pad(top, (0, scales.shape[0] * rows - N)).view(-1, rows).amax(1)
        if scale == "f32":
            # (the scale is a 32-bit number by definition)
            s = torch.clamp((top / TOP).float(), min=2.0 ** -126).double()
        else:
            s = torch.exp2(torch.ceil(torch.log2((top / TOP).clamp(min=2.0 ** -127))))
        scales[:, j] = s
        # (and so is the quotient)
        quotient = (part / s.repeat_interleave(rows)[:N, None]).float()
        q[:, cols] = _nearest_e4m3(quotient.double())
    return {"q": q, "scales": scales}


def _exact_head(x, sx, w, sw):
    z = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device=x.device)
    for j in range(sx.shape[1]):
        cols = slice(j * BLOCK, min(j * BLOCK + BLOCK, x.shape[1]))
        a = x[:, cols].float().double() * sx[:, j, None].float().double()
        b = sw[:, j].float().double().repeat_interleave(BLOCK)[:w.shape[0], None]
        z += a @ (w[:, cols].float().double() * b).T
    return {"logits": z}


def _exact_verify(z, ids, u, y, lens):
    B, D = ids.shape
    accepted = torch.zeros(B, dtype=torch.int32)
    out = torch.full((B, D + 1), -1, dtype=torch.int32)
    logp = torch.zeros(B, D + 1, dtype=torch.float64)
    drafts, chances = ids.tolist(), u.double().tolist()
    counts = [D] * B if lens is None else lens.tolist()
    for b in range(B):
        for i in range(counts[b] + 1):
            row = z[b * (D + 1) + i].double()
            p = torch.softmax(row, 0)
            mass = p
            if i < counts[b]:
                x = drafts[b][i]
                if y is not None:
                    q = torch.softmax(y[b * D + i].double(), 0)
                else:
                    q = torch.zeros_like(p)
                    q[x] = 1.0
                if chances[b][i] * float(q[x]) < float(p[x]):
                    out[b, i] = x
                    logp[b, i] = float(row[x] - torch.logsumexp(row, 0))
                    continue
                mass = torch.relu(p - q)
            accepted[b] = i
            below = torch.cumsum(mass, 0)
            j = int(torch.searchsorted(below, below[-1:] * chances[b][D], right=True))
            out[b, i] = j
            logp[b, i] = float(row[j] - torch.logsumexp(row, 0))
            break
    return {"accepted": accepted, "ids": out, "logp": logp}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return _exact_quantize(s["x"], case["rows"], case["scale"])
    if case["op"] == "head":
        return _exact_head(s["x"], s["sx"], s["w"], s["sw"])
    return _exact_verify(s["z"], s["ids"], s["u"], s["y"], s["lens"])
