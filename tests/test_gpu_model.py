"""The calls around the rows of logits together, as a rollout and a learner use them;
captured in graphs, on other streams, with workspaces of any content."""
import math

import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2606_24143_amd as opd
from gpu_common import DEV, say
from test_gpu_graph import _replays_match

pytestmark = pytest.mark.gpu

V, H, G, R = 1501, 256, 3, 8


def model(seed):
    """A student of one layer: embedding, head (8 bits), and adapters of three requests on
    the head."""
    g = torch.Generator(DEV).manual_seed(seed)
    table = torch.randn(V, H, device=DEV, generator=g).bfloat16()
    head = opd.quantize_blocks(torch.randn(V, H, device=DEV, generator=g) * 0.1, block_rows=128)
    a = (torch.randn(G, R, H, device=DEV, generator=g) * H ** -0.5).bfloat16()
    b = torch.zeros(G, R, 1504, device=DEV, dtype=torch.bfloat16)[:, :, :V]
    b.copy_(torch.randn(G, R, V, device=DEV, generator=g))
    return dict(table=table, head=head, a=a, b=b,
                scales=torch.tensor([0.5, 1.0, 2.0], device=DEV))


def logits(m, x, ids, **kw):
    """Rows of logits of hidden states x, each with its request's adapter."""
    q = opd.quantize_blocks(x)
    y = opd.head_logits(q["q"], q["scales"], m["head"]["q"], m["head"]["scales"],
                        dtype=torch.float32)["logits"]
    return y, opd.add_adapters(y, x, m["a"], m["b"], ids, scales=m["scales"], **kw)


def exact_logits(m, y, x, ids):
    t = np.einsum("nh,nrh->nr", x, m["a"].double().cpu().numpy()[ids])
    s = m["scales"].double().cpu().numpy()[ids][:, None]
    return y + np.einsum("nr,nrv->nv", s * t, m["b"].double().cpu().numpy()[ids])


def test_beam_search_with_adapters():
    """Three steps of a rollout by beams: embed, head, adapters, select, reorder the
    states (here the sum of the embeddings so far)."""
    m = model(1)
    B, W = 3, 4
    ids = torch.arange(B, dtype=torch.int32, device=DEV).repeat_interleave(W)  # a request each
    n_ids = ids.cpu().numpy()
    tokens = torch.tensor([5, 77, 1200], dtype=torch.int32, device=DEV).repeat_interleave(W)
    scores = torch.full((B, W), -math.inf, device=DEV)
    scores[:, 0] = 0.0
    state = torch.zeros(B * W, H, device=DEV)
    for step in range(3):
        x = opd.embed_tokens(m["table"], tokens, scale=0.25, dtype=torch.float32)["hidden"]
        state = (state + x) * 0.7
        h = state.bfloat16()
        y, out = logits(m, h, ids)
        z = out["out"]
        want = exact_logits(m, y.double().cpu().numpy(), h.double().cpu().numpy(), n_ids)
        assert np.abs(z.double().cpu().numpy() - want).max() < 1e-4
        sel = opd.beam_select(z, scores)
        s, parents, toks, near = ref.beams(z.double().cpu().numpy().reshape(B, W, V),
                                           scores.double().cpu().numpy(), W)
        assert near > 1e-6
        assert np.array_equal(sel["parents"].cpu().numpy(), parents)
        assert np.array_equal(sel["ids"].cpu().numpy(), toks)
        before = state.clone()
        opd.reorder_beams(state, sel["parents"], out=state)
        at = torch.from_numpy(parents).to(DEV).long() + torch.arange(B, device=DEV)[:, None] * W
        assert torch.equal(state, before[at.view(-1)])
        scores, tokens = sel["scores"], sel["ids"].view(-1)
    assert scores.isfinite().all() and (tokens >= 0).all()
    say("beams: best score of each request %s" % scores[:, 0].tolist())


def test_a_learners_step_on_adapters_and_embedding():
    """Loss at the logits, back through the adapters to the embedding, against the same in
    64 bits: the loss's gradient at the logits is the library's, all else is linear in it."""
    m = model(2)
    N = 90
    rng = np.random.default_rng(3)
    toks = rng.integers(0, 40, N).astype(np.int32)
    toks[::9] = -1  # past the end of their sequences
    ids = rng.integers(-1, G, N).astype(np.int32)
    t_tok, t_ids = torch.from_numpy(toks).to(DEV), torch.from_numpy(ids).to(DEV)
    x = opd.embed_tokens(m["table"], t_tok)["hidden"]
    y, out = logits(m, x, t_ids, want_low=True)
    sup = opd.topk_support(y, 16)
    loss = opd.loss_fwd_bwd(out["out"], "fkl_topk", idx=sup["idx"], teacher_logp=sup["logp"],
                            mask=t_tok >= 0)
    dz = loss["dlogits"]
    assert loss["loss"].isfinite().all() and float(dz.abs().max()) > 0
    d = opd.adapter_grads(dz, x, m["a"], m["b"], t_ids, scales=m["scales"], low=out["low"])
    de = opd.embed_grads(d["dx"], t_tok, V)["dtable"]
    # in 64 bits from the same dz (rows whose adapter is none have no part here)
    np64 = lambda t: t.double().cpu().numpy()
    want = ref.adapter_grads(np64(dz), np64(x), np64(m["a"]), np64(m["b"]), ids, np64(m["scales"]),
                             "bf16", "f32", low=np64(out["low"]))
    for k in ("da", "db", "dx"):
        value, off = want[k]
        off = off + (ref.HALF["bf16"] if k == "dx" else ref.HALF["f32"]) * (np.abs(value) + off)
        assert (np.abs(np64(d[k]) - value) <= off).all(), k
    value, off = ref.embed_grads(np64(d["dx"]), toks, V, 1.0)
    assert (np.abs(np64(de) - value) <= off + ref.HALF["f32"] * np.abs(value)).all()
    # an update against the gradient
    assert float((d["da"].abs().sum((1, 2)) > 0).sum()) == G


# ---------------------------------------------------------------- streams, graphs, workspaces

def state(seed, N=600):
    g = torch.Generator(DEV).manual_seed(seed)
    ids = torch.randint(-1, G, (N,), device=DEV, generator=g, dtype=torch.int32)
    x = torch.randn(N, H, device=DEV, generator=g)
    y = torch.randn(N, 1504, device=DEV, generator=g)[:, :V]
    m = model(seed)
    return dict(m, x=x.bfloat16(), y=y, ids=ids, dx=x,
                tokens=torch.randint(-1, V, (N,), device=DEV, generator=g, dtype=torch.int32),
                z=y[:64], scores=-torch.rand(8, 8, device=DEV, generator=g),
                parents=torch.randint(0, 8, (8, 8), device=DEV, generator=g, dtype=torch.int32))


CALLS = {
    "embed": lambda s, **kw: opd.embed_tokens(s["table"], s["tokens"], **kw),
    "embed grads": lambda s, **kw: opd.embed_grads(s["dx"], s["tokens"], V, **kw),
    "embed grads of few": lambda s, **kw: opd.embed_grads(s["dx"][:50], s["tokens"][:50], V, **kw),
    "adapters": lambda s, **kw: opd.add_adapters(s["y"], s["x"], s["a"], s["b"], s["ids"],
                                                 scales=s["scales"], want_low=True, **kw),
    "adapter grads": lambda s, **kw: opd.adapter_grads(s["y"], s["x"], s["a"], s["b"], s["ids"],
                                                       scales=s["scales"], **kw),
    "beams": lambda s, **kw: opd.beam_select(s["z"], s["scores"], k=16, **kw),
    "reorder": lambda s, **kw: opd.reorder_beams(s["dx"][:64], s["parents"], **kw),
}
WITH_WORKSPACE = ("embed grads", "adapters", "adapter grads", "beams")


def same(got, want):
    return all(torch.equal(got[k].nan_to_num(), want[k].nan_to_num()) for k in want)


def copied(d):
    return {k: t.clone() for k, t in d.items()}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_calls_on_other_streams_at_once(name):
    """Two calls on two streams, each with its own outputs and workspace, give what one
    after the other gives."""
    call, s, t = CALLS[name], state(1), state(2)
    want = [copied(call(s)), copied(call(t))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for k, (st, inputs) in enumerate(zip(streams, (s, t))):
            with torch.cuda.stream(st):
                got[k].append(copied(call(inputs)))
    torch.cuda.synchronize()
    for k in range(2):
        for x in got[k]:
            assert same(x, want[k])


@pytest.mark.parametrize("name", sorted(CALLS))
def test_stream_argument(name):
    """A call given a stream runs there: it sees what was queued there before it."""
    s = state(3)
    for k in ("x", "dx", "y", "table"):
        s[k].mul_(2)
    want = copied(CALLS[name](dict(s, z=s["y"][:64])))
    s = state(3)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for k in ("x", "dx", "y", "table"):
            s[k].mul_(2)
    got = CALLS[name](dict(s, z=s["y"][:64]), stream=st)
    st.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_a_garbage_workspace_changes_nothing(name):
    """Nothing is taken from what an earlier call, or anyone, left in the workspace, and
    nothing behind it is written."""
    s = state(4)
    want = copied(CALLS[name](s))
    L = opd.lib()
    n = {"embed grads": L.opd_embed_workspace_bytes(600, V, H),
         "adapters": L.opd_adapter_workspace_bytes(600, H, V, G, R, 1, 0, 0),
         "adapter grads": L.opd_adapter_workspace_bytes(600, H, V, G, R, 1, 0, 1),
         "beams": L.opd_beam_workspace_bytes(8, 8, V, 0)}[name]
    for fill in (0x00, 0x01, 0x7F, 0xFF):
        ws = torch.full((n + 512,), fill, dtype=torch.uint8, device=DEV)
        assert same(CALLS[name](s, workspace=ws[:n]), want)
        assert (ws[n:] == fill).all()
    with pytest.raises(opd.OpdError, match="WORKSPACE"):
        CALLS[name](s, workspace=ws[:n - 1])


@pytest.mark.parametrize("name", sorted(CALLS))
def test_replayed_from_a_graph(name):
    """Two captured calls with workspaces of their own, replayed beside eager ones."""
    s, other = state(5), state(6)
    L = opd.lib()
    st = lambda: torch.cuda.current_stream().cuda_stream
    ws = torch.full((1 << 24,), 0xA5, dtype=torch.uint8, device=DEV)
    p = lambda t: t.data_ptr()
    f32 = dict(dtype=torch.float32, device=DEV)
    if name == "embed":
        out = [torch.empty(600, H, dtype=torch.bfloat16, device=DEV)]
        call = lambda: L.opd_embed_tokens(p(s["table"]), 1, V, H, H, p(s["tokens"]), 600, 1.0,
                                          p(out[0]), 1, H, st())
    elif name.startswith("embed grads"):
        N = 50 if name.endswith("few") else 600
        out = [torch.empty(V, H, **f32)]
        call = lambda: L.opd_embed_grads(p(s["dx"]), 0, N, H, H, p(s["tokens"]), V, 1.0, p(out[0]),
                                         0, H, 0, p(ws), ws.numel(), st())
    elif name == "adapters":
        out = [torch.empty(600, 1504, **f32)[:, :V], torch.empty(600, R, **f32)]
        call = lambda: L.opd_add_adapters(
            p(s["y"]), 0, 1504, p(s["x"]), 1, H, p(s["a"]), H, p(s["b"]), 1504, p(s["scales"]),
            p(s["ids"]), 600, H, V, G, R, p(out[0]), 1504, p(out[1]), p(ws), ws.numel(), st())
    elif name == "adapter grads":
        out = [torch.empty(G, R, H, **f32), torch.empty(G, R, 1504, **f32)[:, :, :V],
               torch.empty(600, H, dtype=torch.bfloat16, device=DEV)]
        call = lambda: L.opd_adapter_grads(
            p(s["y"]), 0, 1504, p(s["x"]), 1, H, p(s["a"]), H, p(s["b"]), 1504, p(s["scales"]),
            p(s["ids"]), 600, H, V, G, R, None, None, 0, p(out[2]), H, p(out[0]), H, p(out[1]),
            1504, p(ws), ws.numel(), st())
    elif name == "beams":
        out = [torch.empty(8, 16, **f32), torch.empty(8, 16, dtype=torch.int32, device=DEV),
               torch.empty(8, 16, dtype=torch.int32, device=DEV)]
        call = lambda: L.opd_beam_select(p(s["z"]), 0, 8, 8, V, 1504, p(s["scores"]), None, 16,
                                         *map(p, out), p(ws), ws.numel(), st())
    else:
        out = [torch.empty(64, H, **f32)]
        call = lambda: L.opd_reorder_beams(p(s["dx"]), 8, 8, 1, H * 4, H * 4, H * 4,
                                           p(s["parents"]), 8, p(out[0]), H * 4, H * 4, st())

    def checked():
        assert call() == 0

    _replays_match(name, checked, checked, out, lambda: CALLS[name](other))
