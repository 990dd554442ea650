"""The rollout's calls together, captured in a graph, and on other streams: hidden
states quantised, multiplied by the head, drafts verified, the tokens scored by a
teacher and taken to the learner's loss."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_24143_amd as opd
import rollout_ref as ref
from gpu_common import DEV, say
from test_gpu_graph import _replays_match

pytestmark = pytest.mark.gpu

B, D, V, H = 24, 4, 3001, 384


def model(seed, rows, near=None, noise=0.0):
    g = torch.Generator(DEV).manual_seed(seed)
    x = torch.randn(rows, H, device=DEV, generator=g)
    if near is not None:
        x = near + noise * x
    return x


def head(seed):
    g = torch.Generator(DEV).manual_seed(seed)
    w = opd.quantize_blocks(torch.randn(V, H, device=DEV, generator=g) * 0.12, block_rows=128)
    return w["q"], w["scales"]


def logits(x, w, **kw):
    q = opd.quantize_blocks(x.bfloat16(), **kw)
    return opd.head_logits(q["q"], q["scales"], *w)["logits"]


def exact_logits(x, w):
    """The same in 64 bits: quantised values times quantised values."""
    vq, vs = ref.quantize(x.bfloat16().double().cpu().numpy(), 1, False)
    return ref.head(vq, vs, w[0].double().cpu().numpy(), w[1].double().cpu().numpy())[0]


def test_a_rollout_with_drafts_down_to_the_loss():
    student, teacher = head(1), head(2)
    # Stage 1: the drafter (the student's states, perturbed) drafts, the student verifies
    x = model(3, B * (D + 1))
    xd = model(4, B * (D + 1), near=x, noise=0.15).view(B, D + 1, H)[:, :D].reshape(B * D, H)
    z, y = logits(x, student), logits(xd, student)
    assert z.shape == (B * (D + 1), V) and z.dtype == torch.bfloat16
    off = np.abs(z.double().cpu().numpy() - exact_logits(x, student))
    assert off.max() < 0.05  # bf16 logits of magnitude up to about 10, half a step 2^-8
    g = torch.Generator(DEV).manual_seed(5)
    u = torch.rand(B * D, 1, device=DEV, generator=g)
    drafts = opd.sample_actions(y, u, want_logp=False)["ids"].view(B, D)
    uniforms = torch.rand(B, D + 1, device=DEV, generator=g)
    out = opd.verify_drafts(z, drafts, uniforms, draft_logits=y)
    a, ids, logp, near = ref.verify(z.double().cpu().numpy().reshape(B, D + 1, V),
                                    drafts.cpu().numpy(), uniforms.double().cpu().numpy(),
                                    y.double().cpu().numpy().reshape(B, D, V))
    assert near.min() > 1e-12
    assert np.array_equal(out["accepted"].cpu().numpy(), a)
    assert np.array_equal(out["ids"].cpu().numpy(), ids)
    assert 0 < a.sum() < B * D
    say("rollout: %d of %d drafts kept" % (a.sum(), B * D))
    # Stage 2: the teacher scores the tokens; those past a sequence's last are masked
    tokens = out["ids"].view(-1, 1)
    used = (tokens[:, 0] >= 0)
    xt = model(6, B * (D + 1), near=x, noise=0.3)
    tau = opd.score_actions(logits(xt, teacher), tokens, mask=used)["logp"]
    cache = dict(sampled_ids=tokens, teacher_logp=tau, behav_logp=out["logp"].view(-1, 1))
    assert opd.validate_cache("rkl_mc1", V, sampled_ids=tokens[used].contiguous(),
                              teacher_logp=tau[used].contiguous(),
                              behav_logp=out["logp"].view(-1, 1)[used].contiguous()) == 0
    # Stage 3: the learner's loss on the tokens, one update on
    xl = model(7, B * (D + 1), near=x, noise=0.05)
    zl = opd.head_logits(*(lambda q: (q["q"], q["scales"]))(opd.quantize_blocks(xl)), *student,
                         dtype=torch.float32)["logits"]
    loss = opd.loss_fwd_bwd(zl, "rkl_mc1", mask=used, **cache)
    torch.cuda.synchronize()
    n = used.cpu().numpy()
    want = oracle.rows("rkl_mc1", oracle.F32, zl.cpu().numpy()[n], V, ids=tokens.cpu().numpy()[n],
                       tau=tau.cpu().numpy()[n], beta=cache["behav_logp"].cpu().numpy()[n])
    assert np.allclose(loss["loss"].cpu().numpy()[n], want["loss"], rtol=1e-4, atol=1e-5)
    assert np.allclose(loss["dlogits"].cpu().numpy()[n], want["grad"], atol=1e-4)
    assert (loss["loss"][~used] == 0).all()


CALLS = {
    # (the head's kernels: streamed rows, once and again, tiles, an odd width)
    "few tokens": lambda s: opd.head_logits(s["q"][:9], s["s"][:9], *s["w"])["logits"],
    "more tokens": lambda s: opd.head_logits(s["q"][:300], s["s"][:300], *s["w"])["logits"],
    "tiles": lambda s: opd.head_logits(s["q"], s["s"], *s["w"])["logits"],
    "odd width": lambda s: opd.head_logits(s["q"][:, :120], s["s"][:, :1].contiguous(),
                                           s["w"][0][:, :120],
                                           s["w"][1][:, :1].contiguous())["logits"],
    "quantize": lambda s: opd.quantize_blocks(s["x"])["q"].view(torch.uint8),
    "verify": lambda s: opd.verify_drafts(s["z"], s["ids"], s["u"], draft_logits=s["y"])["ids"],
    "verify copied": lambda s: opd.verify_drafts(s["z"], s["ids"], s["u"])["logp"],
}


def state(seed):
    x = model(seed, 5000)
    q = opd.quantize_blocks(x)
    g = torch.Generator(DEV).manual_seed(seed)
    z = logits(x[:8 * 4], head(seed))
    y = z.view(8, 4, V)[:, :3].reshape(24, V) + 0.3 * torch.randn(24, V, device=DEV, generator=g)
    ybuf = torch.zeros(24, 3008, dtype=torch.bfloat16, device=DEV)
    ybuf[:, :V] = y
    return dict(x=x, q=q["q"], s=q["scales"], w=head(seed), z=z, y=ybuf[:, :V],
                ids=torch.randint(0, V, (8, 3), device=DEV, generator=g, dtype=torch.int32),
                u=torch.rand(8, 4, device=DEV, generator=g))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_calls_on_other_streams_at_once(name):
    """Two calls on two streams, each with its own outputs and workspace, give what
    one after the other gives."""
    call, s, t = CALLS[name], state(1), state(2)
    want = [call(s).clone(), call(t).clone()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for k, (st, inputs) in enumerate(zip(streams, (s, t))):
            with torch.cuda.stream(st):
                got[k].append(call(inputs).clone())
    torch.cuda.synchronize()
    for k in range(2):
        for x in got[k]:
            assert torch.equal(x, want[k])


def test_stream_argument():
    """A call given a stream runs there: it sees what was queued there before it."""
    s = state(3)
    st = torch.cuda.Stream()
    want = opd.quantize_blocks(s["x"] * 2)["q"].view(torch.uint8).clone()
    x = s["x"].clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        x *= 2
    q = opd.quantize_blocks(x, stream=st)
    z = opd.head_logits(q["q"], q["scales"], *s["w"], stream=st)["logits"]
    out = opd.verify_drafts(s["z"], s["ids"], s["u"], draft_logits=s["y"], stream=st)
    st.synchronize()
    assert torch.equal(q["q"].view(torch.uint8), want)
    assert torch.equal(z, opd.head_logits(q["q"], q["scales"], *s["w"])["logits"])
    assert torch.equal(out["ids"], opd.verify_drafts(s["z"], s["ids"], s["u"],
                                                     draft_logits=s["y"])["ids"])


def _c_verify(s, out, ws):
    st = torch.cuda.current_stream().cuda_stream
    rc = opd.lib().opd_verify_drafts(
        s["z"].data_ptr(), s["y"].data_ptr(), 1, 8, 3, V, s["z"].stride(0), s["y"].stride(0),
        s["ids"].data_ptr(), None, s["u"].data_ptr(), None, out[0].data_ptr(), out[1].data_ptr(),
        out[2].data_ptr(), ws.data_ptr(), ws.numel(), st)
    assert rc == 0


def test_verify_replayed_from_a_graph():
    s, other = state(4), state(5)
    ws = torch.full((opd.lib().opd_verify_workspace_bytes(8, 3, V, 1),), 0xA5, dtype=torch.uint8,
                    device=DEV)
    out = [torch.empty(8, dtype=torch.int32, device=DEV),
           torch.empty(8, 4, dtype=torch.int32, device=DEV), torch.empty(8, 4, device=DEV)]
    _replays_match("verify", lambda: _c_verify(s, out, ws), lambda: _c_verify(s, out, ws), out,
                   lambda: opd.verify_drafts(other["z"], other["ids"], other["u"]))


@pytest.mark.parametrize("N", [9, 200, 5000])
def test_head_replayed_from_a_graph(N):
    s, other = state(6), state(7)
    out = torch.empty(N, 3008, dtype=torch.bfloat16, device=DEV)
    q, sc = s["q"][:N], s["s"][:N]
    call = lambda: opd.head_logits(q, sc, *s["w"], out=out)
    _replays_match("head", call, call, [out[:, :V]],
                   lambda: opd.head_logits(other["q"], other["s"], *other["w"]))


def test_a_garbage_workspace_changes_nothing():
    """Nothing is taken from what an earlier call, or anyone, left in the workspace."""
    s = state(8)
    want = opd.verify_drafts(s["z"], s["ids"], s["u"], draft_logits=s["y"])
    n = opd.lib().opd_verify_workspace_bytes(8, 3, V, 1)
    for fill in (0x00, 0x01, 0xFF):
        ws = torch.full((n + 512,), fill, dtype=torch.uint8, device=DEV)
        got = opd.verify_drafts(s["z"], s["ids"], s["u"], draft_logits=s["y"], workspace=ws[:n])
        for k in want:
            assert torch.equal(got[k], want[k])
        assert (ws[n:] == fill).all()
