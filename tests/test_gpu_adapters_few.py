"""Adapters of up to 64 tokens, a decoding step, which the first product groups itself: ids of
any kind, results in place, two streams, used workspaces and graphs; one token more takes
the other way to the same."""
import pytest
import torch

import paper_2606_24143_amd as opd
from gpu_common import DEV
from test_gpu_adapters import DT, KINDS, batch, check
from test_gpu_graph import _replays_match
from test_gpu_model import copied, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,ykind", KINDS)
@pytest.mark.parametrize("N", [1, 2, 50, 63, 64, 65])
def test_bad_ids(kind, ykind, N):
    s = batch(N, N, 40, 90, 3, 6, kind, ykind, bad=False)
    bad = torch.tensor([3, -2, 2 ** 31 - 1, -2 ** 31, 4, -3], dtype=torch.int32, device=DEV)
    s["ids"][::5] = bad.repeat(3)[:len(s["ids"][::5])]
    s["ids"][1::4] = -1
    out, d = check(s, kind, ykind)
    for n in range(0, N, 5):
        if n % 4 != 1:
            assert out["out"][n].isnan().all() and d["dx"][n].isnan().all()
    none = s["ids"] == -1
    assert torch.equal(out["out"][none], s["y"][none]) and (out["low"][none] == 0).all()
    # all of one kind
    for value in (-1, 3):
        s["ids"].fill_(value)
        out, d = check(s, kind, ykind)
        assert all((d[k] == 0).all() for k in ("da", "db"))


@pytest.mark.parametrize("kind,ykind", KINDS)
@pytest.mark.parametrize("N", [1, 50, 64, 65])
def test_in_place(kind, ykind, N):
    s = batch(N + 7, N, 64, 300, 4, 16, kind, ykind)
    if N > 1:
        s["ids"][N // 2] = 9  # (a row of NaN)
    call = dict(x=s["x"], a=s["a"], b=s["b"], adapter_ids=s["ids"], scales=s["scales"])
    want = opd.add_adapters(s["y"], **call)["out"]
    y = torch.full((N, 304), 9.0, dtype=DT[ykind], device=DEV)
    y[:, :300] = s["y"]
    got = opd.add_adapters(y[:, :300], out=y[:, :300], **call)["out"]
    assert got.data_ptr() == y.data_ptr()
    assert torch.equal(got.nan_to_num(5.0), want.nan_to_num(5.0)) and (y[:, 300:] == 9).all()


@pytest.mark.parametrize("N", [1, 50, 64, 65, 600])
def test_the_shared_gradient_in_place(N):
    """dx is dx_shared: the adapters' part is added to it where it lies."""
    H, O, G, r = 64, 304, 4, 16
    s = batch(N + 8, N, H, O, G, r, "bf16", "bf16")
    dx = torch.randn(N, H, device=DEV, generator=torch.Generator(DEV).manual_seed(N)).bfloat16()
    want = opd.adapter_grads(s["y"], s["x"], s["a"], s["b"], s["ids"], scales=s["scales"], dx=dx)
    L = opd.lib()
    ws = torch.full((int(L.opd_adapter_workspace_bytes(N, H, O, G, r, 1, 1, 1)),), 0xA5,
                    dtype=torch.uint8, device=DEV)
    da, db = torch.full((G, r, H), 7.0, device=DEV), torch.full((G, r, O), 7.0, device=DEV)
    buf = torch.full((N + 1, H + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    buf[:N, :H] = dx
    p = lambda t: t.data_ptr()
    assert L.opd_adapter_grads(
        p(s["y"]), 1, s["y"].stride(0) if N > 1 else O, p(s["x"]), 1,
        s["x"].stride(0) if N > 1 else H, p(s["a"]), s["a"].stride(1), p(s["b"]),
        s["b"].stride(1), p(s["scales"]), p(s["ids"]), N, H, O, G, r, None, p(buf), H + 8, p(buf),
        H + 8, p(da), H, p(db), O, p(ws), ws.numel(),
        torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(buf[:N, :H], want["dx"])
    assert (buf[N] == 7).all() and (buf[:, H:] == 7).all()
    assert torch.equal(da, want["da"]) and torch.equal(db, want["db"])


def state(seed, N):
    return batch(seed, N, 256, 1501, 3, 8, "bf16", "f32")


def call(s, **kw):
    return opd.add_adapters(s["y"], s["x"], s["a"], s["b"], s["ids"], scales=s["scales"],
                            want_low=True, **kw)


@pytest.mark.parametrize("N", [1, 50, 64])
def test_two_streams_at_once(N):
    s, t = state(1, N), state(2, N)
    want = [copied(call(s)), copied(call(t))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(3):
        for k, (st, inputs) in enumerate(zip(streams, (s, t))):
            with torch.cuda.stream(st):
                got[k].append(copied(call(inputs)))
    torch.cuda.synchronize()
    assert all(same(x, want[k]) for k in range(2) for x in got[k])


@pytest.mark.parametrize("N", [1, 50, 64])
def test_a_garbage_workspace_changes_nothing(N):
    s = state(3, N)
    want = copied(call(s))
    n = opd.lib().opd_adapter_workspace_bytes(N, 256, 1501, 3, 8, 1, 0, 0)
    for fill in (0x00, 0x01, 0x7F, 0xFF):
        ws = torch.full((n + 512,), fill, dtype=torch.uint8, device=DEV)
        assert same(call(s, workspace=ws[:n]), want)
        assert (ws[n:] == fill).all()
    with pytest.raises(opd.OpdError, match="WORKSPACE"):
        call(s, workspace=ws[:n - 1])


@pytest.mark.parametrize("N", [1, 50, 64])
def test_replayed_from_a_graph(N):
    s, other = state(4, N), state(5, N)
    L = opd.lib()
    ws = torch.full((1 << 22,), 0xA5, dtype=torch.uint8, device=DEV)
    out = [torch.empty(N, 1504, device=DEV)[:, :1501], torch.empty(N, 8, device=DEV)]
    p = lambda t: t.data_ptr()

    def checked():
        assert L.opd_add_adapters(
            p(s["y"]), 0, s["y"].stride(0), p(s["x"]), 1, s["x"].stride(0), p(s["a"]),
            s["a"].stride(1), p(s["b"]), s["b"].stride(1), p(s["scales"]), p(s["ids"]), N, 256, 1501,
            3, 8, p(out[0]), 1504, p(out[1]), p(ws), ws.numel(),
            torch.cuda.current_stream().cuda_stream) == 0

    _replays_match("adapters of %d" % N, checked, checked, out, lambda: call(other))
