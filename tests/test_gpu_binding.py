"""The binding's native path against its interpreted one (which an explicit
stream selects): the same bytes for every form both take, the same errors for
what neither does."""
import numpy as np
import pytest
import torch

import paper_2608_12932_amd as w
from paper_2608_12932_amd import inputs as I
from helpers import bf16_dev, dev, pack, scales_dev

pytestmark = pytest.mark.gpu


class Record:
    """The native module with the results of its calls (None: declined)."""

    def __init__(self, monkeypatch):
        self.native, self.got = w._load_fast(), []
        monkeypatch.setattr(w, "_fast", self)

    def __getattr__(self, name):
        def call(*args):
            self.got.append(getattr(self.native, name)(*args))
            return self.got[-1]
        return call

    def last(self, f, *args, **kw):
        """f's result and what the last native call of it gave."""
        self.got.clear()
        r = f(*args, **kw)
        return r, self.got[-1]


def same(a, b):
    assert a.dtype == b.dtype and a.shape == b.shape
    assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("group", [False, True])
@pytest.mark.parametrize("M", [0, 3, 70])
def test_linear_paths_agree(M, group, swiglu):
    K, N = 256, 96
    x = bf16_dev(I.activations(M, K, 900 + M))
    W, s = I.weights(N, K, 901, group=group)
    wp, sd = pack(W), scales_dev(s)
    q, sx = w.w4a8_quantize_act(x)
    f = w.w4a8_linear_swiglu if swiglu else w.w4a8_linear
    mode = w.SCALE_GROUP_F16 if group else w.SCALE_CHANNEL_F32
    cur = torch.cuda.current_stream()
    for kind in (w.OUT_BF16, w.OUT_F32) + (() if swiglu else (w.OUT_I32_ACC,)):
        for xin, xs in ((x, None), (q, sx)):
            ref = f(xin, wp, sd, N, x_scale=xs, scale_mode=mode, out_kind=kind, stream=cur)
            ws = w.Workspace()
            tensor = torch.zeros(1 << 20, dtype=torch.uint8, device=dev())
            out = torch.empty_like(ref)
            for wk in (None, ws, ws, tensor):
                same(f(xin, wp, sd, N, x_scale=xs, scale_mode=mode, out_kind=kind, workspace=wk), ref)
                assert f(xin, wp, sd, N, x_scale=xs, scale_mode=mode, out_kind=kind, out=out, workspace=wk) is out
                same(out, ref)


def test_workspace_grows_and_changes_stream():
    K, N = 512, 64
    W, s = I.weights(N, K, 902)
    wp, sd, ws = pack(W), scales_dev(s), w.Workspace()
    side = torch.cuda.Stream()
    for M in (2, 200, 5):  # grows at the second
        x = bf16_dev(I.activations(M, K, 903))
        ref = w.w4a8_linear(x, wp, sd, N, stream=torch.cuda.current_stream())
        same(w.w4a8_linear(x, wp, sd, N, workspace=ws), ref)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):  # the buffer of the other stream, recorded for this one
            y = w.w4a8_linear(x, wp, sd, N, workspace=ws)
        side.synchronize()
        same(y, ref)
    assert ws.buf.numel() >= w.w4a8_linear_workspace_bytes(200, N, K)


def test_quantize_norm_and_flow_agree():
    cur = torch.cuda.current_stream()
    for M, K in ((1, 128), (5, 640), (70, 4096)):
        x = bf16_dev(I.activations(M, K, 904))
        g = torch.linspace(0.5, 1.5, K, device=dev()).to(torch.bfloat16)
        for a, b in ((w.w4a8_quantize_act(x), w.w4a8_quantize_act(x, stream=cur)),
                     (w.w4a8_rmsnorm_quantize_act(x, g, 1e-6), w.w4a8_rmsnorm_quantize_act(x, g, 1e-6, stream=cur))):
            same(a[0], b[0])
            same(a[1], b[1])
    for v_new, stats in ((True, True), (True, False), (False, False)):
        got = []
        for stream in (None, cur):
            x = torch.from_numpy(I.flow_state(3, 40, 905)).to(dev())
            v = bf16_dev(I.flow_velocity(3, 40, 906)) if v_new else None
            c = bf16_dev(I.flow_velocity(3, 40, 907))
            st = w.w4a8_flow_step(x, v, c, 0.125, stats=stats, repeat=2, stream=stream)
            got.append((x, c, st))
        same(got[0][0], got[1][0])
        same(got[0][1], got[1][1])
        assert (got[0][2] is None) == (not stats)
        if stats:
            same(got[0][2], got[1][2])


def test_refused_calls():
    K, N = 256, 64
    x = bf16_dev(I.activations(4, K, 908))
    W, s = I.weights(N, K, 909)
    wp, sd = pack(W), scales_dev(s)
    with pytest.raises(TypeError):
        w.w4a8_linear(x.float(), wp, sd, N)
    with pytest.raises(TypeError):
        w.w4a8_linear(x, wp, sd.half(), N)
    with pytest.raises(TypeError):
        w.w4a8_linear(x, wp.cpu(), sd, N)
    with pytest.raises(ValueError):
        w.w4a8_linear(x[:, ::2], wp, sd, N)
    with pytest.raises(ValueError):
        w.w4a8_linear(w.w4a8_quantize_act(x)[0], wp, sd, N)  # codes without scales
    with pytest.raises(ValueError):
        w.w4a8_linear(x, wp, sd, N, out=torch.empty(4, N + 1, dtype=torch.bfloat16, device=dev()))
    with pytest.raises(w.W4A8Error):
        w.w4a8_linear(x, wp, sd, 24)  # not a multiple of 16
    with pytest.raises(w.W4A8Error):
        w.w4a8_linear(x, wp, sd, N, workspace=torch.zeros(16, dtype=torch.uint8, device=dev()))
    with pytest.raises(w.W4A8Error):
        w.w4a8_rmsnorm_quantize_act(x, torch.ones(K, dtype=torch.bfloat16, device=dev()), -1.0)
    with pytest.raises(ValueError):
        w.w4a8_rmsnorm_quantize_act(x, torch.ones(K + 8, dtype=torch.bfloat16, device=dev()), 1e-6)
    with pytest.raises(ValueError):
        w.w4a8_flow_step(torch.zeros(2, 8, device=dev()), None, torch.zeros(2, 4, dtype=torch.bfloat16, device=dev()), 0.1)


def test_native_path_is_taken(monkeypatch):
    K, N, M = 512, 64, 20
    rec = Record(monkeypatch)
    x = bf16_dev(I.activations(M, K, 910))
    (q, sx), got = rec.last(w.w4a8_quantize_act, x)
    assert type(got) is tuple and got[0] is q
    r, got = rec.last(w.w4a8_rmsnorm_quantize_act, x, torch.ones(K, dtype=torch.bfloat16, device=dev()), 1e-6)
    assert r is got
    for f, group in ((w.w4a8_linear, False), (w.w4a8_linear, True), (w.w4a8_linear_swiglu, True)):
        W, s = I.weights(N, K, 911, group=group)
        wp, sd = pack(W), scales_dev(s)
        kw = dict(scale_mode=w.SCALE_GROUP_F16 if group else w.SCALE_CHANNEL_F32)
        ws = w.Workspace()
        need = w.w4a8_linear_workspace_bytes(M, N, K, int(group))
        assert need > 0 and w.w4a8_linear_workspace_bytes(M, N, K, int(group), w.IN_I8) == 0
        for wk in (ws, ws, None, torch.zeros(need, dtype=torch.uint8, device=dev())):
            y, got = rec.last(f, x, wp, sd, N, workspace=wk, **kw)
            assert y is got
        y, got = rec.last(f, q, wp, sd, N, x_scale=sx, **kw)
        assert y is got
        out = torch.empty_like(y)
        y, got = rec.last(f, x, wp, sd, N, workspace=ws, out=out, **kw)
        assert y is out and got is out
    f = lambda v, stats: rec.last(w.w4a8_flow_step, torch.zeros(2, 8, device=dev()), v,
                                  torch.zeros(2, 8, dtype=torch.bfloat16, device=dev()), 0.1, stats=stats)
    v = torch.ones(2, 8, dtype=torch.bfloat16, device=dev())
    st, got = f(v, True)
    assert st is got and st.shape == (2, 4)
    assert f(v, False) == (None, True) and f(None, False) == (None, True)


def test_native_path_declines(monkeypatch):
    import copy
    K, N, M = 512, 64, 20
    rec = Record(monkeypatch)
    x = bf16_dev(I.activations(M, K, 912))
    W, s = I.weights(N, K, 913)
    wp, sd, ws = pack(W), scales_dev(s), w.Workspace()
    ref = w.w4a8_linear(x, wp, sd, N, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # a Workspace of another stream, a copy of one
        y, got = rec.last(w.w4a8_linear, x, wp, sd, N, workspace=ws)
        twin = copy.deepcopy(ws)
    assert got is None
    side.synchronize()
    same(y, ref)
    y, got = rec.last(w.w4a8_linear, x, wp, sd, N, workspace=twin)
    assert got is None
    same(y, ref)

    class Sub(torch.Tensor):
        pass

    y, got = rec.last(w.w4a8_linear, x.as_subclass(Sub), wp, sd, N)
    assert got is None
    same(y.as_subclass(torch.Tensor), ref)


def test_refused_calls_leave_the_workspace_alone():
    K, N, M = 512, 64, 20
    x = bf16_dev(I.activations(M, K, 912))
    W, s = I.weights(N, K, 913)
    wp, sd = pack(W), scales_dev(s)
    ws = w.Workspace()
    for bad in (dict(x=x.float()), dict(x=x[:, ::2]), dict(wp=wp.cpu()), dict(sd=sd.half()),
                dict(out=torch.empty(M, N + 1, dtype=torch.bfloat16, device=dev()))):
        a = dict(x=x, wp=wp, sd=sd, out=None) | bad
        with pytest.raises((TypeError, ValueError)):
            w.w4a8_linear(a["x"], a["wp"], a["sd"], N, out=a["out"], workspace=ws)
        assert ws.buf.numel() == 0, list(bad)


def cache_step(B=3, L=3000, H=8, Hkv=2):
    """A cache of random codes, and a batch of one new token for each sequence."""
    g = torch.Generator(device=dev()).manual_seed(914)
    blocks = -(-L // w.CACHE_BLOCK)
    cache = w.KVCache.empty(B * blocks, B, Hkv, device=dev())
    for t in cache[:2]:
        t.copy_(torch.randint(-127, 128, t.shape, generator=g, device=dev()))
    cache.scales.fill_(0.01)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev())  # noqa: E731
    table = torch.arange(B * blocks, dtype=torch.int32, device=dev()).view(B, blocks)
    qkv = torch.randn(B, H + 2 * Hkv, 128, generator=g, device=dev()).to(torch.bfloat16)
    ang = torch.rand(8, 64, generator=g, device=dev())
    batch = (i32(*range(B + 1)), i32(*[L] * B), table, i32(*range(B)), ang.cos(), ang.sin())
    assert w.w4a8_cache_attention_workspace_bytes(B, B, H, Hkv, blocks * 64) > 0
    return qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], cache, batch


def test_native_path_is_taken_by_the_cache_calls(monkeypatch):
    rec = Record(monkeypatch)
    cur = torch.cuda.current_stream()
    K, M = 512, 20
    x, r = (bf16_dev(I.activations(M, K, s)) for s in (915, 916))
    gain = torch.linspace(0.5, 1.5, K, device=dev()).to(torch.bfloat16)
    ref = w.w4a8_add_rmsnorm_quantize_act(x, r, gain, 1e-6, stream=cur)
    for out in (None, torch.empty_like(x)):
        y, got = rec.last(w.w4a8_add_rmsnorm_quantize_act, x, r, gain, 1e-6, out=out)
        assert y is got and (out is None or y[2] is out)
        for a, b in zip(y, ref):
            same(a, b)

    q, k, v, cache, batch = cache_step()
    twin = w.KVCache(*(t.clone() for t in cache))
    w.w4a8_cache_append(k, v, twin, *batch, stream=cur)
    assert rec.last(w.w4a8_cache_append, k, v, cache, *batch) == (None, True)
    for a, b in zip(cache, twin):
        same(a, b)
    slots = torch.arange(3, dtype=torch.int32, device=dev())
    assert rec.last(w.w4a8_cache_append, k, v, cache, *batch, slots=slots) == (None, True)

    ref = w.w4a8_cache_attention(q, cache, *batch, 0.1, stream=cur)
    need = w.w4a8_cache_attention_workspace_bytes(3, 3, 8, 2, batch[2].shape[1] * 64)
    ws = w.Workspace()
    for wk in (ws, ws, None, torch.zeros(need, dtype=torch.uint8, device=dev())):
        for out in (None, torch.empty_like(ref), torch.empty(8, 3, 128, dtype=torch.bfloat16, device=dev()).transpose(0, 1)):
            y, got = rec.last(w.w4a8_cache_attention, q, cache, *batch, 0.1, workspace=wk, out=out)
            assert y is got and (out is None or y is out)
            same(y, ref)
    y, got = rec.last(w.w4a8_cache_attention, q, cache, *batch, 0.1, max_len=3000, workspace=ws)
    assert y is got
    bare = w.KVCache(*cache[:3])  # rings are the append's alone
    y, got = rec.last(w.w4a8_cache_attention, q, bare, *batch, 0.1, workspace=ws)
    assert y is got
    same(y, ref)


def test_native_path_declines_cache_calls(monkeypatch):
    import copy
    rec = Record(monkeypatch)
    q, k, v, cache, batch = cache_step()
    ws = w.Workspace()
    ref = w.w4a8_cache_attention(q, cache, *batch, 0.1, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # a Workspace of another stream, a copy of one
        y, got = rec.last(w.w4a8_cache_attention, q, cache, *batch, 0.1, workspace=ws)
        twin = copy.deepcopy(ws)
    assert got is None
    side.synchronize()
    same(y, ref)
    y, got = rec.last(w.w4a8_cache_attention, q, cache, *batch, 0.1, workspace=twin)
    assert got is None
    same(y, ref)
    y, got = rec.last(w.w4a8_cache_attention, q, cache, *batch, 1, workspace=ws)  # a scale that is no float
    assert got is None and torch.isfinite(y).all()

    class Sub(torch.Tensor):
        pass

    y, got = rec.last(w.w4a8_cache_attention, q.as_subclass(Sub), cache, *batch, 0.1, workspace=ws)
    assert got is None
    same(y.as_subclass(torch.Tensor), ref)
    rings = [t.clone() for t in cache]
    r, got = rec.last(w.w4a8_cache_append, k.as_subclass(Sub), v, cache, *batch)
    assert r is None and got is None
    w.w4a8_cache_append(k, v, w.KVCache(*rings), *batch)
    for a, b in zip(cache, rings):
        same(a, b)
    x = bf16_dev(I.activations(4, 256, 917))
    gain = torch.ones(256, dtype=torch.bfloat16, device=dev())
    y, got = rec.last(w.w4a8_add_rmsnorm_quantize_act, x.as_subclass(Sub), x, gain, 1e-6)
    assert got is None
    for a, b in zip(y, w.w4a8_add_rmsnorm_quantize_act(x, x, gain, 1e-6)):
        same(a.as_subclass(torch.Tensor), b)


@pytest.mark.parametrize("held", [0, 128])
@pytest.mark.parametrize("native", [True, False])
def test_refused_attention_leaves_the_workspace_alone(held, native):
    q, _, _, cache, batch = cache_step()
    kw = {} if native else dict(stream=torch.cuda.current_stream())
    ws = w.Workspace()
    if held:
        ws.get(held)
    buf, home = ws.buf, ws._home
    odd = torch.zeros(q.numel() + 4, dtype=torch.bfloat16, device=dev())[4:].view(q.shape)  # not 16-byte aligned
    flat = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device=dev()).expand(3, 8, 128)
    for bad in (dict(max_len=0), dict(max_len=1 << 20), dict(q=odd), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=odd),
                dict(out=flat), dict(cos=torch.zeros(8 * 64 + 2, device=dev())[2:].view(8, 64))):
        a = dict(q=q, scale=0.1, max_len=None, out=None, cos=batch[4]) | bad
        with pytest.raises(w.W4A8Error):
            w.w4a8_cache_attention(a["q"], cache, *batch[:4], a["cos"], batch[5], a["scale"], max_len=a["max_len"], out=a["out"],
                                   workspace=ws, **kw)
        assert ws.buf is buf and ws._home is home, list(bad)
    y = w.w4a8_cache_attention(q, cache, *batch, 0.1, workspace=ws, **kw)
    assert ws.buf.numel() > held
    same(y, w.w4a8_cache_attention(q, cache, *batch, 0.1))


@pytest.mark.parametrize("native", [True, False])
def test_calls_that_the_library_refuses_leave_the_workspace_alone(native):
    kw = {} if native else dict(stream=torch.cuda.current_stream())
    K, N, M = 512, 64, 20
    x = bf16_dev(I.activations(M, K, 918))
    W, s = I.weights(N, K, 919)
    wp, sd = pack(W), scales_dev(s)
    shifted = lambda t: torch.cat([t.new_zeros(4), t.flatten()])[4:].view(t.shape)  # noqa: E731  (not 16-byte aligned)
    ws = w.Workspace()
    buf, home = ws.buf, ws._home
    for f in (w.w4a8_linear, w.w4a8_linear_swiglu):
        for bad in (dict(x=shifted(x)), dict(wp=shifted(wp))):
            a = dict(x=x, wp=wp) | bad
            with pytest.raises(w.W4A8Error):
                f(a["x"], a["wp"], sd, N, workspace=ws, **kw)
            assert ws.buf is buf and ws._home is home, list(bad)
    q = bf16_dev(I.activations(2 * 5, 128, 920)).view(2, 5, 128)
    i = torch.arange(5, dtype=torch.int32, device=dev())
    t = torch.ones(5, 64, device=dev())
    for bad in (dict(q=shifted(q)), dict(scale=float("nan"))):
        a = dict(q=q, scale=0.1) | bad
        with pytest.raises(w.W4A8Error):
            w.w4a8_stream_attention(a["q"], q, q, i, i, t, t, a["scale"], workspace=ws, **kw)
        assert ws.buf is buf and ws._home is home, list(bad)
    y = w.w4a8_linear(x, wp, sd, N, workspace=ws, **kw)
    assert ws.buf.numel() > 0
    same(y, w.w4a8_linear(x, wp, sd, N))
