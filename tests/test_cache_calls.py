"""Host-side checks (no GPU needed) of the residual norm and of the 8-bit
cache's calls: malformed ones are rejected before anything is launched, empty
ones do nothing, and the oracle's definitions hold together."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2608_12932_amd as w
from paper_2608_12932_amd import inputs as I

P = ctypes.c_void_p
EINVAL, OK = w.W4A8_EINVAL, w.W4A8_OK


def at(i):
    """A fake address, 4 GiB from the others; never dereferenced."""
    return P((i + 1) << 32)


def test_add_rmsnorm_rejections():
    f = w.lib().w4a8_add_rmsnorm_quantize_act
    X, R, G, S, Q, SC = (at(i) for i in range(6))
    call = lambda x=X, r=R, g=G, eps=1e-6, M=4, K=256, s=S, q=Q, sc=SC: f(x, r, g, eps, M, K, s, q, sc, None)  # noqa: E731
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert call(eps=eps) == EINVAL
    for K in (0, 100, 65536 + 128):
        assert call(K=K) == EINVAL
    assert call(M=-1) == EINVAL and call(M=(1 << 20) + 1) == EINVAL
    for name in ("x", "r", "g", "s", "q", "sc"):
        assert call(**{name: None}) == EINVAL
        assert call(**{name: P(at(9).value + 2)}) == EINVAL  # misaligned
    n = 4 * 256 * 2
    for name, base in (("s", X), ("s", R), ("q", X), ("q", G), ("q", S), ("sc", S), ("sc", Q), ("sc", R)):
        assert call(**{name: P(base.value + 16)}) == EINVAL  # an output inside an input or another output
    assert call(s=P(X.value + n - 16)) == EINVAL
    assert call(q=X) == EINVAL and call(s=G) == EINVAL
    assert call(M=0, x=None, r=None, g=None, s=None, q=None, sc=None) == OK


def cache(pages=10, Hkv=8, slots=4, **over):
    d = dict(k_codes=at(0), v_codes=at(1), scales=at(2), n_pages=pages, Hkv=Hkv, k_recent=at(3), v_recent=at(4), n_slots=slots)
    d.update(over)
    return w._CacheArgs(*(d[n] for n, _ in w._CacheArgs._fields_))


def batch(**over):
    d = dict(starts=at(5), lengths=at(6), table=at(7), max_blocks=16, B=4, T=8, pos=at(8), rope_cos=at(9), rope_sin=at(10), n_pos=64)
    d.update(over)
    return w._BatchArgs(*(d[n] for n, _ in w._BatchArgs._fields_))


BAD_CACHE = [dict(k_codes=None), dict(v_codes=None), dict(scales=None), dict(k_codes=P(24)), dict(v_codes=P(8)), dict(scales=P(4)),
             dict(pages=0), dict(pages=1 << 31), dict(Hkv=0), dict(Hkv=4097)]
BAD_BATCH = [dict(starts=None), dict(lengths=None), dict(table=None), dict(pos=None), dict(rope_cos=None), dict(rope_sin=None),
             dict(rope_cos=P(8)), dict(starts=P(2)), dict(max_blocks=0), dict(max_blocks=(1 << 24) + 1), dict(B=-1), dict(B=65537),
             dict(T=-1), dict(T=(1 << 20) + 1), dict(n_pos=0), dict(n_pos=(1 << 30) + 1)]


def test_append_rejections():
    f = w.lib().w4a8_cache_append
    K, V = at(20), at(21)
    call = lambda c=None, b=None, k=K, kr=6144, kh=128, v=V, vr=6144, vh=128, slots=None: f(  # noqa: E731
        c or cache(), b or batch(), k, kr, kh, v, vr, vh, slots, None)
    for over in BAD_CACHE + [dict(k_recent=None), dict(v_recent=P(8)), dict(slots=0), dict(slots=1 << 31)]:
        assert call(c=cache(**over)) == EINVAL, over
    for over in BAD_BATCH:
        assert call(b=batch(**over)) == EINVAL, over
    for over in (dict(k=None), dict(v=None), dict(k=P(8)), dict(kr=-8), dict(kh=4), dict(vr=100), dict(vh=-128), dict(vr=1 << 41),
                 dict(slots=P(2)), dict(c=cache(slots=3))):  # (the last: four sequences, three rings, and no slots)
        assert call(**over) == EINVAL, over
    assert f(None, batch(), K, 128, 128, V, 128, 128, None, None) == EINVAL
    assert f(cache(), None, K, 128, 128, V, 128, 128, None, None) == EINVAL
    for over in (dict(T=0), dict(B=0)):  # nothing to do
        none = cache(k_codes=None, v_codes=None, scales=None, k_recent=None, v_recent=None)
        assert f(none, batch(starts=None, lengths=None, table=None, pos=None, rope_cos=None, rope_sin=None, **over), None, 0, 0, None, 0, 0,
                 None, None) == OK


def test_attention_rejections():
    f = w.lib().w4a8_cache_attention
    Q, O = at(20), at(21)
    big = (at(22), 1 << 30)
    call = lambda c=None, b=None, q=Q, qr=6144, qh=128, H=32, scale=0.1, max_len=1000, o=O, orow=4096, oh=128, ws=big: f(  # noqa: E731
        c or cache(), b or batch(), q, qr, qh, H, scale, max_len, o, orow, oh, *ws, None)
    for over in BAD_CACHE:
        assert call(c=cache(**over)) == EINVAL, over
    for over in BAD_BATCH:
        assert call(b=batch(**over)) == EINVAL, over
    for over in (dict(q=None), dict(o=None), dict(q=P(8)), dict(qr=-8), dict(qh=4), dict(H=0), dict(H=30), dict(H=8192), dict(max_len=0),
                 dict(max_len=16 * 64 + 1), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-float("inf"))):
        assert call(**over) == EINVAL, over
    # output rows that overlap: heads on heads, tokens on tokens, tokens on heads
    for orow, oh in ((4096, 0), (0, 128), (128, 128), (4096, 120), (4088, 128), (128, 1016)):
        assert call(orow=orow, oh=oh) == EINVAL, (orow, oh)
    # 2^28 rows of a kv head: more are refused, before any memory is touched
    for T, H, Hkv in ((1 << 20, 4096, 1), ((1 << 20) - 1, 4096, 8), (1 << 20, 514, 2)):
        assert call(c=cache(Hkv=Hkv), b=batch(T=T), H=H, orow=H * 128) == w.W4A8_EUNSUPPORTED, (T, H, Hkv)
    # a call that splits its sequences needs the workspace
    need = w.w4a8_cache_attention_workspace_bytes(4, 8, 32, 8, 1000)
    assert need > 64 * 1024
    for ws in ((None, 0), (at(22), need - 1), (P(at(22).value + 16), need)):
        assert call(ws=ws) == EINVAL
    for over in (dict(T=0), dict(B=0)):
        none = cache(k_codes=None, v_codes=None, scales=None, k_recent=None, v_recent=None)
        assert f(none, batch(starts=None, lengths=None, table=None, pos=None, rope_cos=None, rope_sin=None, **over), None, 0, 0, 32, 0.1,
                 1000, None, 0, 0, None, 0, None) == OK


def test_workspace_bytes():
    f = w.w4a8_cache_attention_workspace_bytes
    assert f(64, 64, 32, 8, 64) == 0  # one block: nothing to split
    for bad in ((-1, 8, 32, 8, 100), (4, -1, 32, 8, 100), (4, 8, 30, 8, 100), (4, 8, 32, 0, 100), (4, 8, 32, 8, 0), (0, 8, 32, 8, 100),
                (4, 0, 32, 8, 100), (4, 1 << 21, 32, 8, 100)):
        assert f(*bad) == 0, bad


def test_binding_checks_before_the_device():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    with pytest.raises(TypeError):  # not a device tensor
        w.w4a8_add_rmsnorm_quantize_act(x, x, x[0], 1e-6)
    c = w.KVCache.empty(2, 1, 8, device="cpu")
    assert c.k_codes.shape == (2, 8, 64, 128) and c.v_codes.shape == (2, 8, 128, 64) and c.k_recent.shape == (1, 8, 128, 128)
    i = torch.zeros(1, dtype=torch.int32)
    t = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        w.w4a8_cache_append(x.view(1, 8, 128), x.view(1, 8, 128), c, torch.zeros(2, dtype=torch.int32), i, i[None], i, t, t)
    with pytest.raises(TypeError):
        w.w4a8_cache_attention(x.view(1, 8, 128), c, torch.zeros(2, dtype=torch.int32), i, i[None], i, t, t, 0.1)


def test_workspace_of_another_device():
    class Buffer:  # what the check sees of a device tensor
        is_cuda = True

        def __init__(self, index, n=8):
            self.device, self.n = torch.device("cuda", index), n

        def numel(self):
            return self.n

    def workspace(device, buf):
        ws = w.Workspace.__new__(w.Workspace)
        ws.device, ws.buf = torch.device(device), buf
        return ws

    here = torch.device("cuda", 1)
    for ok in (None, Buffer(1), workspace("cuda", Buffer(0, 0)), workspace("cuda", Buffer(1)), workspace("cuda:1", Buffer(1, 0))):
        w._check_workspace_device(ok, here)
    for bad in (Buffer(0), workspace("cuda", Buffer(0)), workspace("cuda:0", Buffer(0, 0)), workspace("cuda:0", Buffer(0))):
        with pytest.raises(ValueError):
            w._check_workspace_device(bad, here)


# ---- the oracle


def test_oracle_add_norm_is_add_then_norm():
    x, r = I.activations(5, 256, 1), I.activations(5, 256, 2)
    g = I.activations(1, 256, 3, outliers=False)[0]
    q, s, total = oracle.add_rmsnorm_quantize(x, r, g, 1e-6)
    t = torch.from_numpy(x.view(np.int16)).view(torch.bfloat16) + torch.from_numpy(r.view(np.int16)).view(torch.bfloat16)
    np.testing.assert_array_equal(total, t.view(torch.int16).numpy().view(np.uint16))
    q2, s2, _, _ = oracle.rmsnorm_quantize(total, g, 1e-6)
    np.testing.assert_array_equal(q, q2)
    np.testing.assert_array_equal(s, s2)


def test_oracle_cache_block_is_the_token_quantize_of_the_flat_block():
    # one scale for all of a block: the block as one token of the activation quantize
    x = I.activations(64, 128, 4)
    codes, s = oracle.cache_block(x)
    q, s2 = oracle.quantize_act(x.reshape(1, -1))
    np.testing.assert_array_equal(codes.reshape(1, -1), q)
    assert s == s2[0]
    codes, s = oracle.cache_block(np.full((3, 128), 0x0001, np.uint16))  # below 2^-90
    assert s == 0 and not codes.any()


def test_oracle_cache_attention_against_differences_of_the_log_sum():
    # o is the gradient of log sum_j exp(s_j + e . v_j) at e = 0
    rng = np.random.Generator(np.random.PCG64(5))
    n, H, Hkv, L = 3, 4, 2, 20
    q = I.activations(n * H, 128, 6, outliers=False).reshape(n, H, 128)
    k, v = rng.standard_normal((Hkv, L, 128)), rng.standard_normal((Hkv, L, 128))
    cos_t, sin_t = oracle.rope_tables(L, 128)
    pos = np.arange(L - n, L)
    o, bnd, top, peak = oracle.cache_attention(q, pos, k, v, cos_t, sin_t, 0.09, L - n)
    qr = oracle._f32(oracle.rope_rotate(q.reshape(n * H, 128), np.repeat(pos, H), cos_t, sin_t)).astype(np.float64).reshape(n, H, 128)
    assert np.abs(np.abs(qr).max(-1) - top).max() <= 2.0 ** -8 * top.max()
    for i in range(n):
        for h in range(H):
            def lse(e, d):
                q64 = oracle._f32(q).astype(np.float64)[i, h]
                c, s = cos_t[pos[i]].astype(np.float64), sin_t[pos[i]].astype(np.float64)
                t = np.concatenate([q64[:64] * c - q64[64:] * s, q64[64:] * c + q64[:64] * s])
                j = L - n + i + 1
                return np.log(np.exp(0.09 * k[h // 2, :j] @ t + e * v[h // 2, :j, d]).sum())
            for d in (0, 77, 127):
                diff = (lse(1e-4, d) - lse(-1e-4, d)) / 2e-4
                assert abs(diff - o[i, h, d]) <= 1e-6
    assert (np.abs(o) <= bnd + 1e-12).all() and (bnd.max(-1) <= peak + 1e-12).all()
    o0, _, _, _ = oracle.cache_attention(q, pos, k, v, cos_t, sin_t, 0.09, -2)
    assert not o0[:2].any() and np.allclose(o0[2], np.repeat(v[:, 0], 2, 0))
