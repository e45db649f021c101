"""Host-side checks (no GPU needed) of the head norms with the rotation and of
the 4-bit cache's calls: malformed ones are rejected before anything is
launched, empty ones do nothing, and the oracle's definitions hold together."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import oracle
import paper_2608_12932_amd as w
from paper_2608_12932_amd import inputs as I

P = ctypes.c_void_p
EINVAL, OK = w.W4A8_EINVAL, w.W4A8_OK


def at(i, off=0):
    """A fake address, 4 GiB from the others; never dereferenced."""
    return P(((i + 1) << 32) + off)


# ---- the norms with the rotation


def heads(i, **over):
    d = dict(x=at(i), row=6144, head=128, heads=8, gamma=at(i + 1), out=at(i + 2), out_row=1024, out_head=128)
    d.update(over)
    return w._HeadsArgs(*(d[n] for n, _ in w._HeadsArgs._fields_))


def rope(**over):
    d = dict(pos=at(20), n_axes=3, axis=w.rope_axes((24, 20, 20)), rope_cos=at(21), rope_sin=at(22), n_pos=100)
    d.update(over)
    return w._RopeArgs(*(d[n] for n, _ in w._RopeArgs._fields_))


def norm_rope(q=None, k=None, T=4, eps=1e-6, r=None):
    return w.lib().w4a8_qk_norm_rope(heads(0) if q is None else q, heads(10) if k is None else k, T, eps, rope() if r is None else r, None)


def test_norm_rope_rejections():
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert norm_rope(eps=eps) == EINVAL
    assert norm_rope(T=-1) == EINVAL and norm_rope(T=(1 << 20) + 1) == EINVAL
    for over in (dict(x=None), dict(out=None), dict(x=at(0, 8)), dict(out=at(2, 2)), dict(gamma=at(1, 8)), dict(row=-8), dict(row=100), dict(head=4),
                 dict(head=-128), dict(row=1 << 41), dict(heads=-1), dict(heads=4097), dict(out_row=1016), dict(out_head=120), dict(out_row=0),
                 dict(out_head=0), dict(out_row=128)):
        assert norm_rope(q=heads(0, **over)) == EINVAL, over
        assert norm_rope(k=heads(10, **over)) == EINVAL, over
    for over in (dict(pos=None), dict(pos=at(20, 2)), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2), dict(rope_cos=None), dict(rope_sin=at(22, 8)),
                 dict(n_pos=0), dict(n_pos=(1 << 30) + 1), dict(axis=b"\3" * 64)):
        assert norm_rope(r=rope(**over)) == EINVAL, over
    f = w.lib().w4a8_qk_norm_rope
    assert f(heads(0, gamma=None), None, 4, 1e-6, None, None) == EINVAL  # neither a norm nor a rotation
    assert f(heads(0), heads(10, gamma=None), 4, 1e-6, None, None) == EINVAL


def test_norm_rope_overlaps():
    # outputs inside inputs or each other, as far as equal strides or ranges show
    x = 0
    bad = [dict(out=at(x), out_row=6144, out_head=256), dict(out=at(x, 16), out_row=6144), dict(out=at(x, 2 * 7 * 128), out_row=6144),
           dict(out=at(x, 2 * 6144 * 3), out_row=1024)]
    for over in bad:
        assert norm_rope(q=heads(x, **over)) == EINVAL, over
    # q's output where k's input or output is
    assert norm_rope(q=heads(0, out=at(10), out_row=6144)) == EINVAL
    assert norm_rope(q=heads(0, out=at(12))) == EINVAL
    assert norm_rope(q=heads(0, out=at(12, 2 * 7 * 128), out_row=1024)) == EINVAL
    # one matrix's gaps, but not far enough: heads 8 .. 15 of 8 heads more, reaching into the next row
    assert norm_rope(q=heads(0, out=at(0, 2 * (6144 - 1024 + 8)), out_row=6144)) == EINVAL


def test_norm_rope_nothing_to_do():
    f = w.lib().w4a8_qk_norm_rope
    none = dict(x=None, gamma=None, out=None)
    assert norm_rope(q=heads(0, x=None, out=None), k=heads(10, x=None, out=None), T=0) == OK
    assert f(None, None, 4, 1e-6, rope(), None) == OK
    assert f(heads(0, heads=0, **none), heads(10, heads=0, **none), 4, 1e-6, None, None) == OK


def test_rope_axes():
    assert w.rope_axes([64]) == bytes(64)
    assert w.rope_axes((16, 24, 24)) == b"\0" * 16 + b"\1" * 24 + b"\2" * 24
    a = w.rope_axes((24, 20, 20), interleaved=True)
    assert a[:7] == bytes([0, 1, 2, 0, 1, 2, 0]) and a[57:] == bytes([0, 1, 2, 0, 0, 0, 0]) and [a.count(x) for x in range(3)] == [24, 20, 20]
    for bad in ((64, 1), (63,), (16, 16, 16, 8, 8), (), (70, -6)):
        with pytest.raises(ValueError):
            w.rope_axes(bad)
    with pytest.raises(ValueError):
        w.rope_axes((0, 32, 32), interleaved=True)  # 21 pairs of an axis of three


# ---- the cache


def cache(pages=10, Hkv=8, **over):
    d = dict(k_codes=at(0), v_codes=at(1), k_params=at(2), v_params=at(3), n_pages=pages, Hkv=Hkv)
    d.update(over)
    return w._Cache4Args(*(d[n] for n, _ in w._Cache4Args._fields_))


def batch(**over):
    d = dict(starts=at(5), lengths=at(6), table=at(7), max_blocks=16, B=4, T=8, pos=None, rope_cos=None, rope_sin=None, n_pos=0)
    d.update(over)
    return w._BatchArgs(*(d[n] for n, _ in w._BatchArgs._fields_))


BAD_CACHE = [dict(k_codes=None), dict(v_codes=None), dict(k_params=None), dict(v_params=None), dict(k_codes=P(24)), dict(v_codes=P(8)),
             dict(k_params=P(4)), dict(v_params=P(8)), dict(pages=0), dict(pages=1 << 31), dict(Hkv=0), dict(Hkv=4097)]
BAD_BATCH = [dict(starts=None), dict(lengths=None), dict(table=None), dict(starts=P(2)), dict(lengths=P(1)), dict(table=P(6)), dict(max_blocks=0),
             dict(max_blocks=(1 << 24) + 1), dict(B=-1), dict(B=65537), dict(T=-1), dict(T=(1 << 20) + 1)]
NO_CACHE = dict(k_codes=None, v_codes=None, k_params=None, v_params=None)
NO_BATCH = dict(starts=None, lengths=None, table=None)


def test_append_rejections():
    f = w.lib().w4a8_cache4_append
    call = lambda c=None, b=None, k=at(20), kr=6144, kh=128, v=at(21), vr=6144, vh=128: f(  # noqa: E731
        c or cache(), b or batch(), k, kr, kh, v, vr, vh, None)
    for over in BAD_CACHE:
        assert call(c=cache(**over)) == EINVAL, over
    for over in BAD_BATCH:
        assert call(b=batch(**over)) == EINVAL, over
    for over in (dict(k=None), dict(v=None), dict(k=P(8)), dict(kr=-8), dict(kh=4), dict(vr=100), dict(vh=-128), dict(vr=1 << 41)):
        assert call(**over) == EINVAL, over
    assert f(None, batch(), at(20), 128, 128, at(21), 128, 128, None) == EINVAL
    assert f(cache(), None, at(20), 128, 128, at(21), 128, 128, None) == EINVAL
    for over in (dict(T=0), dict(B=0)):
        assert f(cache(**NO_CACHE), batch(**NO_BATCH, **over), None, 0, 0, None, 0, 0, None) == OK


def test_read_rejections():
    f = w.lib().w4a8_cache4_read
    call = lambda c=None, b=None, k=at(20), kr=1024, kh=128, v=at(21), vr=1024, vh=128: f(  # noqa: E731
        c or cache(), b or batch(), k, kr, kh, v, vr, vh, None)
    for over in BAD_CACHE:
        assert call(c=cache(**over)) == EINVAL, over
    for over in BAD_BATCH:
        assert call(b=batch(**over)) == EINVAL, over
    for over in (dict(k=P(8)), dict(v=P(4)), dict(kr=-8), dict(kh=4), dict(vr=100), dict(vr=1 << 41), dict(kr=1016), dict(kh=120), dict(vh=0), dict(vr=0),
                 dict(v=at(20)), dict(v=at(20, 2 * 7 * 1024)), dict(k=at(0)), dict(v=at(3, 1024)), dict(k=at(1, 10 * 8 * 4096 - 16))):
        assert call(**over) == EINVAL, over
    assert call(k=None, v=None) == OK
    for over in (dict(T=0), dict(B=0)):
        assert f(cache(**NO_CACHE), batch(**NO_BATCH, **over), None, 0, 0, None, 0, 0, None) == OK


def test_attention_rejections():
    f = w.lib().w4a8_cache4_attention
    big = (at(22), 1 << 30)
    call = lambda c=None, b=None, q=at(20), qr=6144, qh=128, H=32, scale=0.1, max_len=1000, o=at(21), orow=4096, oh=128, ws=big: f(  # noqa: E731
        c or cache(), b or batch(), q, qr, qh, H, scale, max_len, o, orow, oh, *ws, None)
    for over in BAD_CACHE:
        assert call(c=cache(**over)) == EINVAL, over
    for over in BAD_BATCH:
        assert call(b=batch(**over)) == EINVAL, over
    for over in (dict(q=None), dict(o=None), dict(q=P(8)), dict(qr=-8), dict(qh=4), dict(H=0), dict(H=30), dict(H=8192), dict(max_len=0),
                 dict(max_len=16 * 64 + 1), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-float("inf"))):
        assert call(**over) == EINVAL, over
    for orow, oh in ((4096, 0), (0, 128), (128, 128), (4096, 120), (4088, 128), (128, 1016)):
        assert call(orow=orow, oh=oh) == EINVAL, (orow, oh)
    for T, H, Hkv in ((1 << 20, 4096, 1), ((1 << 20) - 1, 4096, 8), (1 << 20, 514, 2)):
        assert call(c=cache(Hkv=Hkv), b=batch(T=T), H=H, orow=H * 128) == w.W4A8_EUNSUPPORTED, (T, H, Hkv)
    # which calls are split is a matter of what they cost: 1000 long this one is not
    # (16 blocks are four rounds of four waves, less than a merge), 4096 long it is
    need = w.w4a8_cache4_attention_workspace_bytes(4, 8, 32, 8, 4096)
    assert need > 64 * 1024
    for ws in ((None, 0), (at(22), need - 1), (at(22, 16), need)):
        assert call(b=batch(max_blocks=64), max_len=4096, ws=ws) == EINVAL
    for over in (dict(T=0), dict(B=0)):
        assert f(cache(**NO_CACHE), batch(**NO_BATCH, **over), None, 0, 0, 32, 0.1, 1000, None, 0, 0, None, 0, None) == OK


def test_the_largest_finite_numbers_are_taken():
    top = float(np.finfo(np.float32).max)
    for scale in (top, -top, 3.401e38):
        assert w.lib().w4a8_cache4_attention(cache(), batch(T=0), None, 0, 0, 32, scale, 1000, None, 0, 0, None, 0, None) == OK
    for eps in (top, 3.401e38):
        assert norm_rope(T=0, eps=eps) == OK


def test_attention_output_over_inputs():
    # T 8, H 32, q a view of a fused projection's rows: over q, in its gaps but not far enough, over the cache
    f = w.lib().w4a8_cache4_attention
    call = lambda q=at(20), qr=6144, qh=128, o=at(21), orow=4096, oh=128, T=8, H=32: f(  # noqa: E731
        cache(), batch(T=T), q, qr, qh, H, 0.1, 1000, o, orow, oh, at(22), 1 << 30, None)
    for over in (dict(o=at(20), orow=6144), dict(o=at(20)), dict(o=at(20), qr=4096), dict(o=at(20, 2 * 7 * 6144), orow=6144),
                 dict(o=at(20, 2 * (4096 - 8)), orow=6144), dict(o=at(20, 2 * (6144 - 4096)), orow=6144),
                 dict(q=at(21, 2 * (7 * 4096 + 31 * 128 + 120))), dict(q=at(21), qr=0, qh=0),  # one row for all
                 dict(q=at(20), qr=128, qh=1024, o=at(20, 2 * 1024), orow=128, oh=1024), dict(T=1, o=at(20, 2 * 128 * 31))):
        assert call(**over) == EINVAL, over
    for i, n in enumerate((4096, 4096, 512, 512)):  # codes, codes, parameters, parameters of a page's head
        for off in (0, 10 * 8 * n - 16):
            assert call(o=at(i, off)) == EINVAL, (i, off)
        assert call(o=P(((i + 1) << 32) - 16)) == EINVAL, i


def test_workspace_bytes():
    f = w.w4a8_cache4_attention_workspace_bytes
    assert f(64, 64, 32, 8, 64) == 0  # one block: nothing to split
    for bad in ((-1, 8, 32, 8, 100), (4, -1, 32, 8, 100), (4, 8, 30, 8, 100), (4, 8, 32, 0, 100), (4, 8, 32, 8, 0), (0, 8, 32, 8, 100),
                (4, 0, 32, 8, 100), (4, 1 << 21, 32, 8, 100)):
        assert f(*bad) == 0, bad


def test_binding_checks_before_the_device():
    x = torch.zeros(1, 8, 128, dtype=torch.bfloat16)
    c = w.KVCache4.empty(2, 8, device="cpu")
    assert [tuple(t.shape) for t in c] == [(2, 8, 4, 16, 16), (2, 8, 8, 2, 16, 4), (2, 8, 2, 64, 2), (2, 8, 2, 2, 64)]
    i, s, t = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, 64)
    for call in (lambda: w.w4a8_cache4_append(x, x, c, s, i, i[None]), lambda: w.w4a8_cache4_read(c, s, i, i[None], 1),
                 lambda: w.w4a8_cache4_attention(x, c, s, i, i[None], 0.1), lambda: w.w4a8_qk_norm_rope(x, x, None, None, 1e-6, i, t, t)):
        with pytest.raises(TypeError):  # not device tensors
            call()
    assert w.w4a8_qk_norm_rope(None, None, None, None, 1e-6, i, t, t) == (None, None)
    for bad in (c._replace(k_codes=c.k_codes[:, :, :2]), c._replace(v_codes=c.v_codes[:1]), c._replace(k_params=c.v_params),
                c._replace(v_params=c.k_params)):
        with pytest.raises(ValueError):
            w._cache4_args(bad)


# ---- the oracle


def f16(x: Fraction) -> float:
    """A rational number rounded to fp16, to nearest, ties to even."""
    if x == 0:
        return 0.0
    e = max(math.frexp(float(abs(x)))[1] - 1, -14)
    if abs(x) < Fraction(2) ** e and e > -14:
        e -= 1
    step = Fraction(2) ** (e - 10)
    return float(round(x / step) * step)  # round() of a Fraction ties to even


def test_oracle_quantize_by_rational_arithmetic():
    x = I.activations(6, 128, 11).reshape(6, 128).copy()
    x[0] = 0x3F80  # all equal
    x[1, :64] = 0x0001  # below fp16
    x[2, 3], x[2, 70], x[2, 71] = 0x7F80, 0xFF80, 0x7FC0  # infinities and NaN
    codes, s, b = oracle.cache4_quantize(x)
    v = oracle.cache4_values(codes, s, b)
    xs = oracle._f32(x).astype(np.float64)
    xs = np.clip(np.where(np.isnan(xs), 0, xs), -16384, 16384)
    assert np.isfinite(s).all() and np.isfinite(b).all() and codes.max() <= 15
    for r in range(6):
        for g in range(2):
            part = [Fraction(float(a)) for a in xs[r, 64 * g:64 * g + 64]]
            lo, hi = min(part), max(part)
            # the fp32 steps in between can move a result only at a tie of fp16 that is closer than 2^-24
            assert abs(float(s[r, g]) - f16((hi - lo) / 15)) <= 2.0 ** -11 * float(hi - lo) / 15 + 2.0 ** -24
            for d, a in enumerate(part):
                c = int(codes[r, 64 * g + d])
                val = f16(Fraction(float(s[r, g])) * (16 + c) + Fraction(float(b[r, g])))
                assert v[r, 64 * g + d] == val
                # half a step, the offset's and the value's rounding to fp16, the scale's at the group's ends
                lim = Fraction(float(s[r, g])) * Fraction(51, 100) + Fraction(float(abs(b[r, g]))) / 2048 + abs(a) / 1024 + 15 * Fraction(
                    float(s[r, g])) / 2048 + Fraction(17, 2 ** 24)
                assert abs(Fraction(val) - a) <= lim, (r, g, d)
    assert not codes[0].any() and (v[0] == 1.0).all()


def test_oracle_layout_of_words():
    rng = np.random.Generator(np.random.PCG64(12))
    codes = rng.integers(0, 16, (64, 128))
    keys = np.zeros((4, 16, 16), np.uint32)
    vals = np.zeros((8, 2, 16, 4), np.uint32)
    order = [0, 16, 4, 20, 8, 24, 12, 28]  # the bits of elements 0 .. 7
    for t in range(64):
        for d in range(128):
            keys[t % 4, t // 4, d // 8] |= np.uint32(codes[t, d] << order[d % 8])
            vals[t // 8, (d % 8) // 4, d // 8, d % 4] |= np.uint32(codes[t, d] << order[t % 8])
    np.testing.assert_array_equal(oracle.cache4_codes(keys, False), codes)
    np.testing.assert_array_equal(oracle.cache4_codes(vals, True), codes)


def test_oracle_norm_rope_is_a_rotation_of_the_norm():
    x = I.activations(3 * 4, 128, 13, outliers=False).reshape(3, 4, 128)
    g = I.activations(1, 128, 14, outliers=False)[0]
    cos_t, sin_t = oracle.rope_tables(50, 128)
    pos, axis = np.array([[3, 40, 77], [0, 1, -2]]), np.arange(64) % 2
    y, mag = oracle.qk_norm_rope(x, g, 1e-6, pos, axis, cos_t, sin_t)
    h, _ = oracle.qk_norm_rope(x, g, 1e-6, None, axis, cos_t, sin_t)
    z, rot = h[..., :64] + 1j * h[..., 64:], y[..., :64] + 1j * y[..., 64:]
    p = np.array([[3, 40, 49], [0, 1, 0]])  # clamped
    ang = p[axis].T[:, None] * 10000.0 ** (-np.arange(64) / 64)
    np.testing.assert_allclose(rot, z * np.exp(1j * ang), rtol=0, atol=2.0 ** -22 * np.abs(h).max())
    assert (np.abs(y) <= mag + 1e-12).all()
    # gradient of sum_d y_d w_d in x by differences, against the norm's formula: the norm is of the mean square
    n, _ = oracle.qk_norm_rope(x, None, 1e-6, pos, axis, cos_t, sin_t)
    np.testing.assert_allclose((n ** 2).sum(-1), (oracle._f32(x).astype(np.float64) ** 2).sum(-1), rtol=1e-6)
    np.testing.assert_allclose(((h / oracle._f32(g)) ** 2).mean(-1), 1.0, rtol=1e-5)
