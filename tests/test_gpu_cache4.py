"""The 4-bit cache (w4a8_cache4_append, w4a8_cache4_read, w4a8_cache4_attention)
against the oracle.

Append and read are exact: every step is an IEEE operation on both sides, so
codes, scales, offsets and values have to be equal.

Tolerance of the attention, derived.  Against fp64 on the values that the codes
stand for, with A = |scale| sum_d |q_d| |k_d| at its largest over the keys, the
kernel
  - forms scores in fp32: 128 exact products, each addition within 2^-23 of the
    sum of magnitudes so far, 2^-16 A in all; the factor and the exponent, 2^-22
    A; query elements below 2^-28 of the row's largest are off by 2^-39 of it at
    most, |scale| top 2^-39 max_j |k_j|_1: d together, and a weight is off by a
    factor within exp(+-2 d) (its own score and the total's), 2 d (1 + 2 d);
  - rounds weights to fp16, 2^-11 of each, and exponentials to 2^-19;
  - has fp16's smallest weights: the largest lies in [2^12, 2^15], below 2^-14
    half a step is 2^-25, so 2^-37 of the largest at most: with N keys N 2^-37
    max_j P_ij max |v|;
  - adds weighted values and weights in fp32, N / 32 products of 32 after each
    other: (N / 32 + 40) 2^-23 of the sum of magnitudes, twice;
  - rounds the output to bf16, 2^-8 of it.
With B = sum_j P_ij |v_jd| and T = N max_j P_ij max |v|:
  |o - o64| <= 2^-8 |o64| + (1 + 2^-8) ((2^-11 + 2^-19 + 2 d (1 + 2 d) + (N / 16 + 80) 2^-23) B + 2^-37 T)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_12932_amd as w
from paper_2608_12932_amd import inputs as I
from helpers import bf16_dev, dev, to_np_bits

pytestmark = pytest.mark.gpu

D, BLK = 128, w.CACHE_BLOCK
SCALE = D ** -0.5


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev())


def reference(q, k, v, lens, scale):
    """o64 and the tolerance above of rows q [n][D] that see the first lens[i] of
    k, v [L][D], all fp64 on the device."""
    n, L = len(q), len(k)
    if L == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    hidden = torch.arange(L, device=q.device)[None] >= lens[:, None]
    s = (q @ k.t() * scale).masked_fill(hidden, -float("inf"))
    some = (lens > 0)[:, None]
    p = torch.where(some, torch.softmax(s, 1), 0.0).nan_to_num()
    o, B = p @ v, p @ v.abs()
    A = abs(scale) * (q.abs() @ k.abs().t()).masked_fill(hidden, 0.0).amax(1)
    d = A * (2.0 ** -16 + 2.0 ** -22) + abs(scale) * q.abs().amax(1) * 2.0 ** -39 * k.abs().sum(1).max()
    N = lens.clamp(0, L).double()
    T = N * (p * v.abs().amax(1)).amax(1)
    c = 2.0 ** -11 + 2.0 ** -19 + 2 * d * (1 + 2 * d) + (N / 16 + 80) * 2.0 ** -23
    return o, 2.0 ** -8 * o.abs() + (1 + 2.0 ** -8) * (c[:, None] * B + 2.0 ** -37 * T[:, None])


class Model:
    """Sequences of bf16 keys and values, and a cache that is filled with them
    through the calls under test.  What no token fills holds NaN parameters."""

    def __init__(self, Hkv, B, max_len, seed=0, pages=None):
        self.Hkv, self.B, self.blocks = Hkv, B, -(-max_len // BLK)
        self.rng = np.random.Generator(np.random.PCG64(seed))
        n = pages or B * self.blocks + 3
        self.cache = w.KVCache4.empty(n, Hkv, device=dev())
        self.cache.k_codes.fill_(0x77777777)
        self.cache.v_codes.fill_(0x77777777)
        self.cache.k_params.fill_(float("nan"))
        self.cache.v_params.fill_(float("nan"))
        self.table = self.rng.permutation(n)[:B * self.blocks].reshape(B, self.blocks).astype(np.int32)
        self.k = [np.zeros((0, Hkv, D), np.uint16) for _ in range(B)]
        self.v = [np.zeros((0, Hkv, D), np.uint16) for _ in range(B)]

    def values(self, n, H, spread=0.5):
        return I.to_bf16_bits((self.rng.standard_normal((n, H, D)) * np.exp(spread * self.rng.standard_normal((1, H, D)))).astype(np.float32))

    def batch(self, new):
        return i32(np.concatenate([[0], np.cumsum(new)])), i32([len(k) for k in self.k]), i32(self.table)

    def append(self, new, k=None, v=None, behind=0):
        """Appends new[b] tokens to each sequence, k and v being views of one
        matrix, with `behind` rows after the last."""
        T = sum(new) + behind
        k = self.values(T, self.Hkv) if k is None else k
        v = self.values(T, self.Hkv) if v is None else v
        at = 0
        for b, n in enumerate(new):
            self.k[b], self.v[b] = np.concatenate([self.k[b], k[at:at + n]]), np.concatenate([self.v[b], v[at:at + n]])
            at += n
        qkv = bf16_dev(np.concatenate([self.values(T, 3), k, v], 1).reshape(T, -1)).view(T, 3 + 2 * self.Hkv, D)
        w.w4a8_cache4_append(qkv[:, 3:3 + self.Hkv], qkv[:, 3 + self.Hkv:], self.cache, *self.batch(new))
        torch.cuda.synchronize()
        return self

    def cut(self, b, L):
        self.k[b], self.v[b] = self.k[b][:L], self.v[b][:L]

    def held(self, b):
        """Keys and values [L][Hkv][D] that sequence b's codes stand for."""
        return tuple(oracle.cache4_values(*oracle.cache4_quantize(x[b])) for x in (self.k, self.v))

    def check_pages(self):
        """Every code and parameter of every token, and what no token filled."""
        c = self.cache
        kc, vc = c.k_codes.cpu().numpy(), c.v_codes.cpu().numpy()
        kp, vp = c.k_params.cpu().numpy(), c.v_params.cpu().numpy().transpose(0, 1, 2, 4, 3)  # [..][group][token][2]
        for b in range(self.B):
            want = [oracle.cache4_quantize(x[b]) for x in (self.k, self.v)]
            L = len(self.k[b])
            for blk in range(-(-L // BLK)):
                p, n = int(self.table[b, blk]), min(L - blk * BLK, BLK)
                at = slice(blk * BLK, blk * BLK + n)
                for h in range(self.Hkv):
                    for name, words, par, (codes, s, off) in (("k", kc, kp, want[0]), ("v", vc, vp, want[1])):
                        where = (name, b, blk, h)
                        got = oracle.cache4_codes(words[p, h], name == "v")
                        np.testing.assert_array_equal(got[:n], codes[at, h], err_msg=str(where))
                        np.testing.assert_array_equal(par[p, h, :, :n, 0].T.view(np.uint16), s[at, h].view(np.uint16), err_msg=str(where))
                        np.testing.assert_array_equal(par[p, h, :, :n, 1].T.view(np.uint16), off[at, h].view(np.uint16), err_msg=str(where))
                        assert (got[n:] == 7).all() and np.isnan(par[p, h, :, n:]).all(), where
        used = {int(self.table[b, i]) for b in range(self.B) for i in range(-(-len(self.k[b]) // BLK))}
        rest = [p for p in range(kc.shape[0]) if p not in used]
        assert (kc[rest] == 0x77777777).all() and (vc[rest] == 0x77777777).all() and np.isnan(kp[rest]).all() and np.isnan(vp[rest]).all()

    def attend(self, q, new, scale=SCALE, **kw):
        return w.w4a8_cache4_attention(q, self.cache, *self.batch(new), scale, **kw)

    def check_attention(self, new, H, scale=SCALE, q=None, label="", **kw):
        T = sum(new)
        q = self.values(T, H, 0.3) if q is None else q
        qd = bf16_dev(q)
        got = self.attend(qd, new, scale, **kw)
        torch.cuda.synchronize()
        self.compare(got, q, new, scale, label)
        return got

    def compare(self, got, q, new, scale, label=""):
        H, at = q.shape[1], 0
        q64 = torch.from_numpy(oracle._f32(q).astype(np.float64)).to(dev())
        for b, n in enumerate(new):
            k, v = (torch.from_numpy(x).to(dev()) for x in self.held(b))
            L = len(k)
            lens = torch.arange(L - n, L, device=dev()) + 1
            for h in range(H):
                kv = h // (H // self.Hkv)
                o, tol = reference(q64[at:at + n, h], k[:, kv].contiguous(), v[:, kv].contiguous(), lens, scale)
                off = (got[at:at + n, h].double() - o).abs()
                bad = ~(off <= tol)
                assert not bad.any(), (label, b, h, bad.nonzero()[:3].tolist(), off[bad][:3].tolist(), tol[bad][:3].tolist())
            at += n


# ---- append and read


@pytest.mark.parametrize("steps", [[1] * 12, [7, 1, 9], [64, 64, 1], [63, 2, 70], [130], [1, 200, 5], [8, 8, 16]])
def test_append_steps(steps):
    m = Model(3, 1, 300, seed=sum(steps))
    for n in steps:
        m.append([n]).check_pages()


def test_append_ragged_batch():
    m = Model(2, 6, 300, seed=1)
    m.append([5, 0, 64, 1, 17, 130], behind=3).check_pages()
    m.append([1, 1, 1, 1, 1, 1]).check_pages()
    m.append([0, 33, 0, 71, 2, 0]).check_pages()


def test_append_many_sequences():
    m = Model(1, 200, 70, seed=2)
    m.append([b % 5 for b in range(200)])
    m.append([1] * 200).check_pages()


def test_append_does_not_depend_on_the_chunks():
    a, b = Model(2, 1, 200, seed=3), Model(2, 1, 200, seed=3)
    k, v = a.values(150, 2), a.values(150, 2)
    b.table = a.table
    a.append([150], k, v)
    at = 0
    for n in (1, 3, 60, 1, 50, 35):
        b.append([n], k[at:at + n], v[at:at + n])
        at += n
    for x, y in zip(a.cache, b.cache):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("L,back", [(70, 6), (70, 7), (64, 1), (129, 129), (200, 137), (8, 3)])
def test_tokens_taken_back(L, back):
    m = Model(2, 2, 300, seed=L)
    m.append([L, 10])
    m.cut(0, L - back)
    m.append([back + 5, 0])  # over the ones taken back, and past them
    m.check_pages()
    m.cut(0, L - back)
    m.append([1, 1])
    m.check_attention([1, 1], 4)


def test_more_new_tokens_than_the_sequence_holds():
    # the last of them are held
    m = Model(2, 2, 64, seed=40)
    k, v = m.values(30, 2), m.values(30, 2)
    kd, vd = bf16_dev(k), bf16_dev(v)
    w.w4a8_cache4_append(kd, vd, m.cache, i32([0, 20, 30]), i32([13, 10]), i32(m.table))
    m.k, m.v = [k[7:20], k[20:]], [v[7:20], v[20:]]
    m.check_pages()


def test_special_values():
    m = Model(1, 1, 64, seed=4)
    k, v = m.values(16, 1), m.values(16, 1)
    k[0] = 0
    k[1] = 0x3F80                 # equal: held exactly
    k[2, 0, :64] = 0x0001         # below fp16
    k[3, 0, 5] = 0x7F80           # infinity, counted as 2^14
    k[4, 0, 70] = 0xFF80
    k[5, 0, ::3] = 0x7FC0         # NaN, counted as 0
    k[6] = 0x7F7F
    k[7, 0, ::2] = 0xC680         # -2^14 among small ones
    k[8, 0, :64], k[8, 0, 3] = 0x4680, 0xC680  # the widest range
    k[9, 0] = 0x4680
    k[9, 0, 1] = 0x467F           # one step of bf16 apart, far from 0
    k[10] = 0x3380                # 2^-24
    k[11, 0, ::2] = 0x3500
    v[:] = k[::-1]
    m.append([16], k, v)
    for t in m.cache[2:]:
        assert torch.isfinite(t[int(m.table[0, 0])].float()[..., :16 if t is m.cache[3] else 2]).any()
    m.check_pages()
    kv = m.held(0)
    assert all(np.isfinite(x).all() for x in kv)
    read(m, [16])


def read(m, new, **kw):
    rows = sum(new)
    k, v = w.w4a8_cache4_read(m.cache, *m.batch(new), rows, **kw)
    torch.cuda.synchronize()
    at = 0
    for b, n in enumerate(new):
        L = len(m.k[b])
        for got, x in zip((k, v), m.held(b)):
            np.testing.assert_array_equal(to_np_bits(got[at:at + n].contiguous()), I.to_bf16_bits(x[L - n:].astype(np.float32)))
        at += n
    return k, v


@pytest.mark.parametrize("lengths,new", [([1], [1]), ([5, 70, 129], [5, 70, 129]), ([100, 64, 200], [3, 64, 121]), ([0, 9], [0, 4]), ([1000], [1000])])
def test_read(lengths, new):
    m = Model(3, len(lengths), max(lengths), seed=5)
    m.append(lengths)
    read(m, new)


def test_read_layouts_and_rows_of_no_sequence():
    m = Model(3, 2, 100, seed=6).append([70, 20])
    want = read(m, [70, 20])
    kt = torch.full((3, 100, D), 7.0, dtype=torch.bfloat16, device=dev())  # [Hkv][rows][128]
    big = torch.full((100, 9, D), 7.0, dtype=torch.bfloat16, device=dev())
    k, v = w.w4a8_cache4_read(m.cache, *m.batch([70, 20]), 100, k_out=kt.transpose(0, 1), v_out=big[:, 4:7])
    assert torch.equal(kt[:, :90].transpose(0, 1), want[0]) and torch.equal(big[:90, 4:7], want[1])
    assert (kt[:, 90:] == 7).all() and (big[90:] == 7).all() and (big[:, :4] == 7).all() and (big[:, 7:] == 7).all()
    # more rows than tokens: those before the first token are left as they are
    starts = i32([0, 75, 95])
    k.fill_(7.0)
    w.w4a8_cache4_read(m.cache, starts, *m.batch([0, 0])[1:], 100, k_out=k, v_out=v)
    assert (k[:5] == 7).all() and torch.equal(k[5:75], want[0][:70]) and torch.equal(k[75:95], want[0][70:]) and (k[95:] == 7).all()
    # a page out of the pool: zeros
    m.table[0, 0] = 1 << 20
    k, v = w.w4a8_cache4_read(m.cache, *m.batch([70, 20]), 90)
    assert not k[:64].any() and not v[:64].any() and torch.equal(k[64:], want[0][64:]) and torch.equal(v[64:], want[1][64:])


def test_read_feeds_the_streaming_attention():
    # the cache's exact values in the layout of w4a8_stream_attention, which then agrees with the attention over codes
    m = Model(2, 1, 200, seed=7).append([200])
    kt, vt = (torch.empty(2, 200, D, dtype=torch.bfloat16, device=dev()) for _ in range(2))
    w.w4a8_cache4_read(m.cache, *m.batch([200]), 200, k_out=kt.transpose(0, 1), v_out=vt.transpose(0, 1))
    q = bf16_dev(m.values(50, 8, 0.3))
    one, zero = torch.ones(1, 64, device=dev()), torch.zeros(1, 64, device=dev())
    p = i32(np.arange(200))
    o = w.w4a8_stream_attention(q.transpose(0, 1).contiguous(), kt, vt, p[150:].contiguous(), p, one.expand(200, 64).contiguous(),
                                zero.expand(200, 64).contiguous(), SCALE)
    got = m.attend(q, [50])
    # both round weights (bf16 there), values (to bf16 there) and outputs: 3 half steps of bf16 of the values' size
    assert (got.float() - o.transpose(0, 1).float()).abs().max() <= 3 * 2.0 ** -8 * vt.float().abs().max()


# ---- attention


@pytest.mark.parametrize("H,Hkv", [(32, 8), (28, 4), (16, 16), (8, 1), (40, 8), (24, 1), (1, 1)])
def test_decode(H, Hkv):
    m = Model(Hkv, 3, 400, seed=H)
    m.append([400, 65, 1])
    m.check_attention([1, 1, 1], H)


@pytest.mark.parametrize("L,n", [(1, 1), (2, 2), (63, 1), (64, 1), (64, 64), (65, 2), (127, 3), (128, 1), (129, 129), (300, 17)])
def test_lengths(L, n):
    m = Model(2, 1, L, seed=L + n)
    m.append([L])
    m.check_attention([n], 8)


@pytest.mark.parametrize("H,Hkv,n,L", [(32, 8, 16, 700), (28, 4, 33, 500), (8, 1, 40, 333), (4, 4, 150, 400), (32, 8, 300, 1100), (16, 2, 130, 2100)])
def test_chunks(H, Hkv, n, L):
    m = Model(Hkv, 1, L, seed=n)
    m.append([L])
    m.check_attention([n], H)


def test_mixed_batch():
    lengths, new = [1, 700, 64, 333, 1300, 40], [1, 33, 64, 1, 7, 0]
    m = Model(4, 6, 1300, seed=8)
    m.append(lengths)
    m.check_attention(new, 28)


def test_long_cache():
    m = Model(2, 1, 20000, seed=9)
    m.append([20000])
    m.check_attention([1], 8, workspace=w.Workspace())
    m.check_attention([5], 8, workspace=w.Workspace())


def test_every_split_gives_the_same_attention():
    m = Model(2, 1, 3000, seed=10)
    m.append([3000])
    for max_len in (1, 64, 200, 1000, 3000):  # decides the splits alone
        m.check_attention([1], 8, max_len=max_len, label=str(max_len))
        m.check_attention([40], 8, max_len=max_len, label=str(max_len))


def splits_of(B, T, H, Hkv, max_len):
    """The splits of a call, by the partial results that its workspace holds."""
    need = w.w4a8_cache4_attention_workspace_bytes(B, T, H, Hkv, max_len)
    return (need - 65536) // (T * H * (D + 2) * 4) if need else 1


@pytest.mark.parametrize("new", [[1, 1], [9, 40]])
def test_numbers_of_splits(new):
    # one call at the plans of lengths from one block to all of them: empty splits, one block a split, many
    m = Model(2, 2, 12000, seed=37)
    m.append([12000, 5000])
    q = m.values(sum(new), 8)
    qd, seen = bf16_dev(q), set()
    for max_len in (64, 1300, 1700, 2300, 3000, 4500, 6000, 8000, 12000):
        S = splits_of(2, sum(new), 8, 2, max_len)
        if S in seen:
            continue
        seen.add(S)
        print(f"[case] {new} max_len={max_len} splits={S}", flush=True)
        out = m.attend(qd, new, max_len=max_len)
        m.compare(out, q, new, SCALE, f"{S} splits")
        for _ in range(5):
            assert torch.equal(m.attend(qd, new, max_len=max_len), out), S
    assert 1 in seen and len(seen) >= 4, seen


@pytest.mark.parametrize("scale", [0.3, -SCALE, 0.0, -0.0, 1e-30])
def test_scale_of_any_sign(scale):
    m = Model(2, 2, 200, seed=11)
    m.append([200, 70])
    m.check_attention([1, 20], 8, scale=scale)


@pytest.mark.parametrize("scale", [2.3e38, 2.4e38, 3.3e38, -3.3e38])
@pytest.mark.parametrize("n", [1, 40])
def test_scales_near_the_largest(n, scale):
    # |scale| log2(e) passes fp32 from 2.36e38 on; scale times the queries' elements does not
    m = Model(2, 1, 200, seed=38)
    m.append([200])
    q = I.to_bf16_bits((oracle._f32(m.values(n, 8, 0.3)) * np.float32(2.0 ** -128)).astype(np.float32))  # subnormal, in steps of 2^-133
    q[:, 3] = 0  # every token counts alike
    assert np.abs(oracle._f32(q).astype(np.float64) * scale).max() < 2.0 ** 7
    m.check_attention([n], 8, scale=scale, q=q)


def test_rows_that_see_nothing():
    m = Model(2, 3, 100, seed=12)
    m.append([100, 5, 20])
    q = bf16_dev(m.values(30, 8))
    # 12 new tokens of a sequence of 5: the first seven lie before its first token; a length of 0
    starts, lengths, table = i32([0, 10, 22, 30]), i32([100, 5, 0]), i32(m.table)
    out = torch.full((30, 8, D), 9.0, dtype=torch.bfloat16, device=dev())
    w.w4a8_cache4_attention(q, m.cache, starts, lengths, table, SCALE, out=out)
    assert not out[10:17].any() and not out[22:30].any() and out[17:22].any(-1).all()
    k, v = (torch.from_numpy(x).to(dev()) for x in m.held(1))
    for i in range(5):
        for h in range(8):
            o, tol = reference(q[17 + i:18 + i, h].double(), k[:, h // 4], v[:, h // 4], torch.tensor([i + 1], device=dev()), SCALE)
            assert ((out[17 + i, h].double() - o[0]).abs() <= tol[0]).all()


@pytest.mark.parametrize("new", [[1, 1], [50, 30]])
def test_rows_of_no_sequence_stay(new):
    m = Model(2, 2, 300, seed=13)
    m.append([300, 100])
    T = sum(new)
    q = bf16_dev(m.values(T + 9, 8))
    for max_len in (64, 300):
        out = torch.full((T + 9, 8, D), 9.0, dtype=torch.bfloat16, device=dev())
        starts, lengths, table = m.batch(new)
        w.w4a8_cache4_attention(q, m.cache, starts + 4, lengths, table, SCALE, out=out, max_len=max_len)
        assert (out[:4] == 9).all() and (out[T + 4:] == 9).all()
        assert torch.equal(out[4:T + 4], w.w4a8_cache4_attention(q[4:T + 4], m.cache, starts, lengths, table, SCALE, max_len=max_len))


@pytest.mark.parametrize("n", [1, 40])
def test_what_lies_behind_a_sequence_is_not_seen(n):
    # pages that other tokens, infinities and NaN have been in: the model's pages hold NaN parameters behind the last token
    m = Model(2, 1, 200, seed=14)
    m.append([133])
    a = m.check_attention([n], 8)
    for t, x in ((m.cache.k_params, float("inf")), (m.cache.v_params, float("-inf"))):
        t[torch.isnan(t)] = x
    m.cache.k_codes[m.cache.k_codes == 0x77777777] = -1
    assert torch.isfinite(a.float()).all()
    m.check_attention([n], 8)


@pytest.mark.parametrize("n", [1, 30])
def test_queries_that_are_no_numbers(n):
    m = Model(2, 1, 200, seed=15)
    m.append([200])
    q = m.values(n, 8)
    clean = m.attend(bf16_dev(q), [n])
    bad = q.copy()
    bad[0, 1, 3], bad[n - 1, 6, 100] = 0x7FC0, 0x7F80
    got = m.attend(bf16_dev(bad), [n])
    keep = torch.ones(n, 8, dtype=torch.bool)
    keep[0, 1] = keep[n - 1, 6] = False
    assert torch.equal(got[keep], clean[keep]) and torch.isnan(got[0, 1]).all() and torch.isnan(got[n - 1, 6]).all()


@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 26, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("n", [1, 40])
def test_large_scores(size, n):
    # scores far apart: the heaviest key alone counts, whichever block it is in
    m = Model(1, 1, 300, seed=16)
    k, v = m.values(300, 1), m.values(300, 1)
    k[:] = 0
    for t in range(300):
        k[t, 0, 0] = I.to_bf16_bits(np.float32([1.0 + t / 4]))[0]
    m.append([300], k, v)
    q = np.zeros((n, 4, D), np.uint16)
    for i, s in enumerate((size, -size, size, -size)):
        q[:, i, 0] = I.to_bf16_bits(np.float32([s]))[0]
    got = m.attend(bf16_dev(q), [n], 1.0)
    hk, hv = m.held(0)
    hv = torch.from_numpy(hv).to(dev())[:, 0]
    for i in range(n):
        seen = torch.from_numpy(hk[:300 - n + i + 1, 0, 0].copy()).to(dev())
        for h, s in enumerate((size, -size, size, -size)):
            y = seen * s
            p = torch.softmax(y, 0)  # ties share
            # keys are 1/4 apart and more: with 2^10 the next one is e^-100 lighter
            o = p @ hv[:len(seen)]
            b = p @ hv[:len(seen)].abs()
            assert ((got[i, h].double() - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** -10 * b).all(), (i, h)


@pytest.mark.parametrize("n", [1, 30])
def test_rows_beside_large_ones(n):
    # a row's result does not depend on the rows that share its wave
    m = Model(1, 1, 300, seed=17)
    m.append([300])
    q = m.values(n, 8)
    alone = m.attend(bf16_dev(q), [n])
    q[:, 3] = I.to_bf16_bits((oracle._f32(q[:, 3]) * np.float32(2.0 ** 30)).astype(np.float32))
    both = m.attend(bf16_dev(q), [n])
    keep = [h for h in range(8) if h != 3]
    assert torch.equal(alone[:, keep], both[:, keep]) and torch.isfinite(both.float()).all()


def test_growing_and_falling_scores():
    # the running maximum moves in every block, or never again after the first
    for order in (1, -1):
        m = Model(1, 1, 900, seed=18)
        k, v = m.values(900, 1), m.values(900, 1)
        ramp = np.linspace(0.1, 30, 900)[::order].astype(np.float32)
        k[:] = 0
        k[:, 0, 7] = I.to_bf16_bits(ramp)
        m.append([900], k, v)
        q = np.zeros((3, 4, D), np.uint16)
        q[..., 7] = 0x4000
        m.check_attention([3], 4, q=q, scale=1.0)


def test_queries_of_wide_range():
    m = Model(1, 1, 130, seed=19)
    m.append([130])
    q = m.values(4, 2)
    q[0, 0] = I.to_bf16_bits((oracle._f32(q[0, 0]) * np.float32(2.0 ** -120)).astype(np.float32))
    q[1, 0, :100] = I.to_bf16_bits((oracle._f32(q[1, 0, :100]) * np.float32(2.0 ** -27)).astype(np.float32))
    q[2, 0] = 0
    q[3, 1] = I.to_bf16_bits((oracle._f32(q[3, 1]) * np.float32(2.0 ** 100)).astype(np.float32))
    for scale in (SCALE, 2.0 ** -103):
        m.check_attention([4], 2, q=q if scale != SCALE else np.where(np.arange(4)[:, None, None] == 3, 0, q).astype(np.uint16), scale=scale)


def test_pages_out_of_range_are_not_seen():
    for n in (1, 40):
        m = Model(2, 1, 400, seed=20)
        m.append([400])
        k, v = m.held(0)
        gone = [1, 4]
        m.table[0, gone] = [-1, 1 << 30]
        q = m.values(n, 8)
        got = m.attend(bf16_dev(q), [n])
        left = [t for t in range(400) if t // BLK not in gone]
        for i in range(n):
            see = [t for t in left if t <= 400 - n + i]
            for h in range(8):
                o, tol = reference(torch.from_numpy(oracle._f32(q[i:i + 1, h]).astype(np.float64)).to(dev()), torch.from_numpy(k[see, h // 4]).to(dev()),
                                   torch.from_numpy(v[see, h // 4]).to(dev()), torch.tensor([len(see)], device=dev()), SCALE)
                assert ((got[i, h].double() - o[0]).abs() <= tol[0]).all(), (n, i, h)
        m.append([5])  # tokens without a page are not held, the others are
        m.table[0, 6] = -1
        before = [t.clone() for t in m.cache]
        m.append([3])
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, m.cache))


def test_arrays_out_of_range_reach_no_other_memory():
    m = Model(2, 3, 200, seed=21)
    m.append([200, 100, 50])
    q = bf16_dev(m.values(20, 8))
    kv = bf16_dev(m.values(20, 2))
    for starts, lengths in (([-5, 3, 1, 400], [1 << 30, -7, 90]), ([0, 20, 20, 20], [0, 0, 0]), ([9, 2, 30, 5], [100, 1, 2]), ([0, 0, 0, 0], [5, 5, 5])):
        before = m.cache.k_codes.clone()
        out = w.w4a8_cache4_attention(q, m.cache, i32(starts), i32(lengths), i32(m.table), SCALE)
        w.w4a8_cache4_read(m.cache, i32(starts), i32(lengths), i32(m.table), 20)
        w.w4a8_cache4_append(kv, kv, m.cache, i32(starts), i32(lengths), i32(np.full_like(m.table, -1)))
        torch.cuda.synchronize()
        assert out.shape == q.shape and torch.equal(before, m.cache.k_codes)


OUT_OF_RANGE = [([-5, 3, 1, 400], [1 << 30, -7, 90]), ([0, 20, 20, 20], [0, 0, 0]), ([9, 2, 30, 5], [100, 1, 2]), ([0, 0, 0, 0], [5, 5, 5]),
                ([0, 7, 7, 20], [-(1 << 31), (1 << 31) - 1, 1 << 30]), ([-(1 << 31), (1 << 31) - 1, 0, 20], [200, 100, 50])]


@pytest.mark.parametrize("starts,lengths", OUT_OF_RANGE)
def test_arrays_out_of_range_leave_the_rest_alone(starts, lengths):
    m = Model(2, 3, 200, seed=44, pages=3 * 4 + 9)
    m.append([200, 100, 50])
    q, kv = bf16_dev(m.values(20, 8)), bf16_dev(m.values(20, 2))
    s, n, none = i32(starts), i32(lengths), i32(np.full_like(m.table, -1))
    rows = lambda H: torch.full((36, H, D), 9.0, dtype=torch.bfloat16, device=dev())  # noqa: E731
    out, k, v = rows(8), rows(2), rows(2)
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    before = [t.clone() for t in m.cache]
    print(f"[case] {starts} {lengths}", flush=True)
    for table in (i32(m.table), none):
        w.w4a8_cache4_attention(q, m.cache, s, n, table, SCALE, out=out[8:28])
        w.w4a8_cache4_read(m.cache, s, n, table, 20, k_out=k[8:28], v_out=v[8:28])
    w.w4a8_cache4_append(kv, kv, m.cache, s, n, none)
    torch.cuda.synchronize()
    for t in (out, k, v):
        assert (t[:8] == 9).all() and (t[28:] == 9).all()
    assert all(same(a, b) for a, b in zip(before, m.cache))
    # with pages, tokens may be held there, and nowhere else
    w.w4a8_cache4_append(kv, kv, m.cache, s, n, i32(m.table))
    torch.cuda.synchronize()
    others = [p for p in range(21) if p not in m.table]
    assert all(same(a[others], b[others]) for a, b in zip(before, m.cache))


@pytest.mark.parametrize("kind", ["k", "v"])
def test_read_of_one_kind(kind):
    # the library's call with no room for the other: its rows come as with both
    m = Model(3, 2, 100, seed=45).append([70, 20])
    want = dict(zip("kv", read(m, [70, 20])))
    out = torch.full((90, 3, D), 7.0, dtype=torch.bfloat16, device=dev())
    starts, lengths, table = m.batch([70, 20])
    c, _ = w._cache4_args(m.cache)
    b = w._batch4_args(90, starts, lengths, table)
    args = dict(k=(None, 0, 0), v=(None, 0, 0))
    args[kind] = (out.data_ptr(), out.stride(0), out.stride(1))
    assert w.lib().w4a8_cache4_read(c, b, *args["k"], *args["v"], torch.cuda.current_stream().cuda_stream) == w.W4A8_OK
    torch.cuda.synchronize()
    assert torch.equal(out, want[kind])


@pytest.mark.parametrize("L", [300, 5000])
def test_pages_past_the_caches_and_through_them(L):
    # Three new tokens of 8 heads are 24 rows, more than the 16 of a workgroup: pages through the caches.  The same
    # tokens as a sequence each, on the same pages, are 8 rows: past them.  Splits and the order of sums are alike, and
    # tokens that a row does not see add 0, so the bits are the same.
    m = Model(1, 1, L, seed=46)
    m.append([L])
    q = m.values(3, 8)
    want = m.check_attention([3], 8, q=q)
    got = w.w4a8_cache4_attention(bf16_dev(q), m.cache, i32(range(4)), i32([L - 2, L - 1, L]), i32(np.tile(m.table, (3, 1))), SCALE)
    assert torch.equal(got, want)


@pytest.mark.parametrize("H,Hkv,lengths,new", [(32, 8, [300] * 40 + [20000] + [77] * 23, [1] * 64), (16, 16, [500] * 30 + [900] + [64], [1] * 30 + [300, 1])])
def test_sequences_unlike_each_other(H, Hkv, lengths, new):
    # one long sequence among short ones, a chunk among single tokens
    B, blocks = len(lengths), [-(-L // BLK) for L in lengths]
    at = np.cumsum([0] + blocks)
    m = Model(Hkv, 1, BLK, seed=47, pages=int(at[-1]) + 3)
    m.B, m.blocks, m.table = B, max(blocks), np.full((B, max(blocks)), -1, np.int32)  # pages for what each holds
    m.k, m.v = ([np.zeros((0, Hkv, D), np.uint16) for _ in range(B)] for _ in range(2))
    pages = m.rng.permutation(at[-1])
    for b in range(B):
        m.table[b, :blocks[b]] = pages[at[b]:at[b + 1]]
    m.append(lengths)
    m.check_attention(new, H, workspace=w.Workspace())


def test_layouts_of_queries_and_output():
    m = Model(2, 2, 300, seed=22)
    m.append([300, 90])
    new = [9, 30]
    q = m.values(39, 8)
    want = m.check_attention(new, 8, q=q)
    wide = torch.empty(39, 15, D, dtype=torch.bfloat16, device=dev())
    wide[:, 4:12] = bf16_dev(q)
    out = torch.full((39, 11, D), 9.0, dtype=torch.bfloat16, device=dev())
    m.attend(wide[:, 4:12], new, out=out[:, 2:10])
    assert torch.equal(out[:, 2:10], want) and (out[:, :2] == 9).all() and (out[:, 10:] == 9).all()
    headed = bf16_dev(q).transpose(0, 1).contiguous()
    o = torch.empty_like(headed)
    m.attend(headed.transpose(0, 1), new, out=o.transpose(0, 1))
    assert torch.equal(o.transpose(0, 1), want)


def test_read_into_every_other_head():
    m = Model(2, 1, 100, seed=43).append([100])
    want = read(m, [100])
    both = torch.zeros(100, 4, D, dtype=torch.bfloat16, device=dev())
    got = read(m, [100], k_out=both[:, ::2], v_out=both[:, 1::2])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_output_beside_the_queries():
    # one matrix's rows, halves of a token or every other head; over the queries or the cache is refused
    m = Model(2, 2, 300, seed=39)
    m.append([300, 90])
    for new in ([9, 30], [1, 0]):
        T, H = sum(new), 8
        q = m.values(T, H)
        want = m.check_attention(new, H, q=q)
        for both in (torch.zeros(T, 2 * H, D, dtype=torch.bfloat16, device=dev()), torch.zeros(2 * H, T, D, dtype=torch.bfloat16, device=dev()).transpose(0, 1)):
            for qd, o in ((both[:, :H], both[:, H:]), (both[:, H:], both[:, :H]), (both[:, ::2], both[:, 1::2]), (both[:, 1::2], both[:, ::2])):
                qd.copy_(bf16_dev(q))
                o.zero_()
                m.attend(qd, new, out=o)
                assert torch.equal(o, want) and torch.equal(qd, bf16_dev(q))
        both = torch.cat([bf16_dev(q), bf16_dev(q)], 1)
        before, pages = both.clone(), [t.clone() for t in m.cache]
        flat = m.cache.k_codes.view(-1).view(torch.bfloat16)
        for qd, o in ((both[:, :H], both[:, :H]), (both[:, :H], both[:, 1:H + 1]), (both[:, H:], both[:, H - 1:-1]),
                      (both[:, :H], flat[-T * H * D:].view(T, H, D))):
            for kw in (dict(), dict(stream=torch.cuda.current_stream())):
                with pytest.raises(w.W4A8Error):
                    m.attend(qd, new, out=o, **kw)
        torch.cuda.synchronize()
        assert torch.equal(both, before) and all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(m.cache, pages))


def test_shared_pages():
    # two sequences with a common beginning
    m = Model(2, 2, 200, seed=23)
    k, v = m.values(128, 2), m.values(128, 2)
    m.append([128, 0], k, v)
    m.table[1, :2] = m.table[0, :2]
    m.k[1], m.v[1] = m.k[0].copy(), m.v[0].copy()
    m.append([9, 33])
    m.check_attention([9, 33], 8)


def test_pages_past_32_bit_offsets():
    pages = 150000  # 4096 bytes of 8 heads' codes each: 4.9 GB
    m = Model(8, 1, 130, seed=24, pages=pages)
    m.table[0] = [pages - 1, 5, pages - 2]
    m.append([130])
    read(m, [130])
    m.check_attention([1], 8)
    m.check_attention([20], 32)


def test_repeated_calls_agree():
    m = Model(4, 3, 900, seed=25)
    m.append([900, 333, 64])
    for new in ([1, 1, 1], [60, 9, 31]):
        q = bf16_dev(m.values(sum(new), 28))
        first = m.attend(q, new)
        for _ in range(20):
            assert torch.equal(m.attend(q, new), first)


def test_side_streams_and_two_calls_at_once():
    m = Model(4, 2, 1500, seed=26)
    m.append([1500, 700])
    q = [bf16_dev(m.values(2, 16)) for _ in range(2)]
    want = [m.attend(x, [1, 1]) for x in q]
    torch.cuda.synchronize()
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [w.Workspace() for _ in range(2)]
    for _ in range(5):
        got = [m.attend(x, [1, 1], stream=s, workspace=b) for x, s, b in zip(q, streams, ws)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_workspaces():
    m = Model(2, 1, 2000, seed=27)
    m.append([2000])
    q = bf16_dev(m.values(1, 8))
    need = w.w4a8_cache4_attention_workspace_bytes(1, 1, 8, 2, m.blocks * BLK)
    assert need > 65536
    want = m.attend(q, [1])
    buf = torch.full((need,), 77, dtype=torch.uint8, device=dev())
    assert torch.equal(m.attend(q, [1], workspace=buf), want) and (buf[:65536] == 77).all()
    with pytest.raises(w.W4A8Error):
        m.attend(q, [1], workspace=buf[:-1])
    ws = w.Workspace()
    assert torch.equal(m.attend(q, [1], workspace=ws), want) and ws.buf.numel() >= need
    held = ws.buf
    with pytest.raises(w.W4A8Error):
        m.attend(q, [1], workspace=ws, max_len=m.blocks * BLK + 1)
    assert ws.buf is held
    # one Workspace for the linear and the attention
    from helpers import pack, scales_dev
    x, W, sw, K, N = I.workload_inputs("tiny", 4)
    wp, s = pack(W), scales_dev(sw)
    y = w.w4a8_linear(bf16_dev(x), wp, s, N, workspace=ws)
    m.attend(q, [1], workspace=ws)
    assert torch.equal(w.w4a8_linear(bf16_dev(x), wp, s, N, workspace=ws), y)


def test_graph_of_a_step():
    m = Model(2, 2, 700, seed=28)
    m.append([600, 130])
    ws = w.Workspace()
    H = 8
    first = m.values(2, H + 4)
    qkv = bf16_dev(first)
    starts, lengths, table = m.batch([1, 1])
    out = torch.empty(2, H, D, dtype=torch.bfloat16, device=dev())
    back = [torch.empty(2, 2, D, dtype=torch.bfloat16, device=dev()) for _ in range(2)]

    def step(out, back):
        w.w4a8_cache4_append(qkv[:, H:H + 2], qkv[:, H + 2:], m.cache, starts, lengths, table)
        w.w4a8_cache4_read(m.cache, starts, lengths, table, 2, *back)
        w.w4a8_cache4_attention(qkv[:, :H], m.cache, starts, lengths, table, SCALE, out=out, workspace=ws)

    step(out, back)
    for b in range(2):  # in the place of the last token
        m.k[b][-1], m.v[b][-1] = first[b, H:H + 2], first[b, H + 2:]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, back)
    for i in range(5):
        new = m.values(2, H + 4)
        qkv.copy_(bf16_dev(new))
        m.k = [np.concatenate([x, new[b:b + 1, H:H + 2]]) for b, x in enumerate(m.k)]
        m.v = [np.concatenate([x, new[b:b + 1, H + 2:]]) for b, x in enumerate(m.v)]
        lengths += 1
        g.replay()
        torch.cuda.synchronize()
        m.compare(out, new[:, :H], [1, 1], SCALE, f"replay {i}")
        eager = torch.empty_like(out)
        step(eager, [torch.empty_like(b) for b in back])
        assert torch.equal(eager, out)
    m.check_pages()


def test_graphs_that_share_a_workspace():
    m = Model(2, 1, 3000, seed=29)
    m.append([3000])
    ws = w.Workspace()
    q = [bf16_dev(m.values(n, 8)) for n in (1, 6)]
    want = [m.attend(x, [len(x)], workspace=ws) for x in reversed(q)][::-1]
    outs = [torch.empty_like(x) for x in want]
    batches = [m.batch([len(x)]) for x in q]
    graphs = []
    for x, o, b in zip(q, outs, batches):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            w.w4a8_cache4_attention(x, m.cache, *b, SCALE, out=o, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        m.attend(q[0], [1], workspace=ws)
        torch.cuda.synchronize()
        for o, x in zip(outs, want):
            assert torch.equal(o, x)
            o.zero_()


def test_cache_that_is_read_past_the_memory_side_cache():
    # above 160 MB the pages are read with another kind of load
    H, Hkv, L = 8, 8, 1500
    B = -(-(160 << 20) // (144 * Hkv * L)) + 1
    m = Model(Hkv, 2, L, seed=30)
    m.append([L, L - 77])
    q = m.values(2, H)
    want = m.attend(bf16_dev(q), [1, 1], max_len=L)
    table = i32(np.tile(m.table, (B // 2 + 1, 1)))
    lengths = i32(np.tile([L, L - 77], B // 2 + 1))
    n = len(lengths)
    got = w.w4a8_cache4_attention(bf16_dev(np.tile(q, (B // 2 + 1, 1, 1))), m.cache, i32(np.arange(n + 1)), lengths, table, SCALE, max_len=L)
    m.compare(got[:2], q, [1, 1], SCALE)
    m.compare(want, q, [1, 1], SCALE)
    for i in range(0, n, 2):
        assert torch.equal(got[i:i + 2], got[:2])


def test_more_row_blocks_than_an_axis_of_a_launch_holds():
    # 70000 sequences' worth of rows: one token each, of 65536 sequences at most
    B = 65536
    m = Model(1, 1, 64, seed=31)
    m.append([40])
    q = m.values(1, 1)
    want = m.attend(bf16_dev(q), [1], max_len=64)
    T = B
    qd = bf16_dev(q).expand(T, 1, D).contiguous()
    out = w.w4a8_cache4_attention(qd, m.cache, i32(np.arange(B + 1)), i32(np.full(B, 40)), i32(np.tile(m.table[:1], (B, 1))), SCALE, max_len=64)
    assert torch.equal(out, want.expand(T, 1, D))


def test_native_path_takes_the_plain_calls(monkeypatch):
    m = Model(2, 1, 200, seed=32)
    seen = []
    real = w._load_fast()

    class Spy:
        def __getattr__(self, name):
            def call(*a):
                r = getattr(real, name)(*a)
                seen.append((name, r is not None))
                return r
            return call

    monkeypatch.setattr(w, "_fast", Spy())
    m.append([200])
    read(m, [3])
    m.check_attention([3], 8)
    assert seen == [("cache4_append", True), ("cache4_read", True), ("cache4_attention", True)]


def test_refusals():
    m = Model(2, 2, 200, seed=33)
    m.append([200, 30])
    starts, lengths, table = m.batch([1, 1])
    x, q = bf16_dev(m.values(2, 2)), bf16_dev(m.values(2, 8))
    app = lambda k=x, v=x, c=m.cache, s=starts, l=lengths, t=table: w.w4a8_cache4_append(k, v, c, s, l, t)  # noqa: E731
    get = lambda c=m.cache, s=starts, l=lengths, t=table, rows=2, **kw: w.w4a8_cache4_read(c, s, l, t, rows, **kw)  # noqa: E731
    att = lambda x=q, c=m.cache, s=starts, l=lengths, t=table, scale=SCALE, **kw: w.w4a8_cache4_attention(x, c, s, l, t, scale, **kw)  # noqa: E731
    before = [t.clone() for t in m.cache]
    wrong = [dict(c=m.cache._replace(k_codes=m.cache.v_codes)), dict(c=m.cache._replace(v_params=m.cache.k_params)), dict(s=starts[:2]),
             dict(l=lengths[None]), dict(t=table[0])]
    for call in (app, get, att):
        for kw in wrong:
            with pytest.raises(ValueError):
                call(**kw)
        for kw in (dict(c=m.cache._replace(k_params=m.cache.k_params.float())), dict(s=starts.long()), dict(l=lengths.cpu())):
            with pytest.raises(TypeError):
                call(**kw)
    for kw, err in ((dict(k=x.float()), TypeError), (dict(k=x[:, :1]), ValueError), (dict(v=x[:1]), ValueError), (dict(k=x[..., :64], v=x[..., :64]), ValueError),
                    (dict(k=x.cpu(), v=x), TypeError)):
        with pytest.raises(err):
            app(**kw)
    big = torch.empty(4, 2, D, dtype=torch.bfloat16, device=dev())
    for kw, err in ((dict(rows=-1), Exception), (dict(k_out=big), ValueError), (dict(v_out=big[:2].float()), TypeError), (dict(k_out=big[:2], v_out=big[1:3]), w.W4A8Error),
                    (dict(k_out=big[:1].expand(2, 2, D)), w.W4A8Error)):
        with pytest.raises(err):
            get(**kw)
    for kw, err in ((dict(x=q[:, :7]), w.W4A8Error), (dict(x=q.float()), TypeError), (dict(scale=float("nan")), w.W4A8Error), (dict(max_len=0), w.W4A8Error),
                    (dict(out=q[:1]), ValueError), (dict(out=q[:1].expand(2, 8, D)), w.W4A8Error), (dict(max_len=10 ** 9), w.W4A8Error)):
        with pytest.raises(err):
            att(**kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, m.cache))
    # nothing to do
    app(k=x[:0], v=x[:0], s=starts * 0)
    assert att(x=q[:0], s=starts * 0).shape == (0, 8, D) and get(rows=0, s=starts * 0)[0].shape == (0, 2, D)


# ---- together


@pytest.mark.parametrize("axes", [None, (24, 20, 20)])
def test_a_layer_step_by_step(axes):
    """Projection, norms and rotation in place, append, attention, projection:
    a prompt, then single tokens and a draft block, against fp64 from each
    call's own inputs on."""
    K, H, Hkv, T0 = 512, 4, 2, 75
    rng = np.random.Generator(np.random.PCG64(34))
    qkv_n = (H + 2 * Hkv) * D
    from helpers import pack, scales_dev
    Wq, Wo = (rng.integers(-8, 8, s).astype(np.int8) for s in ((qkv_n, K), (K, H * D)))
    sq, so = (np.full(n, 0.02, np.float32) for n in (qkv_n, K))
    wq, wo, dq, do = pack(Wq), pack(Wo), scales_dev(sq), scales_dev(so)
    gamma = [I.to_bf16_bits((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2)]
    dg = [bf16_dev(g) for g in gamma]
    cos, sin = oracle.rope_tables(200, D)
    dt = [torch.from_numpy(t).to(dev()) for t in (cos, sin)]
    ax = w.rope_axes(axes, True) if axes else None
    axis = np.frombuffer(ax, np.uint8) if axes else np.zeros(64, int)
    m = Model(Hkv, 1, 200, seed=35)
    ws = w.Workspace()
    L = 0
    for n in (T0, 1, 1, 8, 1):
        x = I.activations(n, K, 36 + L)
        qkv = w.w4a8_linear(bf16_dev(x), wq, dq, qkv_n, workspace=ws).view(n, H + 2 * Hkv, D)
        raw = to_np_bits(qkv)
        t = np.arange(L, L + n)
        pos = np.stack([t // 6, t // 3 % 2 + t // 6, t % 3 + t // 6]) if axes else t[None]
        dpos = i32(pos) if axes else i32(pos[0])
        q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        w.w4a8_qk_norm_rope(q, k, *dg, 1e-6, dpos, *dt, axes=ax, q_out=q, k_out=k)
        for got, lo, hi, g in ((q, 0, H, gamma[0]), (k, H, H + Hkv, gamma[1])):
            y, mag = oracle.qk_norm_rope(raw[:, lo:hi], g, 1e-6, pos, axis, cos, sin)
            off = np.abs(oracle._f32(to_np_bits(got.contiguous())) - y)
            assert (off <= 2.0 ** -8 * np.abs(y) + (1 + 2.0 ** -8) * 2.0 ** -19 * mag).all()
        np.testing.assert_array_equal(to_np_bits(v.contiguous()), raw[:, H + Hkv:])
        m.k[0] = np.concatenate([m.k[0], to_np_bits(k.contiguous())])
        m.v[0] = np.concatenate([m.v[0], raw[:, H + Hkv:]])
        L += n
        w.w4a8_cache4_append(k, v, m.cache, *m.batch([n]))
        o = w.w4a8_cache4_attention(q, m.cache, *m.batch([n]), SCALE, max_len=L, workspace=ws)
        m.compare(o, to_np_bits(q.contiguous()), [n], SCALE)
        y = w.w4a8_linear(o.view(n, H * D), wo, do, K, workspace=ws)
        ref = oracle.linear(to_np_bits(o).reshape(n, H * D), Wo, s_w=so)
        np.testing.assert_array_equal(to_np_bits(y), ref["y"])
    m.check_pages()


# Calls that take each of the kernel's forms, with and without splits: rows that
# end inside a wave's tile and inside a workgroup, sequences shorter than the
# others, a block without a page, NaN behind the last token.
@pytest.mark.parametrize("H,Hkv,lengths,new", [
    (64, 1, [400], [397]), (128, 1, [2057, 2000, 1999, 700, 64], [14, 14, 14, 9, 14]),    # 128 rows
    (64, 4, [900, 401], [600, 333]), (64, 2, [2057], [262]),                              # 256 rows
    (32, 2, [580, 301], [267, 260]), (64, 8, [2000], [400]), (48, 1, [2171, 2100, 64, 2000, 35], [35] * 5),  # 128 rows in two groups
    (32, 1, [69, 64, 65, 64, 66], [64] * 5), (64, 8, [2577], [22])])            # 32 rows
def test_forms(H, Hkv, lengths, new):
    print(f"[case] forms H={H} Hkv={Hkv} {lengths} {new}", flush=True)
    m = Model(Hkv, len(lengths), max(lengths), seed=sum(new))
    m.append(lengths)
    q = m.values(sum(new), H, 0.3)
    a = m.check_attention(new, H, q=q)
    b = m.attend(bf16_dev(q), new, max_len=64 * m.blocks // 2)  # another plan
    torch.cuda.synchronize()
    m.compare(b, q, new, SCALE, "other plan")
    gone = min(1, m.blocks - 1)
    m.table[0, gone] = -1
    c = m.attend(bf16_dev(q), new)
    k, v = m.held(0)
    L, n = lengths[0], new[0]
    keep = [t for t in range(L) if t // BLK != gone]
    q64 = torch.from_numpy(oracle._f32(q).astype(np.float64)).to(dev())
    lens = torch.tensor([sum(t <= L - n + i for t in keep) for i in range(n)], device=dev())
    for h in range(0, H, 7):
        kk, vv = (torch.from_numpy(x[keep, h // (H // Hkv)]).to(dev()) for x in (k, v))
        o, tol = reference(q64[:n, h], kk, vv, lens, SCALE)
        assert ((c[:n, h].double() - o).abs() <= tol).all(), h
    assert torch.equal(c[n:], a[n:])
