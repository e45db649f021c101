"""The 8-bit cache (w4a8_cache_append, w4a8_cache_attention) against the
oracle.

The append is exact: rotation, scale and code are IEEE fp32 operations on
both sides, so codes, scales and rings have to be equal.

Tolerance of the attention, derived.  Against fp64 on the values that the
codes stand for, the kernel
  - holds the rotated query in 16 bits: an element is off by at most
    top / 65024 (half a step of top / 32512), so a score by at most
    d = |scale| top / 65024 max_j |k_j|_1, and a weight by a factor within
    exp(+-2 d) (its own score and the total's): 2 d (1 + 2 d) of it;
  - rounds weights to fp16, 2^-11 of each, and forms scores and exponentials
    in fp32: exponents up to a few hundred, so within 2^-14 of each weight;
  - has fp16's smallest weights: they are scaled so that the largest of
    P_ij s_v(j) (s_v the values' scale) lies in [2^12, 2^15] (it starts at
    2^12, and only one that would pass 2^15 scales them anew), and below
    2^-14 a step of fp16 is 2^-24, so half a step, 2^-25, is 2^-37 of the
    largest at most; with codes up to 127 and N keys that is
    N 2^-37 max_j P_ij max |v| of j's block at most.  It counts in elements
    d where the heavy keys' values are near 0;
  - rounds the output to bf16, 2^-8 of it.
With B = sum_j P_ij |v_jd| and T = N max_j P_ij max |v| of j's block:
  |o - o64| <= 2^-8 |o64| + (1 + 2^-8) ((2^-11 + 2^-14 + 2 d (1 + 2 d)) B + 2^-37 T)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_12932_amd as w
from paper_2608_12932_amd import inputs as I
from helpers import bf16_dev, dev, to_np_bits

pytestmark = pytest.mark.gpu

D, BLK, RING = 128, w.CACHE_BLOCK, w.CACHE_RECENT
SCALE = D ** -0.5


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev())


def tolerance(o64, bnd, top, peak, k, scale):
    """The bound above, for keys k [Hkv][L][D]."""
    H = o64.shape[1]
    l1 = np.abs(k).sum(-1).max(-1, initial=0.0)[np.arange(H) // (H // len(k))]
    d = abs(scale) * top / 65024 * l1[None]
    return 2.0 ** -8 * np.abs(o64) + (1 + 2.0 ** -8) * ((2.0 ** -11 + 2.0 ** -14 + 2 * d * (1 + 2 * d))[..., None] * bnd + 2.0 ** -37 * peak[..., None])


class Model:
    """Sequences of bf16 keys (before rotation) and values, and a cache that
    is filled with them through the calls under test."""

    def __init__(self, Hkv, B, max_len, seed=0, pages=None, pos0=0):
        self.Hkv, self.B, self.blocks, self.pos0 = Hkv, B, -(-max_len // BLK), pos0
        self.rng = np.random.Generator(np.random.PCG64(seed))
        n = pages or B * self.blocks + 3
        self.cache = w.KVCache.empty(n, B, Hkv, device=dev())
        self.cache.k_codes.fill_(77)  # what no token fills stays as it was
        self.cache.v_codes.fill_(77)
        self.cache.scales.fill_(float("nan"))
        self.table = self.rng.permutation(n)[:B * self.blocks].reshape(B, self.blocks).astype(np.int32)
        self.k = [np.zeros((0, Hkv, D), np.uint16) for _ in range(B)]  # rotated
        self.v = [np.zeros((0, Hkv, D), np.uint16) for _ in range(B)]
        self.taken_back = []  # pages that held tokens which were taken back
        self.cos, self.sin = oracle.rope_tables(pos0 + max_len, D, base=1e6)
        self.dcos, self.dsin = torch.from_numpy(self.cos).to(dev()), torch.from_numpy(self.sin).to(dev())

    def values(self, n, H):
        return I.to_bf16_bits((self.rng.standard_normal((n, H, D)) * np.exp(0.5 * self.rng.standard_normal((1, H, D)))).astype(np.float32))

    def batch(self, new, behind=0):
        """starts, lengths, table, pos of sequences with `new` new tokens each
        (already counted in the model's lengths) and `behind` rows after the last."""
        lengths = [len(k) for k in self.k]
        starts = np.concatenate([[0], np.cumsum(new)])
        pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, lengths)] + [np.zeros(behind, int)]) + self.pos0
        return i32(starts), i32(lengths), i32(self.table), i32(pos)

    def append(self, new, k=None, v=None, behind=0, slots=None, table=None):
        """Appends new[b] tokens to each sequence, k and v being views of one
        matrix [T][(3 + 2 Hkv) * D]."""
        T = sum(new) + behind
        k = self.values(T, self.Hkv) if k is None else k
        v = self.values(T, self.Hkv) if v is None else v
        at = 0
        for b, n in enumerate(new):
            p = np.repeat(np.arange(len(self.k[b]), len(self.k[b]) + n) + self.pos0, self.Hkv)
            rot = oracle.rope_rotate(k[at:at + n].reshape(-1, D), p, self.cos, self.sin).reshape(n, self.Hkv, D)
            self.k[b], self.v[b] = np.concatenate([self.k[b], rot]), np.concatenate([self.v[b], v[at:at + n]])
            at += n
        starts, lengths, tab, pos = self.batch(new, behind)
        qkv = bf16_dev(np.concatenate([self.values(T, 3), k, v], 1).reshape(T, -1)).view(T, 3 + 2 * self.Hkv, D)
        w.w4a8_cache_append(qkv[:, 3:3 + self.Hkv], qkv[:, 3 + self.Hkv:], self.cache, starts, lengths, tab if table is None else table, pos,
                            self.dcos, self.dsin, slots=slots)
        torch.cuda.synchronize()

    def held(self):
        c = self.cache
        return c.k_codes.cpu().numpy(), c.v_codes.cpu().numpy(), c.scales.cpu().numpy(), to_np_bits(c.k_recent), to_np_bits(c.v_recent)

    def check_cache(self, slots=None, kept=2):
        """The pages, and the rings' last `kept` blocks (after tokens were
        taken back the one before the last may have been overwritten)."""
        kc, vc, sc, kr, vr = self.held()
        used = set(self.taken_back)
        for b in range(self.B):
            L = len(self.k[b])
            for blk in range(-(-L // BLK)):
                p = int(self.table[b, blk])
                used.add(p)
                n = min(L - blk * BLK, BLK)
                for h in range(self.Hkv):
                    for codes, x, s, name in ((kc[p, h], self.k[b], sc[p, h, 0], "k"), (vc[p, h].T, self.v[b], sc[p, h, 1], "v")):
                        want, ws = oracle.cache_block(x[blk * BLK:blk * BLK + n, h])
                        assert np.float32(s).view(np.uint32) == np.float32(ws).view(np.uint32), (name, b, blk, h, s, ws)
                        np.testing.assert_array_equal(codes[:n], want, err_msg=f"{name} sequence {b} block {blk} head {h}")
                        assert not codes[n:].any(), (name, b, blk, h)
            slot = b if slots is None else slots[b]
            for t in range(max(0, ((L - 1) // BLK + 1 - kept) * BLK), L):
                np.testing.assert_array_equal(kr[slot, :, t % RING], self.k[b][t], err_msg=f"ring {b} {t}")
                np.testing.assert_array_equal(vr[slot, :, t % RING], self.v[b][t], err_msg=f"ring {b} {t}")
        rest = [p for p in range(kc.shape[0]) if p not in used]
        assert (kc[rest] == 77).all() and (vc[rest] == 77).all() and np.isnan(sc[rest]).all()

    def cut(self, b, L):
        self.taken_back += [int(p) for p in self.table[b, -(-L // BLK):-(-len(self.k[b]) // BLK)]]
        self.k[b], self.v[b] = self.k[b][:L], self.v[b][:L]

    def attend(self, q, new, scale=SCALE, behind=0, **kw):
        starts, lengths, tab, pos = self.batch(new, behind)
        return w.w4a8_cache_attention(q, self.cache, starts, lengths, tab, pos, self.dcos, self.dsin, scale, **kw)

    def expect(self, q_bits, new, scale=SCALE, lengths=None):
        """o64, and the tolerance above, of every row."""
        kc, vc, sc, _, _ = self.held()
        o, tol, at = [], [], 0
        for b, n in enumerate(new):
            L = len(self.k[b]) if lengths is None else lengths[b]
            pages = self.table[b, :-(-L // BLK)]
            k = (kc[pages].astype(np.float64) * sc[pages, :, 0, None, None]).transpose(1, 0, 2, 3).reshape(self.Hkv, -1, D)[:, :L]
            v = (vc[pages].astype(np.float64) * sc[pages, :, 1, None, None]).transpose(1, 0, 3, 2).reshape(self.Hkv, -1, D)[:, :L]
            pos = np.arange(L - n, L) + self.pos0
            P = len(self.cos)
            got = oracle.cache_attention(q_bits[at:at + n], np.clip(pos, 0, P - 1), k, v, self.cos, self.sin, scale, L - n)
            o.append(got[0])
            tol.append(tolerance(*got, k, scale))
            at += n
        return np.concatenate(o), np.concatenate(tol)

    def check_attention(self, H, new, scale=SCALE, label="", q_bits=None, **kw):
        print(f"[case] cache attention {label} H={H} Hkv={self.Hkv} new={new} lengths={[len(k) for k in self.k]} scale={scale}", flush=True)
        q_bits = self.values(sum(new), H) if q_bits is None else q_bits
        o = self.attend(bf16_dev(q_bits), new, scale, **kw)
        torch.cuda.synchronize()
        o = o.float().cpu().numpy().astype(np.float64)
        o64, tol = self.expect(q_bits, new, scale)
        bad = ~(np.abs(o - o64) <= tol + 1e-30)  # a NaN is outside it too
        assert not bad.any(), f"{label}: {bad.sum()} of {bad.size} outside, worst ratio {np.nanmax(np.abs(o - o64) / (tol + 1e-30)):.2f}"
        return o


# ---------------------------------------------------------------- append


@pytest.mark.parametrize("steps", [[1] * 5, [63, 1, 1], [64, 64], [65, 62, 2], [130], [3, 200, 1], [1, 129, 1, 60, 70], [300, 1], [64, 128, 64],
                                   [40, 24, 1], [127, 1, 128, 1], [190, 5, 260, 3]])
def test_append_steps(steps):
    m = Model(2, 1, sum(steps), seed=sum(steps), pos0=5)
    for n in steps:
        print(f"[case] append {n} after {len(m.k[0])}", flush=True)
        m.append([n])
        m.check_cache()


def test_append_ragged_batch():
    # sequences of every kind side by side: none, one, a block's rest, several blocks; rows behind the last
    m = Model(3, 7, 400, seed=21)
    for new in ([1, 0, 64, 63, 130, 7, 200], [1, 1, 1, 1, 0, 57, 33], [0, 0, 0, 0, 0, 0, 1], [62, 130, 1, 64, 128, 2, 99]):
        print(f"[case] append ragged {new}", flush=True)
        m.append(new, behind=3)
        m.check_cache()


def test_append_many_sequences():
    # more sequences than a wave's lanes, most without new tokens
    B = 150
    m = Model(1, B, 80, seed=22)
    m.append([int(x) for x in m.rng.integers(0, 60, B)])
    m.check_cache()
    m.append([1 if b % 9 == 0 else 0 for b in range(B)])
    m.check_cache()


def test_append_does_not_depend_on_the_chunks():
    a, b = Model(2, 1, 333, seed=23), Model(2, 1, 333, seed=23)
    k, v = a.values(333, 2), a.values(333, 2)
    a.append([333], k, v)
    at = 0
    for n in (1, 62, 1, 1, 100, 128, 37, 3):
        b.append([n], k[at:at + n], v[at:at + n])
        at += n
    assert at == 333
    for x, y in zip(a.held()[:3], b.held()[:3]):
        np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("L,back", [(200, 64), (129, 1), (128, 64), (191, 63), (256, 64), (193, 20)])
def test_tokens_taken_back(L, back):
    # a draft's rejected tokens: the sequence goes on from a smaller length
    m = Model(2, 1, L + 80, seed=24 + back)
    m.append([L - back])
    m.append([back])
    m.cut(0, L - back)
    m.append([5])
    m.check_cache(kept=1)
    m.append([70])
    m.check_cache(kept=1)


def test_append_slots_and_wrong_indices():
    # rings by slot; a slot or page out of range writes nothing anywhere
    m = Model(2, 3, 200, seed=25)
    slots = i32([2, 0, 1])
    m.append([70, 20, 100], slots=slots)
    m.append([10, 50, 30], slots=slots)
    m.check_cache(slots=[2, 0, 1])
    before = [t.clone() for t in m.cache]
    bad = i32(m.table)
    bad[:, :] = torch.tensor([-1, 1 << 30, m.cache.k_codes.shape[0]], dtype=torch.int32)[:, None].to(dev())
    print("[case] append with pages and slots out of range", flush=True)
    m.append([4, 4, 4], slots=i32([-1, 3, 1 << 30]), table=bad)
    for x, y in zip(m.cache, before):
        assert torch.equal(x.view(torch.int8), y.view(torch.int8))


@pytest.mark.parametrize("bad", [-1, 3, 1 << 30])
def test_append_without_a_ring(bad):
    # the exact values of a started block's older tokens are not known: it stays as it is; blocks without older tokens are written
    m = Model(2, 3, 300, seed=61)
    m.append([70, 64, 130])
    before = [t.clone() for t in m.cache]
    lengths = [len(k) for k in m.k]
    print(f"[case] append, slots {bad}", flush=True)
    m.append([5, 5, 70], slots=i32([bad] * 3))
    kept, page = [(0, 1), (2, 2)], lambda b, blk: int(m.table[b, blk])  # noqa: E731
    written = {(1, 1): (64, 69), (2, 3): (192, 200)}
    touched = sorted(page(b, blk) for b, blk in written)
    for name, x, y in zip(m.cache._fields, m.cache, before):
        x, y = x.view(torch.int8), y.view(torch.int8)
        if name.endswith("recent"):
            assert torch.equal(x, y), name
            continue
        rest = [p for p in range(len(x)) if p not in touched]
        assert torch.equal(x[rest], y[rest]), (name, [p in [page(*i) for i in kept] for p in rest if not torch.equal(x[p], y[p])])
    assert lengths == [70, 64, 130]
    kc, vc, sc, _, _ = m.held()
    for (b, blk), (lo, hi) in written.items():
        for h in range(2):
            for codes, x, s in ((kc[page(b, blk), h], m.k[b], sc[page(b, blk), h, 0]), (vc[page(b, blk), h].T, m.v[b], sc[page(b, blk), h, 1])):
                want, ws = oracle.cache_block(x[lo:hi, h])
                assert np.float32(s).view(np.uint32) == np.float32(ws).view(np.uint32)
                np.testing.assert_array_equal(codes[:hi - lo], want)
                assert not codes[hi - lo:].any()


def test_append_zero_and_tiny_blocks():
    m = Model(2, 1, 130, seed=26)
    k, v = m.values(130, 2), m.values(130, 2)
    k[:64], v[64:128] = 0, 0
    k[128:] = I.to_bf16_bits(np.full((2, 2, D), 2.0 ** -95, np.float32))    # held as zeros
    v[128:] = I.to_bf16_bits(np.full((2, 2, D), 2.0 ** -80, np.float32))
    m.append([130], k, v)
    m.check_cache()
    sc = m.held()[2]
    assert (sc[m.table[0, 0], :, 0] == 0).all() and (sc[m.table[0, 1], :, 1] == 0).all() and (sc[m.table[0, 2], :, 0] == 0).all()
    m.check_attention(4, [130], label="zero blocks")
    m.check_attention(4, [1], label="zero blocks, one row")


# ---------------------------------------------------------------- attention


HEADS = [(32, 8), (28, 4), (8, 1), (4, 4), (40, 8), (3, 1), (6, 2), (18, 1), (1, 1)]


@pytest.mark.parametrize("H,Hkv", HEADS)
def test_decode(H, Hkv):
    m = Model(Hkv, 5, 200, seed=H)
    m.append([1, 64, 65, 200, 130])
    m.check_attention(H, [1] * 5, label="decode")


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000, 4095])
@pytest.mark.parametrize("n", [1, 2, 16])
def test_lengths(L, n):
    m = Model(2, 1, L, seed=L)
    m.append([L])
    m.check_attention(8, [min(n, L)], label="lengths")


@pytest.mark.parametrize("H,Hkv,n,L", [(8, 2, 33, 100), (8, 2, 64, 64), (4, 1, 100, 357), (7, 1, 70, 500), (4, 4, 200, 201), (28, 4, 40, 170),
                                       (8, 2, 257, 1100), (2, 1, 9, 40), (2, 1, 17, 40), (5, 1, 26, 300)])
def test_chunks(H, Hkv, n, L):
    m = Model(Hkv, 1, L, seed=n)
    m.append([L])
    m.check_attention(H, [n], label="chunk")


def test_mixed_batch():
    # a chunk, drafts, single tokens, a sequence without new tokens; and rows behind the last, left as they were
    m = Model(2, 6, 700, seed=31)
    new = [130, 1, 16, 0, 1, 5]
    m.append([300, 700, 77, 40, 1, 64])
    m.check_attention(8, new, label="mixed")
    q = bf16_dev(m.values(sum(new) + 4, 8))
    for rows in (4, 0):
        out = torch.full((sum(new) + 4, 8, D), 3.0, dtype=torch.bfloat16, device=dev())
        m.attend(q, new, behind=4, out=out)
        assert (out[sum(new):] == 3.0).all() and not (out[:sum(new)] == 3.0).all(-1).any()


@pytest.mark.parametrize("behind", [0, 4])
def test_output_with_and_without_rows_behind(behind):
    m = Model(2, 6, 700, seed=31)
    new = [130, 1, 16, 0, 1, 5]
    m.append([300, 700, 77, 40, 1, 64])
    q = bf16_dev(m.values(sum(new) + behind, 8))
    want = m.attend(q[:sum(new)], new)
    out = torch.full((sum(new) + behind, 8, D), 3.0, dtype=torch.bfloat16, device=dev())
    assert m.attend(q, new, behind=behind, out=out) is out
    # (the number of rows takes part in the choice of the form and splits, so the sums' order may differ by it)
    o64, tol = m.expect(to_np_bits(q)[:sum(new)], new)
    for o in (want, out[:sum(new)]):
        assert (np.abs(o.float().cpu().numpy() - o64) <= tol).all()
    assert (out[sum(new):] == 3.0).all()
    if not behind:
        assert torch.equal(out, want)


def test_many_sequences():
    B = 130
    m = Model(1, B, 100, seed=32)
    m.append([int(x) for x in m.rng.integers(1, 100, B)])
    m.check_attention(4, [1] * B, label="130 sequences")
    new = [int(min(len(k), x)) for k, x in zip(m.k, m.rng.integers(0, 20, B))]
    m.check_attention(4, new, label="130 ragged")


@pytest.mark.parametrize("L,n,H,Hkv", [(30000, 1, 4, 1), (30001, 3, 8, 2), (5000, 40, 4, 1)])
def test_long_cache_in_splits(L, n, H, Hkv):
    assert w.w4a8_cache_attention_workspace_bytes(1, n, H, Hkv, L) > 0
    m = Model(Hkv, 1, L, seed=33)
    m.append([L])
    ws = w.Workspace(dev())
    o = m.check_attention(H, [n], label="splits", workspace=ws)
    q = m.values(n, H)
    few, many = (m.attend(bf16_dev(q), [n], max_len=k, workspace=ws) for k in (1, None))  # max_len splits the work, no more
    o64, tol = m.expect(q, [n])
    for o in (few, many):
        assert (np.abs(o.float().cpu().numpy() - o64) <= tol).all()


def test_rows_that_see_nothing():
    # lengths below the new tokens' number: the first rows see no key
    m = Model(2, 3, 100, seed=34)
    m.append([100, 64, 10])
    for new, lengths in (([5, 20, 3], [3, 0, 3]), ([70, 1, 40], [2, 0, 39])):
        q = m.values(sum(new), 8)
        starts = i32(np.concatenate([[0], np.cumsum(new)]))
        pos = i32(np.concatenate([np.arange(L - n, L) for n, L in zip(new, lengths)]))
        print(f"[case] rows that see nothing {new} {lengths}", flush=True)
        o = w.w4a8_cache_attention(bf16_dev(q), m.cache, starts, i32(lengths), i32(m.table), pos, m.dcos, m.dsin, SCALE)
        o = o.float().cpu().numpy()
        o64, tol = m.expect(q, new, lengths=lengths)
        assert (np.abs(o - o64) <= tol).all()
        at = 0
        for n, L in zip(new, lengths):
            assert not o[at:at + max(n - L, 0)].any()
            at += n


@pytest.mark.parametrize("scale", [-SCALE, 0.0, -0.0, 1e-30, 2.0, -1e-45])
def test_scale_of_any_sign(scale):
    m = Model(1, 2, 150, seed=35)
    m.append([150, 70])
    m.check_attention(2, [1, 1], scale=scale, label="scale")
    m.check_attention(2, [150, 33], scale=scale, label="scale")


@pytest.mark.parametrize("steps", ["rising", "falling", "zigzag", "values"])
def test_blocks_of_differing_size(steps):
    # block scales that move by powers of ten: the running maximum jumps, and
    # with it what the values' scales are taken relative to
    L, H = 640, 4
    m = Model(1, 1, L, seed=36)
    k, v = oracle._f32(m.values(L, 1)), oracle._f32(m.values(L, 1))
    e = np.repeat(np.arange(10), 64)[:, None, None]
    size = {"rising": e - 5, "falling": 5 - e, "zigzag": 6 * (e % 2) - 3, "values": 0 * e}[steps]
    k = k * 2.0 ** np.clip(size, -5, 2)
    v = v * 10.0 ** (size * (3 if steps == "values" else 1) + (steps == "values") * (7 * (e % 3) - 7))
    m.append([L], I.to_bf16_bits(k.astype(np.float32)), I.to_bf16_bits(v.astype(np.float32)))
    for n in (1, 70):
        m.check_attention(H, [n], label=steps)
    m.check_attention(H, [20], scale=20 * SCALE, label=steps + " peaked")


SIZES = [(None, 57), (-90, 45), (-60, 85), (-90, 98), (None, 24), (-53, 24)]  # (the last two: as far apart as the plain way holds)


def sized_values(m, L, pair, order, blk=BLK):
    """bf16 values [L][1][D] whose blocks are of two sizes, 2^pair (None: zeros)."""
    blocks = -(-L // blk)
    which = {"low first": lambda i: i >= blocks // 2, "high first": lambda i: i < blocks // 2, "in turn": lambda i: i % 2 == 1}[order]
    size = np.array([0.0 if pair[which(i)] is None else 2.0 ** pair[which(i)] for i in range(blocks)])
    return I.to_bf16_bits((oracle._f32(m.values(L, 1)) * np.repeat(size, blk)[:L, None, None]).astype(np.float32))


@pytest.mark.parametrize("order", ["low first", "high first", "in turn"])
@pytest.mark.parametrize("pair", SIZES)
def test_values_of_very_different_size(pair, order):
    # blocks whose values are far smaller than others' (or zero) keep their part of the softmax's total: within a
    # wave, between the waves of a workgroup and between splits
    for L, H, news in ((768, 4, (1, 16)), (9000, 4, (1,))):
        m = Model(1, 1, L, seed=57)
        m.append([L], I.to_bf16_bits((0.3 * oracle._f32(m.values(L, 1))).astype(np.float32)), sized_values(m, L, pair, order))
        for n in news:
            m.check_attention(H, [n], label=f"sizes {pair} {order}")


@pytest.mark.parametrize("pair", SIZES)
@pytest.mark.parametrize("n,H", [(150, 32), (400, 32), (768, 32)])
def test_values_of_very_different_size_in_many_rows(n, H, pair):
    # the forms of more rows a workgroup
    L = 768
    m = Model(1, 1, L, seed=58)
    m.append([L], I.to_bf16_bits((0.3 * oracle._f32(m.values(L, 1))).astype(np.float32)), sized_values(m, L, pair, "in turn"))
    m.check_attention(H, [n], label=f"sizes {pair}")


@pytest.mark.parametrize("blocks,B", [(1 << 14, 1), (1 << 13, 64), (1 << 13, 600)])
def test_many_tokens_with_tiny_values(blocks, B):
    # the total counts in units of the values' scale, here the smallest: 2^19 and more equal weights have to fit it.
    # Every block is the same page, every score 0, so the output is the mean of the page's values
    g = np.random.Generator(np.random.PCG64(59))
    codes = g.integers(1, 128, (D, BLK)).astype(np.int8)
    cache = w.KVCache.empty(1, 1, 1, device=dev())
    cache.v_codes[0, 0] = torch.from_numpy(codes).to(dev())
    cache.k_codes.copy_(torch.from_numpy(g.integers(-127, 128, tuple(cache.k_codes.shape)).astype(np.int8)).to(dev()))
    cache.scales[0, 0, 0], cache.scales[0, 0, 1] = 1.0, 2.0 ** -97
    L = blocks * BLK
    cos, sin = torch.ones(4, D // 2, device=dev()), torch.zeros(4, D // 2, device=dev())
    q = torch.zeros(B, 4, D, dtype=torch.bfloat16, device=dev())
    o = w.w4a8_cache_attention(q, cache, i32(np.arange(B + 1)), i32([L] * B), i32(np.zeros((B, blocks))), i32([0] * B), cos, sin, SCALE)
    want = codes.astype(np.float64).mean(1) * 2.0 ** -97
    # all weights are one power of two, exact in fp16, so numerators and totals are integers times a power of two, exact in
    # fp32 below 2^24: in every wave of a split (2^17 tokens of at most 127).  Then the merges, and the rounding to bf16
    tol = (2.0 ** -8 + 2.0 ** -14) * want
    assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("size", [10, 17, 18, 20, 30, 50, 90])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(size, sign):
    # scores up to 2^(size + 14): integers times a unit that is far above 1, so that the heaviest keys alone count, equally.
    # Queries and keys have one element, the tables turn nothing: the query's 16 bits are exact, and so are the products
    L, H = 640, 4
    m = Model(1, 1, L, seed=60)
    m.cos, m.sin = np.ones_like(m.cos), np.zeros_like(m.sin)
    m.dcos, m.dsin = torch.from_numpy(m.cos).to(dev()), torch.from_numpy(m.sin).to(dev())
    k = np.zeros((L, 1, D), np.float32)
    k[:, 0, 60] = m.rng.integers(-127, 128, L)
    if sign < 0:
        k[:, 0, 60] = -np.abs(k[:, 0, 60]) - (k[:, 0, 60] == 0)
    k[::BLK, 0, 60] = -127  # every block's scale is 1
    k[[100, 333, 600], 0, 60] = np.abs(k[:, 0, 60]).max() if sign > 0 else -1
    v = oracle._f32(m.values(L, 1)).clip(-4, 4)
    v[::BLK, 0, 5] = 8.0  # and every block's values have the same
    m.append([L], I.to_bf16_bits(k), I.to_bf16_bits(v))
    for n in (1, 20, 200):
        q = np.zeros((n, H, D), np.float32)
        q[:, :, 60] = 2.0 ** size * np.array([1.0, 1.5, 1.25, 64.0])
        q = I.to_bf16_bits(q)
        print(f"[case] large scores 2^{size} sign {sign} n={n}", flush=True)
        o = m.attend(bf16_dev(q), [n], scale=1.0).double().cpu().numpy()
        kc, vc, sc, _, _ = m.held()
        pages = m.table[0]
        kk = (kc[pages].astype(np.float64) * sc[pages, :, 0, None, None]).transpose(1, 0, 2, 3).reshape(1, -1, D)
        vv = (vc[pages].astype(np.float64) * sc[pages, :, 1, None, None]).transpose(1, 0, 3, 2).reshape(1, -1, D)
        o64, bnd, _, peak = oracle.cache_attention(q, np.arange(n), kk, vv, m.cos, m.sin, 1.0, L - n)
        # the bound above without the query's rounding; other keys' weights are exp(-2^10) and less
        tol = 2.0 ** -8 * np.abs(o64) + (1 + 2.0 ** -8) * ((2.0 ** -11 + 2.0 ** -14) * bnd + 2.0 ** -37 * peak[..., None])
        assert (np.abs(o - o64) <= tol).all()


def test_a_heavy_key_with_small_values():
    # nearly all weight on keys whose values are tiny (or zero): what the others add has to keep its precision
    L = 2000
    m = Model(1, 1, L, seed=37)
    q = np.zeros((1, 4, D), np.float32)
    q[..., 60] = 8.0
    k = 0.1 * m.rng.standard_normal((L, 1, D)).astype(np.float32)
    k[:, :, 60] = 0.0
    k[3, :, 60] = 14.0
    v = m.rng.standard_normal((L, 1, D)).astype(np.float32)
    for tiny in (1e-4, 0.0):
        v[:64] *= tiny
        m2 = Model(1, 1, L, seed=38)
        m2.append([L], I.to_bf16_bits(k), I.to_bf16_bits(v))
        m2.check_attention(4, [1], label="heavy key", q_bits=I.to_bf16_bits(q))


def test_stale_codes_and_scales_are_not_seen():
    # what lies past a sequence's end or in pages that a row does not reach may hold anything
    m = Model(2, 2, 300, seed=39)
    m.append([130, 200])
    new = [40, 150]
    q = m.values(sum(new), 8)
    want = m.attend(bf16_dev(q), new).clone()
    c = m.cache
    for b, L in enumerate((130, 200)):
        p = int(m.table[b, (L - 1) // BLK])
        c.k_codes[p, :, L % BLK:] = -128
        c.v_codes[p, :, :, L % BLK:] = -128
        rest = i32(m.table[b, (L - 1) // BLK + 1:]).long()
        c.scales[rest] = float("inf")
        c.k_codes[rest] = 127
    assert torch.equal(m.attend(bf16_dev(q), new), want)
    # a block whose scales are no numbers: rows before it do not see it
    p = int(m.table[1, 3])
    c.scales[p] = float("nan")
    o = m.attend(bf16_dev(q), new)
    first = 40 + (3 * BLK - 50)  # sequence 1's new tokens begin at 50; its block 3 is seen from token 192 on
    assert torch.equal(o[:first], want[:first]) and o[first:].isnan().all()


@pytest.mark.parametrize("n", [1, 16, 150])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_queries_that_are_no_numbers(n, what):
    # they make their own row's output NaN and no other's
    m = Model(2, 2, 300, seed=52)
    m.append([300, 170])
    q = bf16_dev(m.values(2 * n, 8))
    want = m.attend(q, [n, n]).clone()
    bad = q.clone()
    bad[n - 1, 5, 77] = float(what)
    bad[n, 0, 3] = float(what)
    o = m.attend(bad, [n, n])
    hit = torch.zeros(2 * n, 8, dtype=torch.bool, device=dev())
    hit[n - 1, 5] = hit[n, 0] = True
    assert o[hit].isnan().all() and torch.equal(o[~hit], want[~hit])


@pytest.mark.parametrize("n", [1, 16, 150])
def test_rows_beside_large_ones(n):
    # queries with large scores, and a block with values out of the usual range that only the last rows see, leave the
    # other rows' results as they are
    m = Model(2, 2, 400, seed=62)
    m.append([300, 192 + n])
    q = bf16_dev(m.values(2 * n, 8))
    want = m.attend(q, [n, n]).clone()
    large = q.clone()
    large[n - 1, 5] *= 2.0 ** 40
    large[n, 0] *= -(2.0 ** 40)
    m.cache.scales[int(m.table[1, (191 + n) // BLK]), :, 1] *= 2.0 ** 60
    o = m.attend(large, [n, n])
    hit = torch.zeros(2 * n, 8, dtype=torch.bool, device=dev())
    hit[n - 1, 5] = hit[n, 0] = True
    last = ((191 + n) // BLK) * BLK - 192  # sequence 1's new tokens from here on see its last block
    hit[n + max(last, 0):] = True
    assert torch.equal(o[~hit], want[~hit]) and o.isfinite().all()


def test_pages_out_of_range_are_not_seen():
    m = Model(2, 1, 320, seed=40)
    m.append([320])
    q = m.values(3, 8)
    for bad in (-1, m.cache.k_codes.shape[0], 1 << 30):
        table = i32(m.table)
        table[0, 1] = bad
        table[0, 3] = bad
        print(f"[case] page {bad}", flush=True)
        starts, lengths, _, pos = m.batch([3])
        o = w.w4a8_cache_attention(bf16_dev(q), m.cache, starts, lengths, table, pos, m.dcos, m.dsin, SCALE).float().cpu().numpy()
        # the same as a sequence of the blocks that are there
        kc, vc, sc, _, _ = m.held()
        pages = m.table[0, [0, 2, 4]]
        k = (kc[pages].astype(np.float64) * sc[pages, :, 0, None, None]).transpose(1, 0, 2, 3).reshape(2, -1, D)
        v = (vc[pages].astype(np.float64) * sc[pages, :, 1, None, None]).transpose(1, 0, 3, 2).reshape(2, -1, D)
        got = oracle.cache_attention(q, np.arange(317, 320), k, v, m.cos, m.sin, SCALE, 189)
        assert (np.abs(o - got[0]) <= tolerance(*got, k, SCALE)).all()


def test_layouts_of_queries_and_output():
    m = Model(2, 2, 90, seed=41)
    m.append([90, 70])
    new, H = [20, 7], 8
    q = bf16_dev(m.values(27, H))
    want = m.attend(q, new)
    heads_first = q.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    wide = torch.zeros(27, H + 5, 2 * D, dtype=torch.bfloat16, device=dev())
    wide[:, 3:3 + H, D:] = q
    for view in (heads_first, wide[:, 3:3 + H, D:]):
        assert torch.equal(m.attend(view, new), want)
    out = torch.zeros(H, 27, D, dtype=torch.bfloat16, device=dev()).permute(1, 0, 2)
    assert m.attend(q, new, out=out) is out and torch.equal(out, want)
    out = torch.full((27, H + 5, 2 * D), 7.0, dtype=torch.bfloat16, device=dev())
    m.attend(q, new, out=out[:, 3:3 + H, D:])
    assert torch.equal(out[:, 3:3 + H, D:], want)
    out[:, 3:3 + H, D:] = 7.0
    assert (out == 7.0).all()


def test_shared_pages():
    # two sequences that begin with the same blocks
    m = Model(2, 2, 200, seed=42)
    m.append([150, 0])
    m.table[1, :2] = m.table[0, :2]
    m.k[1], m.v[1] = m.k[0][:128], m.v[0][:128]
    m.append([3, 20])
    m.check_attention(8, [3, 20], label="shared pages")


def test_pages_past_32_bit_offsets():
    # a pool of more than 4 GiB of codes: the pages at its end
    Hkv, L = 8, 200
    m = Model(Hkv, 1, L, seed=43, pages=66000)
    m.table[0] = [65999, 65535, 32768, 65999 - 7]
    for t in m.cache[:2]:
        assert t.numel() > 1 << 32
    k, v = m.values(L, Hkv), m.values(L, Hkv)
    m.append([L], k, v)
    c, pages = m.cache, i32(m.table[0]).long()
    small = Model(Hkv, 1, L, seed=43)
    small.append([L], k, v)
    to = i32(small.table[0]).long()
    for x, y in zip(c[:3], small.cache[:3]):
        assert torch.equal(x[pages].view(torch.int8), y[to].view(torch.int8))
    q = bf16_dev(m.values(5, 32))
    assert torch.equal(m.attend(q, [5]), small.attend(q, [5]))


def test_positions_at_the_ends():
    # positions outside the tables take their ends, in both calls
    m = Model(1, 1, 64, seed=44)
    k, v, q = m.values(8, 1), m.values(8, 1), m.values(8, 2)
    starts, lengths, tab = i32([0, 8]), i32([8]), i32(m.table)
    outs = []
    for pos in ([-5, 0, 63, 64, np.iinfo(np.int32).max, np.iinfo(np.int32).min, 1, 2], [0, 0, 63, 63, 63, 0, 1, 2]):
        w.w4a8_cache_append(bf16_dev(k), bf16_dev(v), m.cache, starts, lengths, tab, i32(pos), m.dcos, m.dsin)
        o = w.w4a8_cache_attention(bf16_dev(q), m.cache, starts, lengths, tab, i32(pos), m.dcos, m.dsin, SCALE)
        outs.append((o, *(t.clone() for t in m.cache)))
    for x, y in zip(*outs):
        assert torch.equal(x.view(torch.int8), y.view(torch.int8))


def test_repeated_calls_agree():
    for new, L in (([1], [9000]), ([16, 16], [900, 333]), ([300], [700])):
        m = Model(2, len(new), max(L), seed=45)
        m.append(L)
        q = bf16_dev(m.values(sum(new), 8))
        first = m.attend(q, new)
        for i in range(20):
            again = m.attend(q, new)
            assert torch.equal(again.view(torch.int16), first.view(torch.int16)), (new, i)


def test_side_streams_and_two_calls_at_once():
    m = Model(2, 1, 4000, seed=46)
    m.append([4000])
    q = bf16_dev(m.values(1, 8))
    want = m.attend(q, [1])
    a, b = torch.cuda.Stream(dev()), torch.cuda.Stream(dev())
    args = m.batch([1])
    torch.cuda.synchronize()
    for i in range(10):  # each with a temporary workspace of its own
        outs = [w.w4a8_cache_attention(q, m.cache, *args, m.dcos, m.dsin, SCALE, stream=s) for s in (a, b)]
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o, want), i
    with torch.cuda.stream(a):
        assert torch.equal(m.attend(q, [1]), want)


def test_workspace_shared_with_the_linear():
    ws = w.Workspace(dev())
    M, N, K = 1, 16, 65536
    assert "S=8 " in w.w4a8_linear_describe(M, N, K, 0, 0)
    x, (W, s) = I.activations(M, K, 47), I.weights(N, K, 48)
    wp = w.w4a8_pack_weights(torch.from_numpy(W).to(dev()))
    want = oracle.linear(x, W, s_w=s, nthreads=8)["y"]
    m = Model(1, 1, 5000, seed=49)
    m.append([5000])
    q = bf16_dev(m.values(1, 8))
    o = m.attend(q, [1])
    for i in range(3):
        assert torch.equal(m.attend(q, [1], workspace=ws), o)
        y = w.w4a8_linear(bf16_dev(x), wp, torch.from_numpy(s).to(dev()), N, workspace=ws)
        np.testing.assert_array_equal(to_np_bits(y), want)


def test_graph_of_a_step():
    # append and attention captured once; the replays follow the batch's arrays
    m, H = Model(2, 3, 400, seed=50), 8
    m.append([60, 127, 300])
    T = 3 * 4
    k, v, q = (torch.empty(T, n, D, dtype=torch.bfloat16, device=dev()) for n in (2, 2, H))
    starts, lengths, tab, pos = i32([0, 4, 8, 12]), i32([0, 0, 0]), i32(m.table), i32([0] * T)
    out = torch.empty(T, H, D, dtype=torch.bfloat16, device=dev())
    ws = torch.zeros(w.w4a8_cache_attention_workspace_bytes(3, T, H, 2, 400), dtype=torch.uint8, device=dev())
    ws2 = w.Workspace(dev())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        w.w4a8_cache_append(k, v, m.cache, starts, lengths, tab, pos, m.dcos, m.dsin)
        w.w4a8_cache_attention(q, m.cache, starts, lengths, tab, pos, m.dcos, m.dsin, SCALE, out=out, workspace=ws)
    torch.cuda.synchronize()
    for rep in range(5):
        kb, vb, qb = m.values(T, 2), m.values(T, 2), m.values(T, H)
        for b in range(3):
            p = np.repeat(np.arange(len(m.k[b]), len(m.k[b]) + 4), 2)
            rot = oracle.rope_rotate(kb[4 * b:4 * b + 4].reshape(-1, D), p, m.cos, m.sin).reshape(4, 2, D)
            m.k[b], m.v[b] = np.concatenate([m.k[b], rot]), np.concatenate([m.v[b], vb[4 * b:4 * b + 4]])
        for dst, src in ((k, bf16_dev(kb)), (v, bf16_dev(vb)), (q, bf16_dev(qb))):
            dst.copy_(src)
        for dst, src in zip((starts, lengths, pos), (m.batch([4, 4, 4])[i] for i in (0, 1, 3))):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        m.check_cache()
        assert torch.equal(out, m.attend(bf16_dev(qb), [4, 4, 4], workspace=ws2)), rep
        o64, tol = m.expect(qb, [4, 4, 4])
        assert (np.abs(out.float().cpu().numpy() - o64) <= tol).all(), rep


def test_graphs_that_share_a_workspace():
    # two captured calls with one workspace, replayed in turn with the linear's
    # counters in front of their partial results
    ms = [Model(2, 1, 3000, seed=52), Model(1, 2, 2000, seed=53)]
    new, heads = ([2], [1, 3]), (8, 4)
    ws = w.Workspace(dev())
    ws.get(max(w.w4a8_cache_attention_workspace_bytes(m.B, sum(n), H, m.Hkv, m.blocks * BLK) for m, n, H in zip(ms, new, heads)))
    calls = []
    for m, n, H in zip(ms, new, heads):
        m.append([m.blocks * BLK - 70] * m.B)
        q, args = torch.empty(sum(n), H, D, dtype=torch.bfloat16, device=dev()), m.batch(n)
        assert w.w4a8_cache_attention_workspace_bytes(m.B, sum(n), H, m.Hkv, m.blocks * BLK) > 0
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = w.w4a8_cache_attention(q, m.cache, *args, m.dcos, m.dsin, SCALE, workspace=ws)
        calls.append((graph, m, n, H, q, o, args))  # the graph reads all of them
    for rep in range(6):
        qs = [bf16_dev(m.values(sum(n), H)) for _, m, n, H, *_ in calls]
        for (graph, _, _, _, q, _, _), new_q in zip(calls, qs):
            q.copy_(new_q)
            graph.replay()
        torch.cuda.synchronize()
        for (_, m, n, _, _, o, _), new_q in zip(calls, qs):
            assert torch.equal(o, m.attend(new_q, n)), rep
    assert not ws.buf[:65536].any()


def test_rounds_past_the_pages_held_at_a_time():
    # a workgroup holds the pages of 64 rounds: more of them, in 128 rows ..
    m = Model(1, 1, 9100, seed=54)
    m.append([9050])
    q = m.values(1600, 16)
    assert w.w4a8_cache_attention_workspace_bytes(1, 1600, 16, 1, 9152) == 0  # not split
    o = m.attend(bf16_dev(q), [1600])
    torch.cuda.synchronize()
    o64, tol = m.expect(q[-6:], [6])
    assert (np.abs(o[-6:].float().cpu().numpy() - o64) <= tol + 1e-30).all()
    o64, tol = m.expect(q[:6], [6], lengths=[9050 - 1600 + 6])
    assert (np.abs(o[:6].float().cpu().numpy() - o64) <= tol + 1e-30).all()
    # .. and in 64 rows, of sequences that share their pages (a shorter length's
    # last page still holds the tokens after it, which no row sees)
    B, n = 256, 4
    for L in (9050, 4400):
        m.cut(0, L)
        pos, tab = i32(np.tile(np.arange(L - n, L), B)), i32(np.repeat(m.table, B, 0))
        if L == 9050:  # two splits of 71 blocks
            assert w.w4a8_cache_attention_workspace_bytes(B, B * n, 16, 1, L) == 65536 + 2 * B * n * 16 * (D + 2) * 4
        q = m.values(n, 16)
        o = w.w4a8_cache_attention(bf16_dev(np.tile(q, (B, 1, 1))), m.cache, i32(np.arange(B + 1) * n), i32([L] * B), tab, pos, m.dcos,
                                   m.dsin, SCALE, max_len=L).view(B, n, 16, D)
        assert torch.equal(o, o[:1].expand_as(o)), L
        o64, tol = m.expect(q, [n])
        assert (np.abs(o[0].float().cpu().numpy() - o64) <= tol + 1e-30).all(), L


def test_cache_that_is_read_past_the_memory_side_cache():
    # the upper bound of the lengths decides; the sequences are short
    m, new, H = Model(8, 3, 700, seed=56), [1, 4, 2], 32
    m.append([700, 64, 129])
    q, max_len = m.values(7, H), 30000
    starts, lengths, tab, pos = m.batch(new)
    wide = torch.full((3, -(-max_len // BLK)), -1, dtype=torch.int32, device=dev())
    wide[:, :m.blocks] = tab
    o64, tol = m.expect(q, new)
    for bound in (700, max_len):
        o = w.w4a8_cache_attention(bf16_dev(q), m.cache, starts, lengths, wide, pos, m.dcos, m.dsin, SCALE, max_len=bound)
        assert (np.abs(o.float().cpu().numpy() - o64) <= tol + 1e-30).all(), bound


def test_more_row_blocks_than_an_axis_of_a_launch_holds():
    # one key each: the output is its value, whatever the query
    B, pages = 65536, 90
    m = Model(1, pages, 64, seed=55)
    m.append([1] * pages)
    new = np.ones(B, int)
    new[::7] = 2  # the first of two tokens sees nothing
    starts = np.concatenate([[0], np.cumsum(new)])
    T = int(starts[-1])
    q = bf16_dev(np.broadcast_to(m.values(1, 1), (T, 1, D)).copy())
    seq = np.arange(B) % pages
    o = w.w4a8_cache_attention(q, m.cache, i32(starts), i32(np.ones(B)), i32(m.table[seq]), i32(np.zeros(T)), m.dcos, m.dsin, SCALE)
    o = o[:, 0].double().cpu().numpy()
    kc, vc, sc, _, _ = m.held()
    p = m.table[seq, 0]
    v = vc[p, 0, :, 0].astype(np.float64) * sc[p, 0, 1, None]
    last = starts[1:] - 1
    # the weight and the total are the same number but for the rounding to
    # fp16 (2^-11) and fp32's products (2^-14 is far above), and one to bf16
    assert (np.abs(o[last] - v) <= (2.0 ** -8 + (1 + 2.0 ** -8) * (2.0 ** -11 + 2.0 ** -14)) * np.abs(v)).all()
    assert (o[starts[:-1][new == 2]] == 0).all()


def test_refusals():
    m = Model(2, 2, 64, seed=51)
    m.append([3, 2])
    k = bf16_dev(m.values(5, 2))
    q = bf16_dev(m.values(5, 8))
    starts, lengths, tab, pos = m.batch([3, 2])
    ok = (starts, lengths, tab, pos, m.dcos, m.dsin)
    for i, t in ((0, starts[:2]), (1, lengths[:1]), (2, tab[:1]), (2, tab[0]), (3, pos[:4]), (4, m.dcos[:, :32])):
        args = list(ok)
        args[i] = t
        with pytest.raises(ValueError):
            w.w4a8_cache_append(k, k, m.cache, *args)
        with pytest.raises(ValueError):
            w.w4a8_cache_attention(q, m.cache, *args, SCALE)
    for i in range(4):
        args = list(ok)
        args[i] = args[i].long()
        with pytest.raises(TypeError):
            w.w4a8_cache_attention(q, m.cache, *args, SCALE)
        args[i] = ok[i].cpu()
        with pytest.raises(TypeError):
            w.w4a8_cache_append(k, k, m.cache, *args)
    with pytest.raises(ValueError):
        w.w4a8_cache_append(k, k, m.cache._replace(k_recent=None), *ok)
    for bad in (m.cache._replace(scales=m.cache.scales[:-1]), m.cache._replace(v_codes=m.cache.k_codes), m.cache._replace(k_codes=m.cache.k_codes[..., :64])):
        with pytest.raises(ValueError):
            w.w4a8_cache_attention(q, bad, *ok, SCALE)
    with pytest.raises(ValueError):
        w.w4a8_cache_append(k, k[:4], m.cache, *ok)
    with pytest.raises(ValueError):
        w.w4a8_cache_append(k, k, m.cache, *ok, slots=i32([0]))
    with pytest.raises(TypeError):
        w.w4a8_cache_attention(q.half(), m.cache, *ok, SCALE)
    with pytest.raises(ValueError):
        w.w4a8_cache_attention(q.transpose(1, 2), m.cache, *ok, SCALE)
    with pytest.raises(ValueError):
        w.w4a8_cache_attention(q, m.cache, *ok, SCALE, out=q[:4])
    for kw in (dict(max_len=0), dict(max_len=65), dict(out=q[:1].expand(5, 8, D))):
        with pytest.raises(w.W4A8Error):
            w.w4a8_cache_attention(q, m.cache, *ok, SCALE, **kw)
    with pytest.raises(w.W4A8Error):  # query heads that the kv heads do not divide
        w.w4a8_cache_attention(q[:, :7], m.cache, *ok, SCALE)
    with pytest.raises(w.W4A8Error):  # rows that are not 16-byte aligned
        w.w4a8_cache_attention(torch.zeros(5 * 8 * D + 4, dtype=torch.bfloat16, device=dev())[4:].view(5, 8, D), m.cache, *ok, SCALE)
    none = w.w4a8_cache_attention(q[:0], m.cache, i32([0, 0, 0]), lengths, tab, pos[:0], m.dcos, m.dsin, SCALE)
    assert none.shape == (0, 8, D)
    w.w4a8_cache_append(k[:0], k[:0], m.cache, i32([0, 0, 0]), lengths, tab, pos[:0], m.dcos, m.dsin)


# ---------------------------------------------------------------- together


def test_a_layer_step_by_step():
    """A decoder layer's steps as a serving program runs them: the residual
    norm, qkv, append, attention, o, the residual norm, the gated MLP and
    down; a prompt's chunk and drafts of 4, with 2 tokens taken back.  Each
    call's output is checked against the oracle on that call's own inputs."""
    H, Hkv, K, F, B = 8, 2, 1024, 1536, 2
    rng_w = lambda N, KK, s: I.weights(N, KK, s)  # noqa: E731
    Wqkv, sqkv = rng_w((H + 2 * Hkv) * D, K, 60)
    Wo, so = rng_w(K, H * D, 61)
    Wgu, sgu = rng_w(2 * F, K, 62)
    Wd, sd = rng_w(K, F, 63)
    pk = lambda W: w.w4a8_pack_weights(torch.from_numpy(W).to(dev()))  # noqa: E731
    sc = lambda s: torch.from_numpy(s).to(dev())  # noqa: E731
    g = [I.activations(1, K, 64 + i, outliers=False)[0] for i in range(2)]
    gd = [bf16_dev(x) for x in g]
    wq, wo, wg, wd = pk(Wqkv), pk(Wo), pk(Wgu), pk(Wd)
    m = Model(Hkv, B, 200, seed=65)
    ws = w.Workspace(dev())
    for step, new in enumerate(([70, 33], [4, 4], [4, 4])):
        T = sum(new)
        if step == 2:
            for b in range(B):
                m.cut(b, len(m.k[b]) - 2)
        x, res = bf16_dev(I.activations(T, K, 70 + step)), bf16_dev(I.activations(T, K, 80 + step))
        resid0 = to_np_bits(res)
        print(f"[case] layer step {step} new={new}", flush=True)
        q8, s8, res = w.w4a8_add_rmsnorm_quantize_act(x, res, gd[0], 1e-6, out=res)
        qo, so_, to = oracle.add_rmsnorm_quantize(to_np_bits(x), resid0, g[0], 1e-6)
        np.testing.assert_array_equal(q8.cpu().numpy(), qo)
        np.testing.assert_array_equal(to_np_bits(res), to)
        qkv = w.w4a8_linear(q8, wq, sc(sqkv), (H + 2 * Hkv) * D, x_scale=s8, workspace=ws)
        np.testing.assert_array_equal(to_np_bits(qkv), oracle.linear_q(qo, so_, Wqkv, s_w=sqkv)["y"])
        heads = qkv.view(T, H + 2 * Hkv, D)
        bits = to_np_bits(qkv).reshape(T, H + 2 * Hkv, D)
        at = 0
        for b, n in enumerate(new):
            p = np.repeat(np.arange(len(m.k[b]), len(m.k[b]) + n), Hkv)
            rot = oracle.rope_rotate(bits[at:at + n, H:H + Hkv].reshape(-1, D), p, m.cos, m.sin).reshape(n, Hkv, D)
            m.k[b], m.v[b] = np.concatenate([m.k[b], rot]), np.concatenate([m.v[b], bits[at:at + n, H + Hkv:]])
            at += n
        starts, lengths, tab, pos = m.batch(new)
        w.w4a8_cache_append(heads[:, H:H + Hkv], heads[:, H + Hkv:], m.cache, starts, lengths, tab, pos, m.dcos, m.dsin)
        o = w.w4a8_cache_attention(heads[:, :H], m.cache, starts, lengths, tab, pos, m.dcos, m.dsin, SCALE, workspace=ws)
        m.check_cache()
        o64, tol = m.expect(bits[:, :H], new)
        assert (np.abs(o.float().cpu().numpy() - o64) <= tol).all()
        y = w.w4a8_linear(o.view(T, H * D), wo, sc(so), K, workspace=ws)
        np.testing.assert_array_equal(to_np_bits(y), oracle.linear(to_np_bits(o).reshape(T, H * D), Wo, s_w=so)["y"])
        before = to_np_bits(res)
        q8, s8, res = w.w4a8_add_rmsnorm_quantize_act(y, res, gd[1], 1e-6, out=res)
        qo, so_, to = oracle.add_rmsnorm_quantize(to_np_bits(y), before, g[1], 1e-6)
        np.testing.assert_array_equal(q8.cpu().numpy(), qo)
        np.testing.assert_array_equal(to_np_bits(res), to)
        h = w.w4a8_linear_swiglu(q8, wg, sc(sgu), 2 * F, x_scale=s8, workspace=ws)
        z = w.w4a8_linear(h, wd, sc(sd), K, workspace=ws)
        np.testing.assert_array_equal(to_np_bits(z), oracle.linear(to_np_bits(h), Wd, s_w=sd)["y"])
