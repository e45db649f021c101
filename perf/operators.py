"""Performance cases of a decoder layer's step around its 8-bit key/value cache.

Three operators, each called as a serving program calls it, on tensors that
are already on the GPU:

  norm       the residual's addition, RMSNorm and the int8 quantize in front
             of a projection
  append     new keys (rotated at their positions) and values into a paged
             cache of int8 codes with a scale for each block of 64 tokens and
             kv head
  attention  the new tokens' attention over that cache

The sizes are those of the decoder layer that the package's inputs describe
(hidden 4096, 32 query heads on 8 kv heads of 128, MLP width 12288) and of
other head counts; queries, keys and values are views of one projection's
output, [tokens][(H + 2 Hkv) * 128].

A batch of B sequences: `starts` [B + 1] are the rows of the new tokens,
`lengths` [B] the tokens a sequence holds with its new ones, `table` [B][..]
the pages of its blocks.  Cases with `ragged` have lengths and counts of new
tokens that differ from sequence to sequence.

`own` picks the framework's kernels; otherwise the operators run in their
plain form.  Codes are returned as the values that they stand for.
"""
import math
import random

import torch

own = False

D = 128            # head dimension
BLOCK = 64         # tokens of a block (a page of the table)
RECENT = 2 * BLOCK # tokens of a sequence's ring of exact values
EPS = 1e-6
TINY = 2.0 ** -90  # a block whose largest magnitude lies below is held as zeros


def listed():
    return [
        # one token of plain decoding: the residual and norm in front of a projection
        dict(name="norm_m1", kind="norm", M=1, K=4096),
        # a ragged number of new-frame tokens
        dict(name="norm_m777", kind="norm", M=777, K=4096),
        # a whole window's prefill
        dict(name="norm_m2048", kind="norm", M=2048, K=4096),
        # one new token each of 16 short sequences
        dict(name="append_b16_n1", kind="append", B=16, n=1, L=256, H=32, Hkv=8, ragged=True, mix=1),
        # the draft blocks of a few sequences, some of them ending inside a page
        dict(name="append_b5_n16", kind="append", B=5, n=16, L=500, H=32, Hkv=8, ragged=True, mix=2),
        # a prompt chunk of one sequence
        dict(name="append_n1024", kind="append", B=1, n=1024, L=1024, H=32, Hkv=8, ragged=False, mix=0),
        # one token of one sequence over a short cache, where latency counts
        dict(name="decode_b1_l1023", kind="attention", B=1, n=1, L=1023, H=32, Hkv=8, ragged=False, mix=0),
        # plain decoding of 64 sequences: the most cache a pass reads
        dict(name="decode_b64_l4096", kind="attention", B=64, n=1, L=4096, H=32, Hkv=8, ragged=False, mix=0),
        # one token over a long cache
        dict(name="decode_b1_l100000", kind="attention", B=1, n=1, L=100000, H=32, Hkv=8, ragged=False, mix=0),
        # draft blocks of 16 tokens under verification
        dict(name="verify_b8_n16", kind="attention", B=8, n=16, L=2500, H=32, Hkv=8, ragged=False, mix=0),
        # a mixed batch: odd lengths, 1 to 33 new tokens a sequence, 7 query heads to a kv head
        dict(name="mixed_b12_n33", kind="attention", B=12, n=33, L=1900, H=28, Hkv=4, ragged=True, mix=3),
        # a prompt chunk over the tokens before it: the most arithmetic
        dict(name="prefill_n1024_l8192", kind="attention", B=1, n=1024, L=8192, H=32, Hkv=8, ragged=False, mix=0),
    ]


HEADS = [(32, 8), (28, 4), (16, 16), (8, 1), (16, 4), (40, 8)]
LARGEST = dict(rows=2048 * 4096, append=1024 * 8, codes=64 * 4096 * 8, pairs=1024 * 8192 * 32)


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choices(["norm", "append", "attention"], [2, 2, 5])[0]
    if kind == "norm":
        K = 128 * log_int(1, 96)
        return dict(kind="norm", M=min(log_int(1, 4096), LARGEST["rows"] // K), K=K)
    H, Hkv = rng.choice(HEADS)
    n = rng.choice([1, log_int(2, 32), log_int(33, 1024)])
    if kind == "append":
        c = dict(kind="append", B=log_int(1, 16), n=n, L=n + log_int(1, 500), H=H, Hkv=Hkv, ragged=rng.random() < 0.7, mix=rng.randrange(10 ** 6))
        while c["B"] > 1 and c["B"] * (c["L"] + BLOCK) * Hkv > LARGEST["append"]:
            c["B"] //= 2
        while c["L"] * Hkv > LARGEST["append"]:
            c["L"], c["n"] = c["L"] // 2, max(1, c["n"] // 2)
        return c
    c = dict(kind="attention", B=log_int(1, 64), n=n, L=n - 1 + log_int(1, 100000), H=H, Hkv=Hkv, ragged=rng.random() < 0.5, mix=rng.randrange(10 ** 6))
    while c["B"] > 1 and (c["B"] * c["L"] * Hkv > LARGEST["codes"] or c["B"] * c["n"] * c["L"] * H > LARGEST["pairs"]):
        c["B"] //= 2
    while c["L"] * Hkv > LARGEST["codes"] or c["n"] * c["L"] * H > LARGEST["pairs"]:
        c["L"] = max(n, c["L"] // 2)
        c["n"] = max(1, c["n"] * 3 // 4)
    return c


# ---------------------------------------------------------------- inputs


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _batch(c):
    """New tokens and lengths of each sequence (plain lists)."""
    r = random.Random(c["mix"])
    new, lengths = [], []
    for _ in range(c["B"]):
        n = r.randint(1, c["n"]) if c["ragged"] else c["n"]
        L = r.randint(max(n, c["L"] // 4), c["L"]) if c["ragged"] else c["L"]
        if c["kind"] == "append" and n > BLOCK:  # chunks of a prompt begin at a block
            L = (L - n) // BLOCK * BLOCK + n
        new.append(n)
        lengths.append(L)
    return new, lengths


def _tokens(g, M, K):
    """Activations: N(0, 1) with 1 % of the channels 20 times larger, in bf16."""
    x = torch.randn(M, K, generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[: round(0.01 * K)]] *= 20.0
    return x.to(torch.bfloat16)


def _norm_inputs(c, seed):
    g = _gen(seed)
    x = torch.randn(c["M"], c["K"], generator=g, device="cuda").to(torch.bfloat16)
    gamma = (1.0 + 0.1 * torch.randn(c["K"], generator=g, device="cuda")).to(torch.bfloat16)
    return x, _tokens(g, c["M"], c["K"]), gamma


def _heads(g, rows, n, spread):
    """Vectors of n heads: channels of differing size, as projections give them."""
    size = torch.exp(spread * torch.randn(n, D, generator=g, device="cuda"))
    return torch.randn(rows, n, D, generator=g, device="cuda") * size


def _quantized(x):
    """Codes and scales of blocks x [..][tokens][D]."""
    a = x.abs().amax((-2, -1))
    s = torch.where(a >= TINY, a / torch.full_like(a, 127.0), torch.zeros_like(a))  # a tensor divides; a number would multiply by its reciprocal
    q = torch.round(x / torch.where(s > 0, s, torch.ones_like(s))[..., None, None])
    return torch.where(s[..., None, None] > 0, q, torch.zeros_like(q)).to(torch.int8), s


def _cache_inputs(c, seed):
    """What both cache operators are given: one projection's output and the
    batch, and the cache as earlier steps left it."""
    g = _gen(seed)
    new, lengths = _batch(c)
    B, H, Hkv, T = c["B"], c["H"], c["Hkv"], sum(new)
    st = dict(c=c, T=T)
    st["qkv"] = torch.cat([_heads(g, T, H, 0.3), _heads(g, T, Hkv, 0.5), _heads(g, T, Hkv, 0.3)], 1).reshape(T, -1).to(torch.bfloat16)
    blocks = [-(-L // BLOCK) for L in lengths]
    pages = sum(blocks)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, max(blocks)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    pos = torch.cat([torch.arange(L - n, L) for n, L in zip(new, lengths)])
    as_i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).to("cuda")  # noqa: E731
    st.update(starts=as_i32(starts), lengths=as_i32(lengths), pos=as_i32(pos), table=table, max_len=max(lengths))
    inv = 1e6 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) * 2 / D)
    ang = torch.arange(max(lengths), device="cuda", dtype=torch.float64)[:, None] * inv
    st["cos"], st["sin"] = ang.cos().float(), ang.sin().float()
    k_codes = torch.empty(pages, Hkv, BLOCK, D, dtype=torch.int8, device="cuda")
    v_codes = torch.empty(pages, Hkv, D, BLOCK, dtype=torch.int8, device="cuda")
    scales = torch.empty(pages, Hkv, 2, device="cuda")
    for p in range(0, pages, 512):
        e = min(pages, p + 512)
        k = _heads(g, (e - p) * BLOCK, Hkv, 0.5).to(torch.bfloat16).float().view(e - p, BLOCK, Hkv, D).transpose(1, 2)
        v = _heads(g, (e - p) * BLOCK, Hkv, 0.3).to(torch.bfloat16).float().view(e - p, BLOCK, Hkv, D).transpose(1, 2)
        k_codes[p:e], scales[p:e, :, 0] = _quantized(k)
        q, scales[p:e, :, 1] = _quantized(v)
        v_codes[p:e] = q.transpose(2, 3)
    st.update(k_codes=k_codes, v_codes=v_codes, scales=scales)
    if c["kind"] == "append":
        st["k_recent"] = _heads(g, B * RECENT, Hkv, 0.5).view(B, RECENT, Hkv, D).transpose(1, 2).to(torch.bfloat16).contiguous()
        st["v_recent"] = _heads(g, B * RECENT, Hkv, 0.3).view(B, RECENT, Hkv, D).transpose(1, 2).to(torch.bfloat16).contiguous()
    return st, new, lengths


def prepare(case, seed):
    if case["kind"] == "norm":
        x, residual, gamma = _norm_inputs(case, seed)
        return dict(c=case, x=x, residual=residual, gamma=gamma)
    st, new, lengths = _cache_inputs(case, seed)
    B, H, Hkv, T = case["B"], case["H"], case["Hkv"], st["T"]
    heads = st["qkv"].view(T, H + 2 * Hkv, D)
    st["q"], st["k"], st["v"] = heads[:, :H], heads[:, H:H + Hkv], heads[:, H + Hkv:]
    # the host's own plan of the batch: which row is which token of which sequence
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(new)])
    idx = torch.cat([torch.arange(L - n, L) for n, L in zip(new, lengths)])
    st["seq"], st["idx"] = seq.to("cuda"), idx.to("cuda")
    if case["kind"] == "attention":
        st["row"] = torch.cat([torch.arange(n) for n in new]).to("cuda")
        st["n"] = max(new)
        st["ws"] = {}
        return st
    # append: the touched blocks, and where each of their tokens comes from (the rings, then the new rows)
    items, src, starts = [], [], 0
    for b, (n, L) in enumerate(zip(new, lengths)):
        for blk in range((L - n) // BLOCK, (L - 1) // BLOCK + 1):
            items.append((b, blk))
            t = torch.arange(blk * BLOCK, blk * BLOCK + BLOCK)
            src.append(torch.where(t >= L, -1, torch.where(t >= L - n, B * RECENT + starts + t - (L - n), b * RECENT + t % RECENT)))
        starts += n
    src = torch.stack(src)
    st["src"], st["live"] = src.clamp(min=0).to("cuda"), (src >= 0).to("cuda")
    st["page"] = st["table"][[b for b, _ in items], [k for _, k in items]].long()
    last = torch.tensor(lengths)[seq]
    st["kept"] = torch.nonzero(idx >= ((last - 1) // BLOCK - 1) * BLOCK)[:, 0].to("cuda")
    return st


# ---------------------------------------------------------------- the plain forms


def _plain_norm(st):
    h0 = (st["x"].float() + st["residual"].float()).to(torch.bfloat16)
    x = h0.float()
    v = (x.double().square().sum(1, keepdim=True) / x.shape[1]).float()
    r = 1.0 / (v + EPS).double().sqrt().float()
    h = (x * r) * st["gamma"].float()
    a = h.abs().amax(1, keepdim=True)
    s = a / torch.full_like(a, 127.0)
    q = torch.round(h / torch.where(s > 0, s, torch.ones_like(s)))
    return h0, q * s


def _rotated(x, pos, cos, sin):
    """Rotate-half of x [rows][heads][D] at pos [rows], in 32 bits."""
    c, s = cos[pos.long()][:, None], sin[pos.long()][:, None]
    a, b = x[..., :D // 2].float(), x[..., D // 2:].float()
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_append(st):
    k = _rotated(st["k"], st["pos"], st["cos"], st["sin"]).to(torch.bfloat16)
    for which, rows, recent in ((0, k, st["k_recent"]), (1, st["v"], st["v_recent"])):
        Hkv = rows.shape[1]
        old = recent.transpose(1, 2).reshape(-1, Hkv, D)
        x = torch.cat([old, rows])[st["src"]].float() * st["live"][:, :, None, None]
        q, s = _quantized(x.transpose(1, 2))
        st["scales"][st["page"], :, which] = s
        if which == 0:
            st["k_codes"][st["page"]] = q
        else:
            st["v_codes"][st["page"]] = q.transpose(2, 3)
        kept = st["kept"]
        recent[st["seq"][kept], :, st["idx"][kept] % RECENT] = rows[kept]
    return _append_outputs(st)


def _append_outputs(st):
    s = st["scales"]
    return dict(k=st["k_codes"] * s[:, :, 0, None, None], v=st["v_codes"] * s[:, :, 1, None, None], scales=s,
                k_recent=st["k_recent"], v_recent=st["v_recent"])


def _plain_attention(st):
    c = st["c"]
    B, H, Hkv, n = c["B"], c["H"], c["Hkv"], st["n"]
    G = H // Hkv
    page = st["table"].long().clamp(min=0)
    keys = page.shape[1] * BLOCK
    s = st["scales"][page]
    k = (st["k_codes"][page] * s[..., 0, None, None]).permute(0, 2, 1, 3, 4).reshape(B * Hkv, keys, D)
    v = (st["v_codes"][page] * s[..., 1, None, None]).permute(0, 2, 1, 4, 3).reshape(B * Hkv, keys, D)
    q = torch.zeros(B, n, H, D, device="cuda")
    q[st["seq"], st["row"]] = _rotated(st["q"], st["pos"], st["cos"], st["sin"])
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B * Hkv, n * G, D)
    p = torch.matmul(q, k.transpose(1, 2).contiguous()) * D ** -0.5
    index = torch.full((B, n), -1, device="cuda")
    index[st["seq"], st["row"]] = st["idx"]
    seen = torch.arange(keys, device="cuda") <= index[:, :, None]
    p = p.view(B, Hkv, n, G, keys).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B * Hkv, n * G, keys), v).view(B, Hkv, n, G, D) / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 2, 1, 3, 4).reshape(B, n, H, D)[st["seq"], st["row"]].to(torch.bfloat16)


# ---------------------------------------------------------------- the framework's calls


def _own(st):
    import paper_2608_12932_amd as w

    kind = st["c"]["kind"]
    if kind == "norm":
        q, s, h0 = w.w4a8_add_rmsnorm_quantize_act(st["x"], st["residual"], st["gamma"], EPS)
        return h0, q * s[:, None]
    cache = w.KVCache(st["k_codes"], st["v_codes"], st["scales"], st.get("k_recent"), st.get("v_recent"))
    if kind == "append":
        w.w4a8_cache_append(st["k"], st["v"], cache, st["starts"], st["lengths"], st["table"], st["pos"], st["cos"], st["sin"])
        return _append_outputs(st)
    if not st["ws"]:  # kept by the program from its first call on
        st["ws"]["ws"] = w.Workspace()
    return w.w4a8_cache_attention(st["q"], cache, st["starts"], st["lengths"], st["table"], st["pos"], st["cos"], st["sin"],
                                  D ** -0.5, max_len=st["max_len"], workspace=st["ws"]["ws"])


def run(state):
    if own:
        return _own(state)
    kind = state["c"]["kind"]
    return _plain_norm(state) if kind == "norm" else _plain_append(state) if kind == "append" else _plain_attention(state)


# ---------------------------------------------------------------- work


def work(case):
    c = case
    if c["kind"] == "norm":  # two inputs and the gains; the sum, the codes and their scales
        M, K = c["M"], c["K"]
        return {"bytes": 4 * M * K + 2 * K + 3 * M * K + 4 * M, "flops": 8 * M * K}
    new, lengths = _batch(c)
    H, Hkv, T = c["H"], c["Hkv"], sum(new)
    if c["kind"] == "append":
        # the rows, the exact values that the first block still has, codes and scales of the touched blocks, the rings
        # (not the values that the outputs above are turned into for comparison)
        touched = sum(min(L, ((L - 1) // BLOCK + 1) * BLOCK) - (L - n) // BLOCK * BLOCK for n, L in zip(new, lengths))
        old = sum((L - n) % BLOCK for n, L in zip(new, lengths))
        kept = sum(min(n, L - ((L - 1) // BLOCK - 1) * BLOCK) for n, L in zip(new, lengths))
        return {"bytes": 2 * Hkv * D * (2 * T + 2 * old + touched + 2 * kept) + T * D * 4, "flops": 2 * Hkv * D * (3 * T + 4 * touched)}
    pairs = sum(n * (L - n) + n * (n + 1) // 2 for n, L in zip(new, lengths))
    cache = sum(2 * L * Hkv * D + -(-L // BLOCK) * Hkv * 8 for L in lengths)
    return {"bytes": cache + 2 * T * H * D * 2 + T * D * 4, "flops": 4 * D * H * pairs}


# ---------------------------------------------------------------- 64-bit reference


def _turned(x, pos, cos, sin):
    """The rotation in 64 bits of 32-bit tables."""
    c, s = cos.double()[pos.long(), None], sin.double()[pos.long(), None]
    lo, hi = x.double().chunk(2, -1)
    return lo * c, hi * s, hi * c, lo * s


def _exact_norm(c, seed):
    x, residual, gamma = _norm_inputs(c, seed)
    h0 = (x.double() + residual.double()).float().to(torch.bfloat16)
    h = h0.double()
    ms = (h * h).mean(1, keepdim=True).float()
    inv = (1 / (ms + EPS).double().sqrt().float().double()).float()
    h = ((h * inv.double()).float().double() * gamma.double()).float().double()  # 32-bit steps, as the codes are defined
    s = (h.abs().amax(1, keepdim=True) / 127).float().double()
    code = torch.where(s > 0, (h / s.clamp(min=1e-300)).float().round().double(), 0.0)
    return h0.double(), code * s


def _exact_append(c, seed):
    st, new, lengths = _cache_inputs(c, seed)
    H, Hkv, T = c["H"], c["Hkv"], st["T"]
    rows = st["qkv"].view(T, H + 2 * Hkv, D)
    ac, bs, bc, as_ = _turned(rows[:, H:H + Hkv], st["pos"], st["cos"], st["sin"])
    f = lambda t: t.float().double()  # noqa: E731  (each step is a 32-bit one, by the definition)
    k = torch.cat([f(f(ac) - f(bs)), f(f(bc) + f(as_))], -1).to(torch.bfloat16)
    v = rows[:, H + Hkv:]
    s = st["scales"].double()
    out = dict(k=st["k_codes"].double() * s[:, :, 0, None, None], v=st["v_codes"].double() * s[:, :, 1, None, None])
    at = 0
    for b, (n, L) in enumerate(zip(new, lengths)):
        for which, name, x in ((0, "k", k), (1, "v", v)):
            ring = st[name + "_recent"][b]
            for blk in range((L - n) // BLOCK, (L - 1) // BLOCK + 1):
                lo, hi, mid = blk * BLOCK, min(L, blk * BLOCK + BLOCK), max(blk * BLOCK, L - n)
                held = torch.cat([ring[:, [t % RECENT for t in range(lo, mid)]], x[at + mid - (L - n):at + hi - (L - n)].transpose(0, 1)], 1).double()
                a = held.abs().amax((1, 2))
                sc = torch.where(a >= TINY, (a / 127).float().double(), 0.0)
                code = (held / sc.clamp(min=1e-300)[:, None, None]).float().round().double() * sc[:, None, None]
                page = int(st["table"][b, blk])
                s[page, :, which] = sc
                whole = torch.zeros(Hkv, BLOCK, D, dtype=torch.float64, device="cuda")
                whole[:, :hi - lo] = code
                out[name][page] = whole if name == "k" else whole.transpose(1, 2)
        for name, x in (("k", k), ("v", v)):  # the rings, once every block has been read
            first = max(L - n, ((L - 1) // BLOCK - 1) * BLOCK)
            st[name + "_recent"][b][:, [t % RECENT for t in range(first, L)]] = x[at + first - (L - n):at + n].transpose(0, 1)
        at += n
    return dict(out, scales=s, k_recent=st["k_recent"].double(), v_recent=st["v_recent"].double())


def _exact_attention(c, seed):
    st, new, lengths = _cache_inputs(c, seed)
    H, Hkv, T = c["H"], c["Hkv"], st["T"]
    ac, bs, bc, as_ = _turned(st["qkv"].view(T, H + 2 * Hkv, D)[:, :H], st["pos"], st["cos"], st["sin"])
    q = torch.cat([ac - bs, bc + as_], -1)
    out, at = torch.zeros(T, H, D, dtype=torch.float64, device="cuda"), 0
    for b, (n, L) in enumerate(zip(new, lengths)):
        pages = st["table"][b, :-(-L // BLOCK)].long()
        for h in range(Hkv):
            sc = st["scales"][pages, h].double()
            k = (st["k_codes"][pages, h].double() * sc[:, 0, None, None]).reshape(-1, D)[:L]
            v = (st["v_codes"][pages, h].double() * sc[:, 1, None, None]).transpose(1, 2).reshape(-1, D)[:L]
            hidden = torch.arange(L, device="cuda")[None] > torch.arange(L - n, L, device="cuda")[:, None]
            for g in range(h * (H // Hkv), (h + 1) * (H // Hkv)):
                s = (q[at:at + n, g] @ k.t()) / math.sqrt(D)
                out[at:at + n, g] = torch.softmax(s.masked_fill(hidden, -math.inf), 1) @ v
        at += n
    return out


def exact(case, seed):
    return {"norm": _exact_norm, "append": _exact_append, "attention": _exact_attention}[case["kind"]](case, seed)
