"""The operators on a paged key/value cache (include/flame_kv.h) against the oracle in 64 bits, on the same rounded inputs.

Tolerances, per value, are derived from the roundings that the header allows.  Attention, with u the half step of the element type (2^-8 bf16, 2^-11 f16, 2^-24 f32),
W = sum w |v| of the row and Z its largest scale * sum |q||k|:
  a logit is off by (dim + 3) 2^-24 Z at most (fp32 accumulation, scale, product with log2 e) and its difference to the maximum by 4 * 2^-24 Z more; the exponential by 2^-22:
  d = (dim + 7) 2^-24 Z + 2^-22 relative per weight, in numerator and denominator;
  n fp32 additions in both: n 2^-24 each, and as much again for the factors of new maxima;
  the weights' rounding u_w (16-bit types: u) in the numerator, and an absolute 2^-25 for f16 weights below its normal range (their sum is at least 1);
  the output's rounding u |o|, and f16's smallest step.
Rotation: three fp32 roundings of (|a| + |b|) and cosines off by 2^-21, then u of the value."""
import math

import numpy as np
import pytest

from oracle import kv_oracle

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2509_22681_amd import binding
    return binding


def torch_type(dtype):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]


def rand(gen, dtype, *shape):
    import torch
    return torch.randn(*shape, generator=gen, device=DEV).to(torch_type(dtype))


def generator(seed):
    import torch
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def ints(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def host(t):
    return t.detach().double().cpu().numpy()


def offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def attention_bound(dtype, dim, n, want, spread, size):
    u = HALF_STEP[dtype]
    uw = 0.0 if dtype == "f32" else u
    d = (dim + 7) * 2.0 ** -24 * size[..., None] + 2.0 ** -22
    b = u * np.abs(want) + spread * (uw + 2 * d + 4 * n * 2.0 ** -24)
    if dtype == "f16":
        b = b + 2.0 ** -24 + n * 2.0 ** -25 * 6         # (the largest |v| here is below 6)
    return b + 1e-30


def check_attention(got, q, k, v, dtype, scale=None, seen=None, what=""):
    """got [m, Hq, dim] of one sequence against the oracle on q, k, v (host arrays)."""
    dim = q.shape[2]
    want, spread, size = kv_oracle.attend(q, k, v, dim ** -0.5 if scale is None else scale, seen)
    bound = attention_bound(dtype, dim, k.shape[0], want, spread, size)
    off = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (off <= bound).all(), (what, float((off / bound).max()), float(off.max()))


class Cache:
    """Sequences of n tokens in scattered pages of a pool of random values, with a few pages that nobody has."""

    def __init__(self, B, gen, dtype, hq, hkv, dim, lens, page, head_major=False, seed=0, room=0, tokens=0):
        self.cfg, self.page, self.lens = B.make_kv_config(dtype, hq, hkv, dim), page, list(lens)
        used = [-(-(n + room) // page) for n in lens]
        self.n_pages = sum(used) + 3
        shape = (self.n_pages, hkv, page, dim) if head_major else (self.n_pages, page, hkv, dim)
        self.k, self.v = rand(gen, dtype, *shape), rand(gen, dtype, *shape)
        if head_major:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        order = np.random.default_rng(seed).permutation(self.n_pages)
        # (room in the table for `tokens` tokens; entries that nobody reads name no page)
        self.table_host = np.full((len(lens), max(max(used + [1]) + 1, -(-tokens // page))), -7, np.int32)
        for b, first in enumerate(np.cumsum([0] + used[:-1])):
            self.table_host[b, :used[b]] = order[first:first + used[b]]
        self.table = ints(self.table_host)
        self.packed = B.pack_kv_cache(self.cfg, self.k, self.v, self.table)

    def rows(self, b, n):
        page, slot, ok = kv_oracle.page_rows(self.table_host[b], self.page, self.n_pages, n)
        k, v = host(self.k), host(self.v)
        return k[page, slot], v[page, slot]


def spread(n, dtype, hkv):
    """Sequences without tokens behind the others, that make a launch count as a larger one: the forms with four, two and one wavefront per 32 rows (thresholds in
    kv_api.cpp: 160 and 384 or 576 workgroups, fp32 150 and 512 or 640)."""
    return [0] * (0 if n == 0 else (300 if dtype != "f32" else 450) // hkv if n == 1 else 700 // hkv + 1)


# ---------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype,hq,hkv,dim,rot,inter,page,head_major", [
    ("bf16", 8, 2, 64, 64, False, 16, False), ("bf16", 32, 8, 128, 128, True, 24, True), ("f16", 4, 4, 32, 32, False, 1, False), ("f16", 6, 1, 128, 64, False, 7, False),
    ("f32", 8, 8, 64, 32, True, 100, True), ("f32", 3, 3, 128, 128, False, 16, False), ("bf16", 5, 5, 32, 16, True, 64, False), ("f32", 2, 1, 32, 0, False, 5, False)])
def test_append(B, dtype, hq, hkv, dim, rot, inter, page, head_major):
    import torch
    gen = generator(dim + page)
    new, before = [1, 0, 5, 70, 1, 33], [0, 9, 100, 3, 47, 64]
    lens = [a + b for a, b in zip(new, before)]
    c = Cache(B, gen, dtype, hq, hkv, dim, lens, page, head_major)
    n = sum(new)
    rows = rand(gen, dtype, n + 3, hq + 2 * hkv, dim)                   # slices of wider rows, three rows behind the last sequence
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    q_out = torch.full((n + 3, hq, dim), 7.0, device=DEV, dtype=torch_type(dtype))
    f = B.flame_kv_rotation_frequencies(rot) if rot else np.zeros(0)
    want_k, want_v = host(c.k), host(c.v)
    keep_k, keep_v = c.k.clone(), c.v.clone()
    faults = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_append(c.cfg, c.packed, k, v, ints(offsets(new)), ints(lens), q=q, q_out=q_out, rotation=B.make_kv_rotation(f, inter) if rot else None, faults=faults)
    torch.cuda.synchronize()
    assert int(faults[0]) == 0
    position = np.concatenate([np.arange(a, a + m) for a, m in zip(before, new)])
    seq = np.repeat(np.arange(len(new)), new)
    page_of, slot = c.table_host[seq, position // page], position % page

    def near(got, x, what):
        turned = kv_oracle.rotate(x, position, f, inter)
        pair = np.abs(x).max(-1, keepdims=True) * 2
        bound = HALF_STEP[dtype] * np.abs(turned) + (pair * 2.0 ** -21 if rot else 0) + (2.0 ** -25 if dtype == "f16" else 0)
        assert (np.abs(got - turned) <= bound).all(), (what, np.abs(got - turned).max())

    near(host(c.k)[page_of, slot], host(k[:n]), "k")
    near(host(q_out)[:n], host(q[:n]), "q")
    assert np.array_equal(host(c.v)[page_of, slot], host(v[:n]))
    assert bool((q_out[n:] == 7.0).all())                               # rows behind the last sequence
    untouched = np.ones(want_k.shape[:2], bool)
    untouched[page_of, slot] = False
    assert np.array_equal(host(c.k)[untouched], host(keep_k)[untouched]) and np.array_equal(host(c.v)[untouched], host(keep_v)[untouched])
    # in place, and without queries: the same bits
    first, again = c.k.clone(), q.clone()
    B.flame_kv_append(c.cfg, c.packed, k, v, ints(offsets(new)), ints(lens), q=again, q_out=again, rotation=B.make_kv_rotation(f, inter) if rot else None)
    assert torch.equal(again[:n], q_out[:n]) and torch.equal(again[n:], q[n:]) and torch.equal(c.k, first)
    c.k.copy_(keep_k)
    B.flame_kv_append(c.cfg, c.packed, k, v, ints(offsets(new)), ints(lens), rotation=B.make_kv_rotation(f, inter) if rot else None)
    assert torch.equal(c.k, first)


@pytest.mark.parametrize("inter", [False, True])
def test_append_far_positions(B, inter):
    """Angles of positions up to 2^31 - 2^16: the table names the same few pages again and again."""
    import torch
    gen, page, width = generator(1), 65536, 32767
    cfg = B.make_kv_config("f32", 2, 1, 64)
    k_pool, v_pool = torch.zeros(2, page, 1, 64, device=DEV), torch.zeros(2, page, 1, 64, device=DEV)
    cache = B.pack_kv_cache(cfg, k_pool, v_pool, torch.ones(3, width, dtype=torch.int32, device=DEV))
    lens = np.array([page * width, (1 << 30) + 12345, 100003], np.int64)
    q, k = rand(gen, "f32", 6, 2, 64), rand(gen, "f32", 6, 1, 64)
    f = B.flame_kv_rotation_frequencies(64, 10000.0)
    f[1] *= -1
    f[2] = 5.0                                                          # more than a revolution in eight positions, and a turn to the other side
    out = torch.empty_like(q)
    B.flame_kv_append(cfg, cache, k, k, ints([0, 2, 4, 6]), ints(lens), q=q, q_out=out, rotation=B.make_kv_rotation(f, inter))
    position = np.concatenate([[n - 2, n - 1] for n in lens])
    want = kv_oracle.rotate(host(q), position, f, inter)
    # the frequency's own rounding to 64 bits: 2^31 * 2^-64 revolutions, far below the bound
    assert np.abs(host(out) - want).max() <= 2.0 ** -24 * np.abs(want).max() + 2 * np.abs(host(q)).max() * 2.0 ** -21
    turned = kv_oracle.rotate(host(k), position, f, inter)
    assert np.abs(host(k_pool)[1, position % page] - turned).max() <= 2.0 ** -24 * np.abs(turned).max() + 2 * np.abs(host(k)).max() * 2.0 ** -21


def test_append_reports_what_it_cannot_place(B):
    """Bad pages, lengths beyond the table's row and below the new tokens, offsets that decrease: nothing out of range is written, and the rest is."""
    import torch
    gen = generator(2)
    cfg = B.make_kv_config("bf16", 2, 1, 32)
    pool_k, pool_v = torch.zeros(6, 4, 1, 32, device=DEV, dtype=torch.bfloat16), torch.zeros(6, 4, 1, 32, device=DEV, dtype=torch.bfloat16)
    guard_k, guard_v = pool_k[1:5], pool_v[1:5]                         # pages on both sides that no entry may reach
    k = rand(gen, "bf16", 12, 1, 32)

    def append(table, off, lens):
        pool_k.zero_(), pool_v.zero_()
        faults = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.flame_kv_append(cfg, B.pack_kv_cache(cfg, guard_k, guard_v, ints(table)), k, k, ints(off), ints(lens), faults=faults)
        torch.cuda.synchronize()
        assert not pool_k[0].any() and not pool_k[5].any() and not pool_v[0].any() and not pool_v[5].any()
        assert torch.equal(pool_k, pool_v)
        return int(faults[0]), [tuple(x) for x in (pool_k[1:5].abs().sum((2, 3)) > 0).nonzero().tolist()]

    assert append([[0, 1], [2, 3]], [0, 2, 4], [2, 8]) == (0, [(0, 0), (0, 1), (3, 2), (3, 3)])
    assert append([[0, 4], [-1, 3]], [0, 2, 6], [6, 6]) == (1, [(3, 0), (3, 1)])
    assert append([[0, 1], [2, 3]], [0, 3, 5], [2, 9]) == (2, [(0, 0), (0, 1), (3, 3)])
    append([[0, 1], [2, 3]], [0, 4, 2], [4, 2])                         # offsets that decrease
    append([[0, 1], [2, 3]], [-3, 4, 5], [4, 2])
    fault, there = append([[0, 1], [2, 3]], [0, 8, 20], [8, 8])         # twelve rows are there, and eight of the second sequence are not
    assert fault & 4 and all(p in (0, 1, 2, 3) for p, _ in there)


# ---------------------------------------------------------------------------------------------- prompt
HEADS = [("bf16", 8, 2, 64), ("bf16", 4, 4, 128), ("f16", 6, 2, 128), ("f16", 3, 3, 32), ("bf16", 8, 1, 32), ("f16", 4, 4, 64), ("f32", 4, 2, 64), ("f32", 2, 2, 128), ("f32", 3, 1, 32)]
LENGTHS = [[1], [0, 1, 2, 0, 31, 32, 33], [63, 64, 65, 1], [127, 128, 129], [300, 5, 257], [700]]


@pytest.mark.parametrize("dtype,hq,hkv,dim", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("size", [0, 1, 2])
def test_prompt(B, dtype, hq, hkv, dim, lengths, size):
    import torch
    lengths = lengths + spread(size, dtype, hkv)
    gen, n = generator(len(lengths) + dim), sum(lengths)
    rows = rand(gen, dtype, n + 5, hq + 2 * hkv, dim)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    out = torch.full((n + 5, hq, dim), 7.0, device=DEV, dtype=torch_type(dtype))
    off, faults = offsets(lengths), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_prompt(B.make_kv_config(dtype, hq, hkv, dim), q, k, v, ints(off), out, faults=faults)
    torch.cuda.synchronize()
    assert int(faults[0]) == 0 and bool((out[n:] == 7.0).all())
    for b, m in enumerate(lengths):
        s = slice(off[b], off[b + 1])
        if m:
            check_attention(host(out[s]), host(q[s]), host(k[s]), host(v[s]), dtype, what=(lengths[:8], b))


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 64), ("f16", 4, 4, 128), ("f32", 2, 1, 64), ("bf16", 4, 2, 32)])
def test_prompt_with_other_key_lengths(B, dtype, hq, hkv, dim):
    """More keys than queries, fewer (rows that see nothing are zeros), none; a scale; head-major queries and outputs; one fault bit for offsets behind the rows."""
    import torch
    gen, nq, nk = generator(dim), [5, 40, 3, 0, 130, 7], [70, 10, 0, 20, 131, 7]
    q = rand(gen, dtype, hq, sum(nq), dim).transpose(0, 1)
    k, v = rand(gen, dtype, hkv, sum(nk), dim).transpose(0, 1), rand(gen, dtype, sum(nk), hkv, dim)
    out = torch.full((hq, sum(nq), dim), 7.0, device=DEV, dtype=torch_type(dtype)).transpose(0, 1)
    cfg, qo, ko = B.make_kv_config(dtype, hq, hkv, dim, scale=0.3), offsets(nq), offsets(nk)
    B.flame_kv_prompt(cfg, q, k, v, ints(qo), out, k_offsets=ints(ko))
    for b in range(len(nq)):
        sq, sk = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        check_attention(host(out[sq]), host(q[sq]), host(k[sk]), host(v[sk]), dtype, scale=float(np.float32(0.3)), what=b)
        hidden = max(0, nq[b] - nk[b])
        assert not out[sq][:hidden].any()
    faults = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_prompt(cfg, q, k, v, ints(qo), out, k_offsets=ints(ko + 1), faults=faults)
    assert int(faults[0]) == 4


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("size", [0, 1, 2])
def test_prompt_rows_do_not_feel_what_they_do_not_see(B, dtype, dim, size):
    """Later tokens of the same sequence and other sequences hold infinities and NaN: earlier rows keep their bits, rows that see a NaN value have it, and one that sees an infinite value is infinite there."""
    import torch
    gen = generator(3)
    cfg, off = B.make_kv_config(dtype, 4, 2, dim), offsets([200, 90] + spread(size, dtype, 2))
    q, k, v = rand(gen, dtype, 290, 4, dim), rand(gen, dtype, 290, 2, dim), rand(gen, dtype, 290, 2, dim)
    clean, dirty = torch.empty_like(q), torch.empty_like(q)
    B.flame_kv_prompt(cfg, q, k, v, ints(off), clean)
    for at in (0, 77, 130, 199):
        for value, where in ((math.nan, "v"), (math.inf, "v"), (-math.inf, "v"), (math.nan, "k"), (math.inf, "k")):
            k2, v2 = k.clone(), v.clone()
            (v2 if where == "v" else k2)[at, 1, 3] = value
            B.flame_kv_prompt(cfg, q, k2, v2, ints(off), dirty)
            assert torch.equal(dirty[:at], clean[:at]) and torch.equal(dirty[200:], clean[200:]), (at, value, where)
            assert torch.equal(dirty[:, :2], clean[:, :2])              # query heads of the other key head
            if where == "v":
                changed = dirty[at:200, 2:, 3].float()
                assert bool((changed.isnan() if math.isnan(value) else changed == value).all()), (at, value)
                others = [i for i in range(dim) if i != 3]
                assert torch.equal(dirty[:, :, others], clean[:, :, others])
            elif math.isnan(value):
                assert bool(dirty[at:200, 2:].isnan().all())


def test_prompt_of_large_logits(B):
    """Logits of hundreds, of both signs: the maximum is taken out before the exponential, wherever in the row it comes."""
    import torch
    gen = generator(4)
    for dtype, dim in (("bf16", 64), ("f16", 128), ("f32", 32)):
        q, k, v = 30 * rand(gen, dtype, 400, 2, dim), 3 * rand(gen, dtype, 400, 2, dim), rand(gen, dtype, 400, 2, dim)
        out = torch.empty_like(q)
        B.flame_kv_prompt(B.make_kv_config(dtype, 2, 2, dim), q, k, v, ints([0, 400]), out)
        check_attention(host(out), host(q), host(k), host(v), dtype, what=dtype)


# ---------------------------------------------------------------------------------------------- extend and decode
def workspace_for(B, cfg, n_seqs, n_tokens=None):
    import torch
    return torch.full((B.flame_kv_workspace_bytes(cfg, n_seqs, n_tokens),), 0xff, dtype=torch.uint8, device=DEV)     # it holds nothing between calls: NaN


@pytest.mark.parametrize("dtype,hq,hkv,dim", HEADS + [("bf16", 32, 1, 64), ("f16", 40, 2, 32), ("f32", 20, 1, 64)])
@pytest.mark.parametrize("page,head_major", [(16, False), (24, True), (1, False), (300, True)])
def test_decode(B, dtype, hq, hkv, dim, page, head_major):
    import torch
    gen, lens = generator(page), [1, 0, 31, 32, 33, 700, 64, 129]
    c = Cache(B, gen, dtype, hq, hkv, dim, lens, page, head_major)
    q = rand(gen, dtype, len(lens), hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_decode(c.cfg, c.packed, q, ints(lens), out, workspace_for(B, c.cfg, len(lens)), faults=faults)
    assert int(faults[0]) == 0
    for b, n in enumerate(lens):
        check_attention(host(out[b:b + 1]), host(q[b:b + 1]), *c.rows(b, n), dtype, what=(b, n))


@pytest.mark.parametrize("dtype,factor", [("f32", 2.0 ** 106), ("bf16", 2.0 ** 106), ("f16", 8192.0)])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_values_near_the_end_of_the_range(B, dtype, factor, dim):
    """Values below 2^(120 - 11) with up to 2000 keys, and fp16 ones up to its largest, on row tiles, in parts and split: finite outputs, as exact as others."""
    import torch
    gen = generator(dim)
    lens, new = [2000, 90, 700], [70, 90, 1]
    c = Cache(B, gen, dtype, 4, 2, dim, lens, 16, tokens=4096)
    c.v.clamp_(-4, 4).mul_(factor)
    off, n = offsets(new), sum(new)
    q = 3 * rand(gen, dtype, n, 4, dim)                       # (the largest logit moves)
    out = torch.empty_like(q)
    B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, 3, n))
    last = q[torch.tensor(off[1:] - 1, device=DEV).long()].contiguous()
    single = torch.empty_like(last)
    B.flame_kv_decode(c.cfg, c.packed, last, ints(lens), single, workspace_for(B, c.cfg, 3))
    small = torch.empty_like(q)
    keys, values = c.rows(1, 90)
    B.flame_kv_prompt(c.cfg, q[70:160], torch.tensor(keys, dtype=q.dtype, device=DEV), torch.tensor(values, dtype=q.dtype, device=DEV), ints([0, 90]), small[70:160])
    for b, n_b in enumerate(lens):
        keys, values = c.rows(b, n_b)
        s = slice(off[b], off[b + 1])
        # (scaled back exactly: powers of two, and no result is subnormal but in fp16, whose bound has an absolute part of the scaled values' size)
        check_attention(host(out[s]) / factor, host(q[s]), keys, values / factor, dtype, what=("extend", b))
        check_attention(host(single[b:b + 1]) / factor, host(last[b:b + 1]), keys, values / factor, dtype, what=("decode", b))
        if b == 1:
            check_attention(host(small[s]) / factor, host(q[s]), keys, values / factor, dtype, what="prompt")


@pytest.mark.parametrize("dtype,hq,hkv,dim,n_seqs", [("bf16", 8, 2, 64, 65), ("f16", 4, 1, 128, 200), ("bf16", 8, 2, 32, 4200), ("f32", 4, 4, 32, 5000), ("f16", 32, 2, 64, 700)])
def test_decode_of_many_sequences(B, dtype, hq, hkv, dim, n_seqs):
    """More sequences than lanes, and more rows of heads than workgroups of the join; some of them long, so that their keys are cut."""
    import torch
    gen, rng = generator(n_seqs), np.random.default_rng(n_seqs)
    lens = rng.integers(0, 30, n_seqs)
    long = [0, 1, n_seqs // 2, n_seqs - 1]
    lens[long] = [3000, 700, 1999, 4001]
    c = Cache(B, gen, dtype, hq, hkv, dim, lens.tolist(), 16)
    q = rand(gen, dtype, n_seqs, hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_decode(c.cfg, c.packed, q, ints(lens), out, workspace_for(B, c.cfg, n_seqs), faults=faults)
    assert int(faults[0]) == 0 and not bool((out == 7.0).all(-1).any())
    pool_k, pool_v, got, want = host(c.k), host(c.v), host(out), host(q)
    for b in long + rng.integers(0, n_seqs, 60).tolist():
        page, slot, _ = kv_oracle.page_rows(c.table_host[b], c.page, c.n_pages, int(lens[b]))
        check_attention(got[b:b + 1], want[b:b + 1], pool_k[page, slot], pool_v[page, slot], dtype, what=(b, int(lens[b])))


@pytest.mark.parametrize("dtype,hq,hkv,dim,n_seqs", [("bf16", 4, 1, 64, 70), ("f16", 2, 2, 128, 300), ("f32", 4, 2, 32, 90), ("bf16", 2, 1, 32, 4500)])
@pytest.mark.parametrize("paged", [False, True])
def test_many_ragged_sequences(B, dtype, hq, hkv, dim, n_seqs, paged):
    """More sequences than lanes, of zero to 300 rows each, on row tiles: packed, and over caches."""
    import torch
    gen, rng = generator(n_seqs), np.random.default_rng(n_seqs)
    new = rng.integers(0, 20, n_seqs)
    new[rng.integers(0, n_seqs, n_seqs // 4)] = 0
    new[[0, n_seqs // 3, n_seqs - 1]] = [300, 129, 40]
    lens = new + (rng.integers(0, 70, n_seqs) if paged else 0)
    off, n = offsets(new), int(new.sum())
    q = rand(gen, dtype, n + 5, hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    if paged:
        c = Cache(B, gen, dtype, hq, hkv, dim, lens.tolist(), 16)
        B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, n_seqs, n + 5), faults=faults)
        pool_k, pool_v = host(c.k), host(c.v)
    else:
        k, v = rand(gen, dtype, n, hkv, dim), rand(gen, dtype, n, hkv, dim)
        B.flame_kv_prompt(B.make_kv_config(dtype, hq, hkv, dim), q, k, v, ints(off), out, faults=faults)
        pool_k, pool_v = host(k), host(v)
    assert int(faults[0]) == 0 and bool((out[n:] == 7.0).all()) and not bool((out[:n] == 7.0).all(-1).any())
    got, want = host(out), host(q)
    for b in [0, n_seqs // 3, n_seqs - 1] + rng.integers(0, n_seqs, 40).tolist():
        s = slice(off[b], off[b + 1])
        if paged:
            page, slot, _ = kv_oracle.page_rows(c.table_host[b], c.page, c.n_pages, int(lens[b]))
            check_attention(got[s], want[s], pool_k[page, slot], pool_v[page, slot], dtype, what=(int(b), int(lens[b])))
        else:
            check_attention(got[s], want[s], pool_k[s], pool_v[s], dtype, what=int(b))


@pytest.mark.parametrize("dtype,hq,hkv,dim,n_seqs", [("bf16", 4, 2, 64, 130), ("f32", 4, 1, 32, 300), ("f16", 2, 2, 128, 5000)])
def test_extend_of_many_sequences(B, dtype, hq, hkv, dim, n_seqs):
    """Few new tokens in all, of more sequences than lanes (most of which have none), split over the keys; with rows behind the last sequence."""
    import torch
    gen, rng = generator(n_seqs), np.random.default_rng(n_seqs)
    new, lens = np.zeros(n_seqs, np.int64), rng.integers(0, 30, n_seqs)
    some = np.unique(rng.integers(0, n_seqs, 60))
    new[some] = rng.integers(1, 4, some.size)
    new[some[3]] = 70                                         # (several blocks of rows that read the same keys)
    lens[some] += rng.choice([0, 5, 900, 1500], some.size)
    lens[some[3]] = 1300
    c = Cache(B, gen, dtype, hq, hkv, dim, lens.tolist(), 16, tokens=2000)
    off, n = offsets(new), int(new.sum())
    q = rand(gen, dtype, n + 3, hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, n_seqs, n + 3), faults=faults)
    assert int(faults[0]) == 0 and bool((out[n:] == 7.0).all())
    pool_k, pool_v, got, want = host(c.k), host(c.v), host(out), host(q)
    for b in some:
        page, slot, _ = kv_oracle.page_rows(c.table_host[b], c.page, c.n_pages, int(lens[b]))
        s = slice(off[b], off[b + 1])
        check_attention(got[s], want[s], pool_k[page, slot], pool_v[page, slot], dtype, what=(int(b), int(lens[b])))


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 64), ("f16", 4, 4, 128), ("f32", 4, 2, 64), ("bf16", 16, 2, 128), ("f16", 6, 3, 32)])
@pytest.mark.parametrize("size", [0, 1, 2])
@pytest.mark.parametrize("tokens", [0, 2000])
@pytest.mark.parametrize("new,lens,page", [([1, 3, 0, 7, 2], [1, 400, 20, 65, 2], 16), ([40, 200, 1], [40, 333, 600], 24), ([5, 9], [3, 0], 8), ([130], [1000], 64)], ids=str)
def test_extend(B, dtype, hq, hkv, dim, new, lens, page, size, tokens):
    import torch
    new, lens = new + spread(size, dtype, hkv), lens + spread(size, dtype, hkv)
    gen = generator(len(new))
    c = Cache(B, gen, dtype, hq, hkv, dim, lens, page, tokens=tokens)        # (a table with more room: few rows take the split kernel)
    off, n = offsets(new), sum(new)
    q = rand(gen, dtype, n + 4, hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, len(lens), n + 4), faults=faults)
    assert int(faults[0]) == 0 and bool((out[n:] == 7.0).all())
    for b, n_b in enumerate(lens):
        s = slice(off[b], off[b + 1])
        if new[b]:
            check_attention(host(out[s]), host(q[s]), *c.rows(b, n_b), dtype, what=(b, n_b))


@pytest.mark.parametrize("dtype,heads,dim", [("bf16", 128, 128), ("bf16", 160, 128), ("f16", 128, 64), ("f16", 160, 64), ("bf16", 150, 32), ("bf16", 200, 32), ("f32", 200, 64), ("f32", 256, 64),
                                             ("f32", 150, 128), ("f32", 256, 128), ("f32", 160, 32), ("f32", 256, 32)])
def test_extend_of_many_heads(B, dtype, heads, dim):
    """Launches of two and one wavefront per 32 rows over pages (300 new tokens: three workgroups a head)."""
    import torch
    gen = generator(heads)
    c = Cache(B, gen, dtype, heads, heads, dim, [340], 24)
    q = rand(gen, dtype, 300, heads, dim)
    out = torch.full_like(q, 7.0)
    B.flame_kv_extend(c.cfg, c.packed, q, ints([0, 300]), ints([340]), out, workspace_for(B, c.cfg, 1, 300))
    keys, values = c.rows(0, 340)
    for h in (0, 1, heads // 2, heads - 1):
        check_attention(host(out[:, h:h + 1]), host(q[:, h:h + 1]), keys[:, h:h + 1], values[:, h:h + 1], dtype, what=h)
    assert bool(out.isfinite().all()) and not bool((out == 7.0).all(-1).any())


@pytest.mark.parametrize("dtype,hq,hkv,dim,new,lens", [
    ("bf16", 64, 64, 64, [20], [1500]), ("f16", 32, 32, 128, [50], [1200]), ("bf16", 8, 2, 64, [200, 3], [900, 2000]), ("f16", 16, 2, 128, [70, 1, 30], [1100, 2500, 31]),
    ("bf16", 32, 1, 32, [129], [1700]), ("f32", 64, 16, 64, [140], [1300]), ("f32", 32, 16, 128, [300], [1000]), ("f32", 256, 256, 32, [40], [1030]), ("f32", 128, 128, 64, [65, 2], [700, 640])])
def test_extend_in_parts(B, dtype, hq, hkv, dim, new, lens):
    """Tables with room for 8192 tokens: the keys of a row tile are cut into parts and joined; with a page that the table does not name, and with a NaN in the newest token."""
    import torch
    gen = generator(hq)
    c = Cache(B, gen, dtype, hq, hkv, dim, lens, 16, tokens=8192)
    table = c.table_host.copy()
    table[0, 5] = -1
    packed = B.pack_kv_cache(c.cfg, c.k, c.v, ints(table))
    off, n = offsets(new), sum(new)
    q = rand(gen, dtype, n, hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = workspace_for(B, c.cfg, len(lens), n)
    B.flame_kv_extend(c.cfg, packed, q, ints(off), ints(lens), out, ws, faults=faults)
    assert int(faults[0]) == 1 and bool(out.isfinite().all())
    group = hq // hkv
    for b, n_b in enumerate(lens):
        keys, values = c.rows(b, n_b)
        s = slice(off[b], off[b + 1])
        for h in sorted({0, 1, hq // 2, hq - 1}):
            kv = slice(h // group, h // group + 1)
            seen = np.arange(n_b) // 16 != 5 if b == 0 else None
            check_attention(host(out[s, h:h + 1]), host(q[s, h:h + 1]), keys[:, kv], values[:, kv], dtype, seen=seen, what=(b, h))
    page, slot, _ = kv_oracle.page_rows(c.table_host[0], 16, c.n_pages, lens[0])
    c.v[int(page[-1]), int(slot[-1]), hkv - 1, 2] = math.nan
    dirty = torch.full_like(q, 7.0)
    B.flame_kv_extend(c.cfg, packed, q, ints(off), ints(lens), dirty, ws)
    last = int(off[1]) - 1
    assert bool(dirty[last, hq - group:, 2].isnan().all())
    dirty[last, hq - group:, 2] = out[last, hq - group:, 2]
    assert torch.equal(dirty, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_pages_and_lengths(B, dtype):
    """Keys in a page that the table does not name are not seen; lengths are cut to what the table has room for; both are reported."""
    import torch
    gen, lens = generator(5), [150, 90]
    c = Cache(B, gen, dtype, 4, 2, 64, lens, 16)
    q = rand(gen, dtype, 6, 4, 64)
    for entry in (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = c.table_host.copy()
        table[0, 3] = entry
        packed = B.pack_kv_cache(c.cfg, c.k, c.v, ints(table))
        seen = np.arange(150) // 16 != 3
        keys, values = c.rows(0, 150)
        for new in (1, 5):
            rows = q[:2] if new == 1 else q
            out, faults = torch.empty_like(rows), torch.zeros(1, dtype=torch.int32, device=DEV)
            if new == 1:
                B.flame_kv_decode(c.cfg, packed, rows, ints(lens), out, workspace_for(B, c.cfg, 2), faults=faults)
            else:
                B.flame_kv_extend(c.cfg, packed, rows, ints([0, 5, 6]), ints(lens), out, workspace_for(B, c.cfg, 2, 6), faults=faults)
            assert int(faults[0]) == 1
            check_attention(host(out[:new]), host(rows[:new]), keys, values, dtype, seen=seen, what=(entry, new))
            check_attention(host(out[new:]), host(rows[new:]), *c.rows(1, 90), dtype, what=(entry, new))
    # every page bad: nothing is seen, zeros
    packed = B.pack_kv_cache(c.cfg, c.k, c.v, torch.full_like(c.table, -1))
    out = torch.full_like(q[:2], 7.0)
    B.flame_kv_decode(c.cfg, packed, q[:2], ints(lens), out, workspace_for(B, c.cfg, 2))
    assert not out.any()
    # lengths: below 0 is 0, beyond the row's room is the room
    width = c.table_host.shape[1]
    table = np.resize(c.table_host[0, :9], (2, width)).astype(np.int32)
    packed = B.pack_kv_cache(c.cfg, c.k, c.v, ints(table))
    faults = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kv_decode(c.cfg, packed, q[:2], ints([-5, 2 ** 31 - 1]), out, workspace_for(B, c.cfg, 2), faults=faults)
    assert int(faults[0]) == 2 and not out[0].any()
    page, slot, _ = kv_oracle.page_rows(table[1], 16, c.n_pages, 16 * width)
    check_attention(host(out[1:]), host(q[1:2]), host(c.k)[page, slot], host(c.v)[page, slot], dtype, what="room")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_unused_slots_and_unseen_tokens_do_not_count(B, dtype):
    """Slots behind the last token, pages of others and tokens that a row does not see hold NaN: no output changes a bit."""
    import torch
    gen, lens = generator(6), [100, 37, 1]
    c = Cache(B, gen, dtype, 4, 2, 128, lens, 16)
    q, ws = rand(gen, dtype, 9, 4, 128), workspace_for(B, c.cfg, 3, 9)
    clean, dirty = torch.empty_like(q), torch.empty_like(q)
    off = ints([0, 4, 8, 9])
    B.flame_kv_extend(c.cfg, c.packed, q, off, ints(lens), clean, ws)
    single = torch.empty_like(q[:3])
    B.flame_kv_decode(c.cfg, c.packed, q[:3], ints(lens), single, ws)
    owned = np.zeros((c.n_pages, 16), bool)
    for b, n in enumerate(lens):
        page, slot, _ = kv_oracle.page_rows(c.table_host[b], 16, c.n_pages, n)
        owned[page, slot] = True
    for pool in (c.k, c.v):
        pool[torch.from_numpy(~owned).to(DEV)] = math.nan
    B.flame_kv_extend(c.cfg, c.packed, q, off, ints(lens), dirty, ws)
    again = torch.empty_like(single)
    B.flame_kv_decode(c.cfg, c.packed, q[:3], ints(lens), again, ws)
    assert torch.equal(clean, dirty) and torch.equal(single, again)
    # the newest token of sequence 0: of its four rows only the last sees it
    page, slot, _ = kv_oracle.page_rows(c.table_host[0], 16, c.n_pages, 100)
    for pool in (c.v, c.k):
        pool[int(page[99]), int(slot[99])] = math.nan
        B.flame_kv_extend(c.cfg, c.packed, q, off, ints(lens), dirty, ws)
        assert torch.equal(clean[:3], dirty[:3]) and torch.equal(clean[4:], dirty[4:]) and bool(dirty[3].isnan().all())


def test_pools_beyond_32_bits(B):
    """Pools of 5 GiB: a sequence in the last pages of them."""
    import torch
    gen, pages = generator(7), 81920
    cfg = B.make_kv_config("bf16", 8, 4, 128)
    k, v = (torch.empty(pages, 64, 4, 128, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    names = [81919, 40000, 81900, 2, 70000]
    for pool in (k, v):
        for p in names:
            pool[p] = rand(gen, "bf16", 64, 4, 128)
    cache, n = B.pack_kv_cache(cfg, k, v, ints([names])), 300
    new, q = rand(gen, "bf16", 2, 4, 128), rand(gen, "bf16", 2, 8, 128)
    B.flame_kv_append(cfg, cache, new, new, ints([0, 2]), ints([n]))
    keys = torch.cat([k[p] for p in names])[:n]
    values = torch.cat([v[p] for p in names])[:n]
    assert torch.equal(keys[n - 2:], new) and torch.equal(values[n - 2:], new)
    out = torch.empty_like(q)
    B.flame_kv_extend(cfg, cache, q, ints([0, 2]), ints([n]), out, workspace_for(B, cfg, 1, 2))
    check_attention(host(out), host(q), host(keys), host(values), "bf16")
    B.flame_kv_decode(cfg, cache, q[1:], ints([n]), out[1:], workspace_for(B, cfg, 1))
    check_attention(host(out[1:]), host(q[1:]), host(keys), host(values), "bf16")


# ---------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 64), ("f16", 8, 8, 128), ("f32", 4, 2, 32)])
def test_a_history_that_grows(B, dtype, hq, hkv, dim):
    """As a server runs them: prompts go into the cache and are attended to from there, then in pieces, then token by token; every row is that of attention within the whole sequence."""
    import torch
    gen, steps = generator(8), [[70, 0, 33], [1, 50, 1], [1, 1, 1], [0, 1, 130], [1, 1, 1]]
    total = np.sum(steps, 0)
    c = Cache(B, gen, dtype, hq, hkv, dim, [int(n) for n in total], 16)
    rot = B.make_kv_rotation(B.flame_kv_rotation_frequencies(dim))
    q, k, v = ([rand(gen, dtype, int(n), h, dim) for n in total] for h in (hq, hkv, hkv))
    got = [[] for _ in total]
    turned_q = [[] for _ in total]
    done = np.zeros(3, int)
    for new in steps:
        done = done + new
        rows_q = torch.cat([q[b][done[b] - new[b]:done[b]] for b in range(3)])
        rows_k = torch.cat([k[b][done[b] - new[b]:done[b]] for b in range(3)])
        rows_v = torch.cat([v[b][done[b] - new[b]:done[b]] for b in range(3)])
        off, lens, now_q, out = ints(offsets(new)), ints(done), torch.empty_like(rows_q), torch.empty_like(rows_q)
        B.flame_kv_append(c.cfg, c.packed, rows_k, rows_v, off, lens, q=rows_q, q_out=now_q, rotation=rot)
        if new == [1, 1, 1]:
            B.flame_kv_decode(c.cfg, c.packed, now_q, lens, out, workspace_for(B, c.cfg, 3))
        else:
            B.flame_kv_extend(c.cfg, c.packed, now_q, off, lens, out, workspace_for(B, c.cfg, 3, len(now_q)))
        at = 0
        for b, m in enumerate(new):
            got[b].append(out[at:at + m])
            turned_q[b].append(now_q[at:at + m])
            at += m
    for b, n in enumerate(total):
        keys, values = c.rows(b, int(n))
        assert np.array_equal(values, host(v[b]))
        check_attention(host(torch.cat(got[b])), host(torch.cat(turned_q[b])), keys, values, dtype, what=b)
    # and the prompt operator on the same rows, in no cache
    rows = [torch.cat(x) for x in turned_q]
    keys = [torch.from_numpy(c.rows(b, int(n))[0]).to(DEV).to(torch_type(dtype)) for b, n in enumerate(total)]
    out = torch.empty_like(torch.cat(rows))
    B.flame_kv_prompt(c.cfg, torch.cat(rows), torch.cat(keys), torch.cat(v), ints(offsets(total)), out)
    off = offsets(total)
    for b, n in enumerate(total):
        s = slice(off[b], off[b + 1])
        check_attention(host(out[s]), host(rows[b]), host(keys[b]), host(v[b]), dtype, what=("prompt", b))


def test_graphs_follow_the_device_arrays(B):
    """A decoding step (append, attend) captured once and replayed while the lengths grow; two graphs share a workspace; eager work in between."""
    import torch
    gen, lens0, steps = generator(9), [5, 130, 0, 1000], 6
    c = Cache(B, gen, "bf16", 8, 2, 64, lens0, 16, room=steps)
    twin = Cache(B, generator(9), "bf16", 8, 2, 64, lens0, 16, room=steps)
    rot = B.make_kv_rotation(B.flame_kv_rotation_frequencies(64))
    lens, off = ints(lens0), ints([0, 1, 2, 3, 4])
    q, k, v = (torch.zeros(4, h, 64, device=DEV, dtype=torch.bfloat16) for h in (8, 2, 2))
    out, turned, ext = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    ws = workspace_for(B, c.cfg, 4, 4)
    ws = torch.full((max(ws.numel(), B.flame_kv_workspace_bytes(c.cfg, 4)),), 0xff, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    graphs = []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for op in ("decode", "extend"):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                if op == "decode":
                    B.flame_kv_append(c.cfg, c.packed, k, v, off, lens, q=q, q_out=turned, rotation=rot)
                    B.flame_kv_decode(c.cfg, c.packed, turned, lens, out, ws)
                else:
                    B.flame_kv_extend(c.cfg, c.packed, turned, off, lens, ext, ws)
            graphs.append(g)
    torch.cuda.synchronize()
    for step in range(steps):
        lens.copy_(ints([n + step + 1 for n in lens0]))
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        # eager, on a cache of its own
        out2, turned2, ext2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
        ws2 = torch.full_like(ws, 0xff)
        B.flame_kv_append(twin.cfg, twin.packed, k, v, off, lens, q=q, q_out=turned2, rotation=rot)
        B.flame_kv_decode(twin.cfg, twin.packed, turned2, lens, out2, ws2)
        B.flame_kv_extend(twin.cfg, twin.packed, turned2, off, lens, ext2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(turned, turned2) and torch.equal(ext, ext2) and torch.equal(c.k, twin.k), step
        for b in range(4):
            check_attention(host(out[b:b + 1]), host(turned[b:b + 1]), *c.rows(b, lens0[b] + step + 1), "bf16", what=(step, b))


def test_other_streams_and_a_padded_batch(B):
    """Work on a stream of its own; sequences of a padded batch that have no rows (length 0, offsets that stand still) and offsets that end before the rows do."""
    import torch
    gen, lens = generator(10), [300, 0, 45, 0]
    c = Cache(B, gen, "f16", 4, 2, 64, lens, 32)
    q = rand(gen, "f16", 12, 4, 64)
    off = ints([0, 3, 3, 5, 5])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = torch.full_like(q, 7.0)
        ws = workspace_for(B, c.cfg, 4, 12)
    lens_dev = ints(lens)
    torch.cuda.synchronize()
    B.flame_kv_extend(c.cfg, c.packed, q, off, lens_dev, out, ws, stream=side)
    side.synchronize()
    assert bool((out[5:] == 7.0).all())
    check_attention(host(out[:3]), host(q[:3]), *c.rows(0, 300), "f16")
    check_attention(host(out[3:5]), host(q[3:5]), *c.rows(2, 45), "f16")


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 64), ("f16", 4, 4, 128), ("f32", 4, 1, 32), ("f32", 3, 3, 128)])
def test_strided_rows(B, dtype, hq, hkv, dim):
    """Queries, keys and values as slices of one projection's rows, outputs as a slice of wider rows and head by head: what lies beside them stays."""
    import torch
    gen, new, lens = generator(14), [40, 1, 9], [1500, 60, 9]
    off, n = offsets(new), sum(new)
    rows = rand(gen, dtype, n, hq + 2 * hkv + 1, dim)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:hq + 2 * hkv]
    for head_major in (False, True):
        for room in (0, 4096):                                          # row tiles whole, in parts or split
            c = Cache(B, gen, dtype, hq, hkv, dim, lens, 16, head_major, tokens=room)
            for kind in ("prompt", "extend", "decode"):
                m = 3 if kind == "decode" else n
                wide = torch.full((hq + 2, m, dim) if head_major else (m, hq + 2, dim), 7.0, dtype=q.dtype, device=DEV)
                out = (wide.transpose(0, 1) if head_major else wide)[:, 1:hq + 1]
                if kind == "prompt":
                    B.flame_kv_prompt(c.cfg, q, k, v, ints(off), out)
                elif kind == "extend":
                    B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, 3, n))
                else:
                    B.flame_kv_decode(c.cfg, c.packed, q[:3], ints(lens), out, workspace_for(B, c.cfg, 3))
                beside = wide.transpose(0, 1) if head_major else wide
                assert bool((beside[:, 0] == 7.0).all()) and bool((beside[:, -1] == 7.0).all())
                for b, n_b in enumerate(lens):
                    rows_b = slice(b, b + 1) if kind == "decode" else slice(off[b], off[b + 1])
                    keys, values = (host(k[rows_b]), host(v[rows_b])) if kind == "prompt" else c.rows(b, n_b)
                    check_attention(host(out[rows_b]), host(q[rows_b]), keys, values, dtype, what=(kind, head_major, room, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("empty", [0, 100])
@pytest.mark.parametrize("off", [[0, 40, 20, 60], [-5, 40, 50, 60], [0, 30, 90, 90], [0, 30, 2 ** 31 - 1, 60], [70, 80, 90, 2 ** 31 - 1], [0, -2 ** 31, 2 ** 31 - 1, 60]], ids=str)
def test_offsets_that_are_none(B, dtype, empty, off):
    """Offsets that decrease, begin below 0 or end behind the rows are reported, and nothing is written outside the 60 rows (on row tiles, in parts, split; of up to 64
    sequences and of more).  A first sequence that is one has its rows."""
    import torch
    gen, lens = generator(15), [900, 60, 90] + [0] * empty
    off = off + [off[-1]] * empty
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    for room, hq in ((0, 4), (4096, 64), (4096, 2)):
        c = Cache(B, gen, dtype, hq, hq, 64, lens, 16, tokens=room)
        q, k = rand(gen, dtype, 60, hq, 64), rand(gen, dtype, 60, hq, 64)
        for kind in ("prompt", "extend"):
            buffer = torch.full((180, hq, 64), 7.0, dtype=q.dtype, device=DEV)
            out = buffer[60:120]
            fault.zero_()
            if kind == "prompt":
                B.flame_kv_prompt(c.cfg, q, k, k, ints(off), out, faults=fault)
            else:
                B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, len(lens), 60), faults=fault)
            assert int(fault[0]) == 4, (kind, room)
            assert bool((buffer[:60] == 7.0).all()) and bool((buffer[120:] == 7.0).all())
            if off[:2] == [0, 30]:
                keys, values = (host(k[:30]), host(k[:30])) if kind == "prompt" else c.rows(0, 900)
                check_attention(host(out[:30, :1]), host(q[:30, :1]), keys[:, :1], values[:, :1], dtype, what=(kind, room, hq))


def test_two_calls_at_once(B):
    """Calls on two streams that share a cache, each with a workspace of its own."""
    import torch
    gen, lens = generator(16), [5000, 3000]
    c = Cache(B, gen, "bf16", 8, 2, 64, lens, 16)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    q = [rand(gen, "bf16", 2, 8, 64) for _ in streams]
    out, ws, n = [torch.empty_like(x) for x in q], [workspace_for(B, c.cfg, 2) for _ in streams], ints(lens)
    torch.cuda.synchronize()
    for _ in range(20):
        for i, stream in enumerate(streams):
            B.flame_kv_decode(c.cfg, c.packed, q[i], n, out[i], ws[i], stream=stream)
    torch.cuda.synchronize()
    for i in (0, 1):
        for b, n_b in enumerate(lens):
            check_attention(host(out[i][b:b + 1]), host(q[i][b:b + 1]), *c.rows(b, n_b), "bf16", what=(i, b))


def test_the_same_call_gives_the_same_bits(B):
    """The same call twice gives the same bits, at sizes where the work is split and joined."""
    import torch
    gen, lens = generator(11), [5000, 17, 3000]
    c = Cache(B, gen, "bf16", 16, 2, 128, lens, 16)
    q = rand(gen, "bf16", 3, 16, 128)
    outs = []
    for _ in range(3):
        out = torch.empty_like(q)
        B.flame_kv_decode(c.cfg, c.packed, q, ints(lens), out, workspace_for(B, c.cfg, 3))
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    for b, n in enumerate(lens):
        check_attention(host(outs[0][b:b + 1]), host(q[b:b + 1]), *c.rows(b, n), "bf16", what=b)


def test_refusals_on_the_device(B):
    import torch
    cfg = B.make_kv_config("bf16", 8, 2, 64)
    pool = torch.zeros(4, 16, 2, 64, device=DEV, dtype=torch.bfloat16)
    q, kv, i = torch.zeros(3, 8, 64, device=DEV, dtype=torch.bfloat16), torch.zeros(3, 2, 64, device=DEV, dtype=torch.bfloat16), ints([0, 1, 2, 3])
    table = ints(np.zeros((3, 2)))
    cache = B.pack_kv_cache(cfg, pool, pool.clone(), table)
    lens = ints([1, 1, 1])
    wide = torch.zeros(3, 8, 68, device=DEV, dtype=torch.bfloat16)[..., :64]
    for bad, kind in ((lambda: B.flame_kv_append(cfg, cache, kv, kv[:2], i, lens), ValueError), (lambda: B.flame_kv_append(cfg, cache, kv, kv, i, lens, q=q), ValueError),
                      (lambda: B.flame_kv_append(cfg, cache, kv, kv, i, lens, q_out=q), ValueError), (lambda: B.flame_kv_append(cfg, cache, kv, kv, i, lens, q=q, q_out=q[:2]), ValueError),
                      (lambda: B.flame_kv_prompt(cfg, q, kv, kv[:2], i, q), ValueError), (lambda: B.flame_kv_prompt(cfg, q, kv, kv, i, q[:2]), ValueError),
                      (lambda: B.flame_kv_extend(cfg, cache, q, i, lens, q[:2]), ValueError), (lambda: B.flame_kv_decode(cfg, cache, q, lens, q[:2]), ValueError),
                      (lambda: B.flame_kv_append(cfg, cache, kv.cpu(), kv, i, lens), ValueError), (lambda: B.flame_kv_append(cfg, cache, kv, kv, i.cpu(), lens), ValueError),
                      (lambda: B.flame_kv_append(cfg, cache, kv, kv, i[:3], lens), ValueError), (lambda: B.flame_kv_prompt(cfg, q, kv, kv, i, q[:1].expand(3, 8, 64)), ValueError),
                      (lambda: B.flame_kv_prompt(cfg, wide, kv, kv, i, q), B.FlameGRError), (lambda: B.flame_kv_decode(B.make_kv_config("f16", 8, 2, 64), cache, q.half(), lens, q.half()), ValueError),
                      (lambda: B.flame_kv_decode(cfg, cache, torch.zeros(4, 8, 64, device=DEV, dtype=torch.bfloat16), ints([1] * 4), torch.zeros(4, 8, 64, device=DEV, dtype=torch.bfloat16)), ValueError),
                      (lambda: B.pack_kv_cache(cfg, pool, pool.transpose(1, 2).contiguous().transpose(1, 2), table), ValueError),
                      (lambda: B.pack_kv_cache(cfg, pool[:1].expand(4, 16, 2, 64), pool[:1].expand(4, 16, 2, 64), table), ValueError),
                      (lambda: B.flame_kv_decode(cfg, cache, q, lens, torch.empty_like(q), torch.zeros(8, device="cpu")), ValueError)):
        with pytest.raises(kind):
            bad()
    # heads and rows of one: whatever stride torch gives such a dimension is not looked at
    one = B.make_kv_config("bf16", 1, 1, 64)
    x = torch.as_strided(rand(generator(1), "bf16", 400), (5, 1, 64), (64, 3, 1))
    out = torch.empty(5, 1, 64, device=DEV, dtype=torch.bfloat16)
    B.flame_kv_prompt(one, x, x, x, ints([0, 5]), out)
    check_attention(host(out), host(x), host(x), host(x), "bf16")


def test_one_workspace_for_every_smaller_batch(B):
    """As a server has it: asked for once, for its largest batch, and used by every call."""
    import torch
    gen, lens = generator(17), [1500, 60, 900]
    c = Cache(B, gen, "bf16", 8, 2, 64, lens, 16, tokens=8192)
    ws = workspace_for(B, c.cfg, 64, 4096)
    for new in ([1, 0, 0], [1, 1, 1], [30, 2, 1], [300, 0, 200]):
        off, n = offsets(new), sum(new)
        q = rand(gen, "bf16", n, 8, 64)
        out = torch.full_like(q, 7.0)
        B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, ws)
        for b, n_b in enumerate(lens):
            check_attention(host(out[off[b]:off[b + 1]]), host(q[off[b]:off[b + 1]]), *c.rows(b, n_b), "bf16", what=(new, b))
    q = rand(gen, "bf16", 3, 8, 64)
    out = torch.full_like(q, 7.0)
    B.flame_kv_decode(c.cfg, c.packed, q, ints(lens), out, ws)
    for b, n_b in enumerate(lens):
        check_attention(host(out[b:b + 1]), host(q[b:b + 1]), *c.rows(b, n_b), "bf16", what=("decode", b))


WRONG_OFFSETS = [[0, 30, -2 ** 31, 60], [0, 30, -2 ** 31, 2 ** 31 - 1], [0, 30, 5, 60], [0, 30, 29, 29], [0, 30, 0, 60], [0, 20, 30, 10, 60, 0, 60], [0, 30, -1, 60, 0, 60, 0, 60], [-5, 40, 50, 60]]


def before_the_wrong(off):
    """Sequences before the first offset that decreases or is below 0."""
    n = 0
    while n < len(off) - 1 and 0 <= off[n] <= off[n + 1]:
        n += 1
    return n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", WRONG_OFFSETS, ids=str)
def test_sequences_before_offsets_that_are_none(B, dtype, off):
    """Of up to 64 sequences those before the first offset that decreases or is below 0 have their results, whatever the others claim (their rows, most of the keys, millions of rows);
    rows of no such sequence stay as they were.  Row tiles, in parts, split."""
    import torch
    gen, n_seqs, good = generator(18), len(off) - 1, before_the_wrong(off)
    lens = [900] + [1200, 90, 1500, 64, 1300, 1400][:n_seqs - 1]
    rows = off[good] if good else 0
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    for room, hq in ((0, 4), (4096, 64), (4096, 2)):
        c = Cache(B, gen, dtype, hq, hq, 64, lens, 16, tokens=room)
        q, k = rand(gen, dtype, 60, hq, 64), rand(gen, dtype, 60, hq, 64)
        for kind in ("prompt", "extend"):
            buffer = torch.full((180, hq, 64), 7.0, dtype=q.dtype, device=DEV)
            out = buffer[60:120]
            fault.zero_()
            if kind == "prompt":
                B.flame_kv_prompt(c.cfg, q, k, k, ints(off), out, faults=fault)
            else:
                ws = torch.zeros(B.flame_kv_workspace_bytes(c.cfg, n_seqs, 60), dtype=torch.uint8, device=DEV)
                B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, ws, faults=fault)
            assert int(fault[0]) == 4, (kind, room)
            assert bool((buffer[:60] == 7.0).all()) and bool((buffer[60 + rows:] == 7.0).all()), (kind, room)
            for b in range(good):
                s = slice(off[b], off[b + 1])
                keys, values = (host(k[s]), host(k[s])) if kind == "prompt" else c.rows(b, lens[b])
                check_attention(host(out[s, :1]), host(q[s, :1]), keys[:, :1], values[:, :1], dtype, what=(kind, room, hq, b))


@pytest.mark.parametrize("off", WRONG_OFFSETS, ids=str)
def test_append_before_offsets_that_are_none(B, off):
    """The same of append: reported, and exactly the tokens of the sequences before are written."""
    import torch
    gen, n_seqs, good = generator(19), len(off) - 1, before_the_wrong(off)
    cfg = B.make_kv_config("bf16", 2, 1, 32)
    table = np.arange(n_seqs * 8, dtype=np.int32).reshape(n_seqs, 8)
    k_pool, v_pool = (torch.zeros(n_seqs * 8, 16, 1, 32, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    k, q = rand(gen, "bf16", 60, 1, 32), rand(gen, "bf16", 60, 2, 32)
    q_out, fault = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    lens = [100 + b for b in range(n_seqs)]
    B.flame_kv_append(cfg, B.pack_kv_cache(cfg, k_pool, v_pool, ints(table)), k, k, ints(off), ints(lens), q=q, q_out=q_out, faults=fault)
    assert int(fault[0]) == 4
    rows = off[good] if good else 0
    assert torch.equal(q_out[:rows], q[:rows]) and bool((q_out[rows:] == 7.0).all())
    want = torch.zeros_like(k_pool)
    for b in range(good):
        for i in range(off[b], off[b + 1]):
            t = lens[b] - off[b + 1] + i
            want[int(table[b, t // 16]), t % 16] = k[i]
    assert torch.equal(k_pool, want) and torch.equal(v_pool, want)


def test_append_reports_offsets_and_writes_the_rest(B):
    """Offsets that decrease, begin below 0 or end behind the rows: the bit, and the slots that are written.  Rows ahead of the first sequence are like those behind the last one."""
    import torch
    gen = generator(20)
    cfg = B.make_kv_config("bf16", 2, 1, 32)
    k_pool, v_pool = torch.zeros(4, 4, 1, 32, device=DEV, dtype=torch.bfloat16), torch.zeros(4, 4, 1, 32, device=DEV, dtype=torch.bfloat16)
    cache = B.pack_kv_cache(cfg, k_pool, v_pool, ints([[0, 1], [2, 3]]))
    k = rand(gen, "bf16", 12, 1, 32)
    first, second = [(0, i) for i in range(4)] + [(1, i) for i in range(4)], [(2, i) for i in range(4)]
    for off, lens, fault, slots in (([0, 4, 2], [4, 2], 4, first[:4]), ([-3, 4, 5], [4, 2], 4, []), ([0, 8, 20], [8, 12], 4, first + second), ([2, 4, 6], [2, 3], 0, first[:2] + second[1:3])):
        k_pool.zero_(), v_pool.zero_()
        faults = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.flame_kv_append(cfg, cache, k, k, ints(off), ints(lens), faults=faults)
        there = [tuple(x) for x in (k_pool.abs().sum((2, 3)) > 0).nonzero().tolist()]
        assert (int(faults[0]), there) == (fault, slots), off
        assert torch.equal(k_pool, v_pool)
    # attention has the same view of rows ahead of the first sequence
    q, fault = rand(gen, "bf16", 12, 2, 32), torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 7.0)
    B.flame_kv_prompt(cfg, q, k, k, ints([2, 4, 9]), out, faults=fault)
    assert int(fault[0]) == 0 and bool((out[:2] == 7.0).all()) and bool((out[9:] == 7.0).all()) and not bool((out[2:9] == 7.0).all(-1).any())


def test_fp16_weights_far_below_the_largest(B):
    """One key with a logit of 17.47 and a value of 0, thousands with logits of 0 and values of 1: weights of 2^-25.2, which fp16 does not have, make up the result together.
    An fp16 weight is off by half a step or by 2^-32 of the row's largest (2^-40 where the keys are split)."""
    import torch
    c = float(np.float16(17.47))
    w, n = math.exp(-c), 4096

    def inputs(dim, tokens, hq):
        q, k = torch.zeros(tokens, hq, dim, device=DEV, dtype=torch.float16), torch.zeros(n, 2, dim, device=DEV, dtype=torch.float16)
        v = torch.ones_like(k)
        q[..., 0], k[0, :, 0], v[0] = c, 1.0, 0.0
        return q, k, v

    def check(got, last, dim, lost, what):
        others = np.asarray(last, np.float64)[:, None, None]               # keys but the first that a row sees
        want = others * w / (1 + others * w)
        bound = want * (2 * 2.0 ** -11 + 2 * ((dim + 7) * 2.0 ** -24 * c + 2.0 ** -22) + 4 * n * 2.0 ** -24) + n * lost + 2.0 ** -24
        off = np.abs(host(got) - want)
        assert (off <= bound).all(), (what, float((off / bound).max()))

    for dim in (32, 64, 128):
        cfg = B.make_kv_config("f16", 8, 2, dim, scale=1.0)
        for size in (0, 1, 2):
            q, k, v = inputs(dim, n, 8)
            out = torch.full_like(q, 7.0)
            B.flame_kv_prompt(cfg, q, k, v, ints(offsets([n] + spread(size, "f16", 2))), out)
            check(out, np.arange(n), dim, 2.0 ** -32, ("prompt", dim, size))
        pools = [x.reshape(256, 16, 2, dim) for x in inputs(dim, 1, 8)[1:]]
        for seqs, new in ((1, 100), (8, 300), (256, 1)):                  # in parts, whole, split: all sequences have the same pages
            cache = B.pack_kv_cache(cfg, *pools, ints(np.tile(np.arange(256), (seqs, 1))))
            q = inputs(dim, seqs * new, 8)[0]
            out, lens = torch.full_like(q, 7.0), ints([n] * seqs)
            if new == 1:
                B.flame_kv_decode(cfg, cache, q, lens, out, workspace_for(B, cfg, seqs))
            else:
                B.flame_kv_extend(cfg, cache, q, ints(offsets([new] * seqs)), lens, out, workspace_for(B, cfg, seqs, seqs * new))
            check(out, np.tile(np.arange(n - new, n), seqs), dim, 2.0 ** -40 if new == 1 else 2.0 ** -32, (dim, seqs, new))


@pytest.mark.parametrize("dtype,power", [("f16", 30), ("bf16", 100), ("f32", 100)])
def test_infinite_values_of_small_weights(B, dtype, power):
    """A weight of 2^-30 (fp16) or 2^-100 of the largest is a weight: an infinite value that it has makes the row infinite, on every route."""
    import torch
    n, dim, room = 3000, 64, 4096
    gen = generator(21)
    cfg = B.make_kv_config(dtype, 8, 2, dim, scale=1.0)
    k, v = torch.zeros(room, 2, dim, device=DEV, dtype=torch_type(dtype)), rand(gen, dtype, room, 2, dim)
    k[..., 0] = -math.log(2.0) * power / 8                             # logits of -power ln 2,
    k[5, :, 0] = 0.0                                                   # and one of 0
    v[40, :, 3], v[41, :, 4] = math.inf, -math.inf
    cache = B.pack_kv_cache(cfg, k.reshape(256, 16, 2, dim), v.reshape(256, 16, 2, dim), ints(np.tile(np.arange(256), (64, 1))))
    for seqs, new in ((1, 100), (8, 300), (64, 1)):
        q = torch.zeros(seqs * new, 8, dim, device=DEV, dtype=torch_type(dtype))
        q[..., 0] = 8.0
        out, lens = torch.full_like(q, 7.0), ints([n] * seqs)
        if new == 1:
            B.flame_kv_decode(cfg, cache, q, lens, out, workspace_for(B, cfg, seqs))
        else:
            B.flame_kv_extend(cfg, cache, q, ints(offsets([new] * seqs)), lens, out, workspace_for(B, cfg, seqs, seqs * new))
        assert bool((out[..., 3] == math.inf).all()) and bool((out[..., 4] == -math.inf).all()), (seqs, new)
        assert bool(out[..., 5:].isfinite().all()) and bool(out[..., :3].isfinite().all()), (seqs, new)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_rows_without_a_logit_above_minus_infinity(B, dtype, dim):
    """Every logit is -infinity: zeros on every route, whatever the values hold."""
    import torch
    gen, n = generator(22), 1500
    cfg = B.make_kv_config(dtype, 8, 2, dim)
    k, v = rand(gen, dtype, 4096, 2, dim), rand(gen, dtype, 4096, 2, dim)
    k[..., 0] = -math.inf
    v[100, :, 3], v[200, :, 4], v[1400, :, 5] = math.inf, math.nan, -math.inf

    def queries(tokens):
        q = torch.zeros(tokens, 8, dim, device=DEV, dtype=torch_type(dtype))
        q[..., 0] = 1.0
        return q

    for size in (0, 1, 2):
        q = queries(n)
        out = torch.full_like(q, 7.0)
        B.flame_kv_prompt(cfg, q, k[:n], v[:n], ints(offsets([n] + spread(size, dtype, 2))), out)
        assert not bool(out.any()), ("prompt", size)
    for seqs, new, pages in ((1, 100, 256), (8, 300, 256), (8, 3, 256), (8, 1, 256), (2, 40, 10)):
        cache = B.pack_kv_cache(cfg, k.reshape(256, 16, 2, dim), v.reshape(256, 16, 2, dim), ints(np.tile(np.arange(pages), (seqs, 1))))
        q, lens = queries(seqs * new), ints([min(n, pages * 16)] * seqs)
        out = torch.full_like(q, 7.0)
        B.flame_kv_extend(cfg, cache, q, ints(offsets([new] * seqs)), lens, out, workspace_for(B, cfg, seqs, seqs * new))
        assert not bool(out.any()), ("extend", seqs, new)
        if new == 1:
            out.fill_(7.0)
            B.flame_kv_decode(cfg, cache, q, lens, out, workspace_for(B, cfg, seqs))
            assert not bool(out.any()), "decode"


@pytest.mark.parametrize("n_seqs", [1, 63, 64, 65, 129, 700, 4096, 4200])
@pytest.mark.parametrize("ahead", [0, 5])
def test_append_of_many_sequences(B, n_seqs, ahead):
    """More sequences than lanes, most of them with a token or none, with rows ahead of the first and behind the last one: every token in its slot, and nothing else written."""
    import torch
    gen, rng = generator(n_seqs), np.random.default_rng(n_seqs)
    new = rng.integers(0, 3, n_seqs)
    new[[0, n_seqs // 2, n_seqs - 1]] = [7, 70, 3]
    lens = new + rng.integers(0, 20, n_seqs)
    off, n = offsets(new) + ahead, int(new.sum())
    used = -(-lens // 16)
    table = np.full((n_seqs, int(used.max())), -7, np.int32)
    order = rng.permutation(int(used.sum()))
    for b, first in enumerate(np.cumsum(used) - used):
        table[b, :used[b]] = order[first:first + used[b]]
    cfg = B.make_kv_config("f16", 2, 1, 32)
    k_pool, v_pool = (torch.zeros(len(order), 16, 1, 32, device=DEV, dtype=torch.float16) for _ in range(2))
    k, v, q = rand(gen, "f16", n + ahead + 6, 1, 32), rand(gen, "f16", n + ahead + 6, 1, 32), rand(gen, "f16", n + ahead + 6, 2, 32)
    q_out, fault = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = B.pack_kv_cache(cfg, k_pool, v_pool, ints(table))
    B.flame_kv_append(cfg, cache, k, v, ints(off), ints(lens), q=q, q_out=q_out, faults=fault)
    seq = np.repeat(np.arange(n_seqs), new)
    position = np.arange(n) - (off - ahead)[seq + 1] + lens[seq]
    page, slot = (torch.tensor(x, device=DEV).long() for x in (table[seq, position // 16], position % 16))
    for pool, x in ((k_pool, k), (v_pool, v)):
        want = torch.zeros_like(pool)
        want[page, slot] = x[ahead:ahead + n]
        assert torch.equal(pool, want)
    assert int(fault[0]) == 0
    assert torch.equal(q_out[ahead:ahead + n], q[ahead:ahead + n]) and bool((q_out[:ahead] == 7.0).all()) and bool((q_out[ahead + n:] == 7.0).all())
    # the last sequence's end behind the rows is seen, whichever workgroup looks at it
    off[-1] += 100
    B.flame_kv_append(cfg, cache, k, v, ints(off), ints(lens + 100 * (np.arange(n_seqs) == n_seqs - 1)), faults=fault)
    assert int(fault[0]) & 4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs", [3, 64, 65, 300])
def test_attention_with_rows_ahead_of_the_first_sequence(B, dtype, n_seqs):
    """offsets that do not begin at 0, as those of a part of a larger batch: row tiles, in parts, split."""
    import torch
    gen, rng, ahead = generator(23), np.random.default_rng(n_seqs), 40
    new = rng.integers(0, 4, n_seqs)
    new[[0, n_seqs - 1]] = [50, 33]
    off, n = offsets(new) + ahead, int(new.sum()) + ahead
    lens = new + rng.integers(0, 30, n_seqs)
    lens[0] = 900
    for room, hq in ((0, 4), (4096, 16), (4096, 2)):
        c = Cache(B, gen, dtype, hq, 2, 64, lens.tolist(), 16, tokens=room)
        q, k = rand(gen, dtype, n + 7, hq, 64), rand(gen, dtype, n + 7, 2, 64)
        pool_k, pool_v = host(c.k), host(c.v)
        for kind in ("prompt", "extend"):
            out, fault = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
            if kind == "prompt":
                B.flame_kv_prompt(c.cfg, q, k, k, ints(off), out, faults=fault)
            else:
                B.flame_kv_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, n_seqs, n + 7), faults=fault)
            assert int(fault[0]) == 0
            assert bool((out[:ahead] == 7.0).all()) and bool((out[n:] == 7.0).all())
            for b in [0, n_seqs // 2, n_seqs - 1]:
                s = slice(off[b], off[b + 1])
                if kind == "prompt":
                    keys = values = host(k[s])
                else:
                    page, slot, _ = kv_oracle.page_rows(c.table_host[b], 16, c.n_pages, int(lens[b]))
                    keys, values = pool_k[page, slot], pool_v[page, slot]
                check_attention(host(out[s]), host(q[s]), keys, values, dtype, what=(kind, room, hq, b))
