"""The cache of 8 or 4 bits (include/flame_kvq.h) and attention over shared histories (flame_kv_shared, flame_kvq_shared) against the oracle in 64 bits.

Tolerances.  Without rotation codes, scales and values read back are exact.  With it, a stored value is off by the half step that the header states (2^-4 or 2^-2 of the value, or
2^-10 or 2^-2 of the block's scale), where the scale is at most twice the block's largest size over 464 or 7, and by the rotation's error ahead of it, 2^-21 of the pair's sizes.
Attention is held to what flame_kv.h allows (tests/test_gpu_kv.py derives it) against the oracle on the values that the cache holds:
u |o| + W (u_w + 2 ((dim + 7) 2^-24 Z + 2^-22) + 4 n 2^-24), and for f16 outputs 2^-24 and weights 2^-25 n max|v|."""
import math

import numpy as np
import pytest

from oracle import kv_oracle
from test_gpu_kv import B, DEV, HALF_STEP, generator, host, ints, offsets, rand, torch_type  # noqa: F401

pytestmark = pytest.mark.gpu

FORMS = ("f8", "f4")
HALF = {"f8": (2.0 ** -4, 2.0 ** -10, 464.0), "f4": (2.0 ** -2, 2.0 ** -2, 7.0)}


def check_attention(got, q, k, v, dtype, seen=None, what=""):
    dim, n = q.shape[2], k.shape[0]
    want, spread, size = kv_oracle.attend(q, k, v, dim ** -0.5, seen)
    u = HALF_STEP[dtype]
    d = (dim + 7) * 2.0 ** -24 * size[..., None] + 2.0 ** -22
    bound = u * np.abs(want) + spread * ((0 if dtype == "f32" else u) + 2 * d + 4 * n * 2.0 ** -24) + 1e-30
    if dtype == "f16":
        bound = bound + 2.0 ** -24 + n * 2.0 ** -25 * (np.abs(v).max() if n else 0)
    off = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (off <= bound).all(), (what, float((off / bound).max()), float(off.max()))


class Cache:
    """Sequences of n tokens in scattered pages of a quantised pool (form None: a plain one) of random values, with pages that nobody has; groups: lists of sequences that share their
    first p tokens' pages."""

    def __init__(self, B, gen, form, dtype, hq, hkv, dim, lens, page, head_major=False, seed=0, tokens=0, groups=(), prefix=()):
        import torch
        self.B, self.form, self.page, self.lens, self.dtype = B, form, page, list(lens), dtype
        self.cfg = B.make_kv_config(dtype, hq, hkv, dim)
        full = np.zeros(len(lens), np.int64)
        for g, p in zip(groups, prefix):
            for b in g:
                full[b] = p // page
        need = np.array([max(0, -(-n // page)) for n in lens])
        for g, p in zip(groups, prefix):
            if g:
                need[g[0]] = max(need[g[0]], -(-p // page))            # the first sequence's row names the whole history
        own = np.maximum(0, need - full)
        trunk = [p // page for g, p in zip(groups, prefix)]
        self.n_pages = int(own.sum() + sum(trunk)) + 3
        order = list(np.random.default_rng(seed).permutation(self.n_pages))
        self.table_host = np.full((len(lens), max(int(need.max(initial=1)) + 1, -(-tokens // page))), -7, np.int32)
        for g, t in zip(groups, trunk):
            pages = [order.pop() for _ in range(t)]
            for i, b in enumerate(g):
                # (the rows of others name no pages where these are shared alone)
                self.table_host[b, :t] = pages if i == 0 else -7
        for b in range(len(lens)):
            self.table_host[b, full[b]:full[b] + own[b]] = [order.pop() for _ in range(own[b])]
        self.table = ints(self.table_host)
        shape = (self.n_pages, hkv, page, dim) if head_major else (self.n_pages, page, hkv, dim)
        turn = (lambda t: t.transpose(1, 2)) if head_major else (lambda t: t)
        if form is None:
            self.k, self.v = turn(rand(gen, dtype, *shape)), turn(rand(gen, dtype, *shape))
            self.pack()
            return
        parts = {}
        for x in "kv":
            codes, scales, _ = kv_oracle.quantise(host(rand(gen, dtype, *shape)), form, dtype)
            codes = codes if form == "f8" else codes[..., 0::2] | codes[..., 1::2] << 4
            parts[x] = turn(torch.tensor(codes.astype(np.uint8), device=DEV))
            parts[x + "s"] = turn(torch.tensor(scales.astype(np.uint8), device=DEV))
        self.k, self.v, self.ks, self.vs = parts["k"], parts["v"], parts["ks"], parts["vs"]
        self.pack()

    def pack(self):
        self.packed = self.B.pack_kv_cache(self.cfg, self.k, self.v, self.table) if self.form is None else \
            self.B.pack_kvq_cache(self.cfg, self.form, self.k, self.v, self.ks, self.vs, self.table)

    def pools(self):
        """Values of the pools, in 64 bits."""
        if self.form is None:
            return host(self.k), host(self.v)
        return tuple(kv_oracle.stored_values(kv_oracle.unpack(p.cpu().numpy(), self.form), s.cpu().numpy(), self.form) for p, s in ((self.k, self.ks), (self.v, self.vs)))

    def rows(self, b, n, trunk=0, trunk_seq=0, pools=None):
        """Keys and values of tokens 0..n-1 of sequence b, the first `trunk` of them where sequence trunk_seq has them."""
        k, v = pools or self.pools()
        t = np.arange(n)
        page = np.where(t < trunk, self.table_host[trunk_seq, t // self.page], self.table_host[b, t // self.page])
        return k[page, t % self.page], v[page, t % self.page]


def call(B, c, op, *args, **more):
    return getattr(B, ("flame_kv_" if c.form is None else "flame_kvq_") + op)(c.cfg, c.packed, *args, **more)


# ---------------------------------------------------------------------------------------------- append and read
APPENDS = [("f8", "bf16", 8, 2, 64, 64, False, 16, False), ("f4", "bf16", 32, 8, 128, 128, True, 24, True), ("f8", "f16", 4, 4, 32, 32, False, 1, False), ("f4", "f16", 6, 1, 128, 64, False, 7, False),
           ("f8", "f32", 8, 8, 64, 32, True, 100, True), ("f4", "f32", 3, 3, 128, 128, False, 16, False), ("f4", "bf16", 5, 5, 32, 16, True, 64, False), ("f8", "bf16", 4, 2, 128, 16, False, 16, True),
           ("f8", "f32", 2, 1, 32, 0, False, 5, False), ("f4", "bf16", 3, 3, 64, 0, False, 16, True), ("f8", "f16", 20, 20, 128, 48, False, 33, False), ("f4", "f32", 2, 2, 32, 0, False, 16, False)]


@pytest.mark.parametrize("form,dtype,hq,hkv,dim,rot,inter,page,head_major", APPENDS)
def test_append(B, form, dtype, hq, hkv, dim, rot, inter, page, head_major):  # noqa: F811
    import torch
    gen = generator(dim + page)
    new, before = [1, 0, 5, 70, 1, 33], [0, 9, 100, 3, 47, 64]
    lens = [a + b for a, b in zip(new, before)]
    c = Cache(B, gen, form, dtype, hq, hkv, dim, lens, page, head_major)
    n = sum(new)
    rows = rand(gen, dtype, n + 3, hq + 2 * hkv, dim)                   # slices of wider rows, three rows behind the last sequence
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    q_out = torch.full((n + 3, hq, dim), 7.0, device=DEV, dtype=torch_type(dtype))
    f = B.flame_kv_rotation_frequencies(rot) if rot else np.zeros(0)
    rotation = B.make_kv_rotation(f, inter) if rot else None
    keep = [t.clone() for t in (c.k, c.v, c.ks, c.vs)]
    faults = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kvq_append(c.cfg, c.packed, k, v, ints(offsets(new)), ints(lens), q=q, q_out=q_out, rotation=rotation, faults=faults)
    torch.cuda.synchronize()
    assert int(faults[0]) == 0
    position = np.concatenate([np.arange(a, a + m) for a, m in zip(before, new)])
    seq = np.repeat(np.arange(len(new)), new)
    where = c.table_host[seq, position // page], position % page
    pool_k, pool_v = c.pools()
    codes, scales, values = kv_oracle.quantise(host(v[:n]), form, dtype)
    assert np.array_equal(kv_oracle.unpack(c.v.cpu().numpy(), form)[where], codes) and np.array_equal(c.vs.cpu().numpy()[where], scales) and np.array_equal(pool_v[where], values)
    turned = kv_oracle.rotate(host(k[:n]), position, f, inter)
    if not rot:
        codes, scales, _ = kv_oracle.quantise(turned, form, dtype)
        assert np.array_equal(kv_oracle.unpack(c.k.cpu().numpy(), form)[where], codes) and np.array_equal(c.ks.cpu().numpy()[where], scales)
    relative, least, limit = HALF[form]
    pair = np.abs(host(k[:n])).max(-1, keepdims=True) * 2 * 2.0 ** -21 if rot else 0
    scale = np.repeat((np.abs(turned).reshape(*turned.shape[:-1], -1, 32).max(-1) + pair) * 2 / limit, 32, -1)
    assert (np.abs(pool_k[where] - turned) <= pair * (1 + relative) + np.maximum(relative * np.abs(turned), least * scale)).all()
    want_q = kv_oracle.rotate(host(q[:n]), position, f, inter)
    wide = np.abs(host(q[:n])).max(-1, keepdims=True) * 2
    assert (np.abs(host(q_out)[:n] - want_q) <= HALF_STEP[dtype] * np.abs(want_q) + (wide * 2.0 ** -21 if rot else 0) + (2.0 ** -25 if dtype == "f16" else 0)).all()
    assert bool((q_out[n:] == 7.0).all())                               # rows behind the last sequence
    untouched = np.ones(c.k.shape[:2], bool)
    untouched[where] = False
    untouched = torch.tensor(untouched, device=DEV)
    for was, now in zip(keep, (c.k, c.v, c.ks, c.vs)):
        assert torch.equal(was[untouched], now[untouched])
    # in place, and without queries: the same bits
    first, again = [t.clone() for t in (c.k, c.ks)], q.clone()
    B.flame_kvq_append(c.cfg, c.packed, k, v, ints(offsets(new)), ints(lens), q=again, q_out=again, rotation=rotation)
    assert torch.equal(again[:n], q_out[:n]) and torch.equal(again[n:], q[n:])
    c.k.copy_(keep[0]), c.ks.copy_(keep[2])
    B.flame_kvq_append(c.cfg, c.packed, k, v, ints(offsets(new)), ints(lens), rotation=rotation)
    assert torch.equal(c.k, first[0]) and torch.equal(c.ks, first[1])
    # and back: exactly the values, in rows of both layouts
    for turn in (False, True):
        shape = (hkv, n + 3, dim) if turn else (n + 3, hkv, dim)
        rk, rv = (torch.full(shape, 7.0, device=DEV, dtype=torch_type(dtype)) for _ in range(2))
        rk, rv = (rk.transpose(0, 1), rv.transpose(0, 1)) if turn else (rk, rv)
        B.flame_kvq_read(c.cfg, c.packed, ints(offsets(new)), ints(lens), rk, rv, faults=faults)
        assert np.array_equal(host(rk)[:n], pool_k[where]) and np.array_equal(host(rv)[:n], pool_v[where]) and int(faults[0]) == 0
        assert bool((rk[n:] == 7.0).all()) and bool((rv[n:] == 7.0).all())


def edge_blocks(dtype):
    """Blocks of 32 whose largest sizes lie on both sides of every border, over the type's range, with each of the other features anywhere below."""
    import torch
    rng = np.random.default_rng(5)
    step = {"bf16": 2.0 ** -7, "f16": 2.0 ** -10, "f32": 2.0 ** -23}[dtype]
    exps = np.arange(-24, 16) if dtype == "f16" else np.concatenate([np.arange(-149, -100), np.arange(-20, 20), np.arange(110, 128)])
    blocks = []
    for e in exps:
        for f in (1.0, 1.5, 1.75 - step, 1.75, 1.75 + step, 1.8125 - step, 1.8125, 1.8125 + step, 1.875, 2 - step):
            top = f * 2.0 ** float(e)
            x = top * rng.choice([1, -1], 32) * np.concatenate([[1], 2.0 ** rng.uniform(-12, 0, 15), np.arange(16) / 16])
            blocks.append(x)
    blocks.append(np.zeros(32))
    blocks.append(np.where(np.arange(32) % 2, -0.0, 0.0))
    t = torch.tensor(np.array(blocks), dtype=torch.float64).to(torch_type(dtype))
    odd = t[:6].clone()
    for i, x in enumerate((math.inf, -math.inf, math.nan, math.inf, 65504.0, -math.nan)):
        odd[i, 7 * i % 32] = x
    t = torch.cat([t, odd])
    return t[torch.isfinite(t).all(1) | (torch.arange(len(t)) >= len(t) - 6)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_every_border_of_the_codes(B, form, dtype):  # noqa: F811
    """Largest sizes at the borders of the exponents, halves between codes, the smallest and largest values of the type, signs of zero, infinities and NaN: codes and scales bit for bit, and
    the values back (a value below the normal range of fp32 may be taken as zero)."""
    import torch
    x = edge_blocks(dtype)
    x = x[:len(x) // 4 * 4].reshape(-1, 1, 128).to(DEV)
    n = len(x)
    cfg = B.make_kv_config(dtype, 1, 1, 128)
    pool = B.make_kvq_pool(cfg, form, 2, n)
    cache = B.pack_kvq_cache(cfg, form, *pool, ints([[1]]))
    B.flame_kvq_append(cfg, cache, x, x.flip(2).contiguous(), ints([0, n]), ints([n]))
    back_k, back_v = torch.empty_like(x), torch.empty_like(x)
    B.flame_kvq_read(cfg, cache, ints([0, n]), ints([n]), back_k, back_v)
    for data, codes_t, scales_t, back in ((x, pool[0], pool[2], back_k), (x.flip(2), pool[1], pool[3], back_v)):
        codes, scales, values = kv_oracle.quantise(host(data), form, dtype)
        got = kv_oracle.unpack(codes_t[1].cpu().numpy(), form)
        whole = np.repeat(scales != 255, 32, -1)
        flushed = (np.abs(host(data)) < 2.0 ** -126) & (got % (128 if form == "f8" else 8) == 0)
        assert np.array_equal(scales_t[1].cpu().numpy(), scales)
        assert (got == codes)[whole & ~flushed].all(), np.argwhere((got != codes) & whole & ~flushed)[:5]
        assert np.array_equal(host(back)[whole & ~flushed], values[whole & ~flushed]) and np.isnan(host(back)[~whole]).all()
        assert np.isfinite(host(back)[whole]).all()


@pytest.mark.parametrize("form", FORMS)
def test_append_and_read_report_what_they_cannot_place(B, form):  # noqa: F811
    """Bad pages, lengths beyond the table's row and below the new tokens, offsets that decrease: nothing out of range is touched, and the rest is done."""
    import torch
    gen = generator(2)
    cfg = B.make_kv_config("bf16", 2, 1, 32)
    pool = B.make_kvq_pool(cfg, form, 6, 4)
    guarded = [p[1:5] for p in pool]                                    # pages on both sides that no entry may reach
    k = rand(gen, "bf16", 12, 1, 32).abs() + 0.5

    def both(table, off, lens):
        [p.zero_() for p in pool]
        faults = torch.zeros(2, dtype=torch.int32, device=DEV)
        cache = B.pack_kvq_cache(cfg, form, *guarded, ints(table))
        B.flame_kvq_append(cfg, cache, k, k, ints(off), ints(lens), faults=faults[:1])
        torch.cuda.synchronize()
        for p in pool:
            assert not p[0].any() and not p[5].any()
        assert torch.equal(pool[0], pool[1]) and torch.equal(pool[2], pool[3])
        rk, rv = torch.full_like(k, 7.0), torch.full_like(k, 7.0)
        B.flame_kvq_read(cfg, cache, ints(off), ints(lens), rk, rv, faults=faults[1:])
        assert int(faults[0]) == int(faults[1]) and torch.equal(rk, rv)
        return int(faults[0]), [tuple(x) for x in (pool[0][1:5].int().sum((2, 3)) > 0).nonzero().tolist()], [i for i in range(12) if bool((rk[i] != 7.0).any())]

    assert both([[0, 1], [2, 3]], [0, 2, 4], [2, 8]) == (0, [(0, 0), (0, 1), (3, 2), (3, 3)], [0, 1, 2, 3])
    assert both([[0, 4], [-1, 3]], [0, 2, 6], [6, 6]) == (1, [(3, 0), (3, 1)], [4, 5])
    assert both([[0, 1], [2, 3]], [0, 3, 5], [2, 9]) == (2, [(0, 0), (0, 1), (3, 3)], [1, 2, 3])
    both([[0, 1], [2, 3]], [0, 4, 2], [4, 2])                           # offsets that decrease
    both([[0, 1], [2, 3]], [-3, 4, 5], [4, 2])
    fault, there, _ = both([[0, 1], [2, 3]], [0, 8, 20], [8, 8])        # twelve rows are there, and eight of the second sequence are not
    assert fault & 4 and all(p in (0, 1, 2, 3) for p, _ in there)


# ---------------------------------------------------------------------------------------------- attention over quantised caches
HEADS = [("bf16", 8, 2, 64), ("bf16", 4, 4, 128), ("f16", 6, 2, 128), ("f16", 3, 3, 32), ("bf16", 8, 1, 32), ("f16", 4, 4, 64), ("f32", 4, 2, 64), ("f32", 2, 2, 128), ("f32", 3, 1, 32)]


def workspace_for(B, cfg, n_seqs, n_tokens=None):  # noqa: F811
    import torch
    return torch.full((B.flame_kv_workspace_bytes(cfg, n_seqs, n_tokens),), 0xff, dtype=torch.uint8, device=DEV)     # it holds nothing between calls: NaN


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,hq,hkv,dim", HEADS + [("bf16", 32, 1, 64), ("f16", 40, 2, 32), ("f32", 20, 1, 64)])
@pytest.mark.parametrize("page,head_major", [(16, False), (24, True), (1, False), (300, True)])
def test_decode(B, form, dtype, hq, hkv, dim, page, head_major):  # noqa: F811
    import torch
    gen, lens = generator(page), [1, 0, 31, 32, 33, 700, 64, 129]
    c = Cache(B, gen, form, dtype, hq, hkv, dim, lens, page, head_major)
    q = rand(gen, dtype, len(lens), hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kvq_decode(c.cfg, c.packed, q, ints(lens), out, workspace_for(B, c.cfg, len(lens)), faults=faults)
    assert int(faults[0]) == 0
    pools = c.pools()
    for b, n in enumerate(lens):
        check_attention(host(out[b:b + 1]), host(q[b:b + 1]), *c.rows(b, n, pools=pools), dtype, what=(b, n))


EXTENDS = [([1, 3, 0, 2, 5], [1, 40, 7, 300, 90], 0), ([70, 200, 1], [700, 200, 33], 0), ([300], [900], 4096), ([3, 1, 17], [2000, 1500, 40], 8192), ([9, 5], [4, 5], 0), ([130, 60, 2], [1100, 61, 1], 2048),
           ([33] * 70, [50] * 70, 0)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,hq,hkv,dim", HEADS)
@pytest.mark.parametrize("new,lens,tokens", EXTENDS, ids=lambda x: str(x)[:24])
def test_extend(B, form, dtype, hq, hkv, dim, new, lens, tokens):  # noqa: F811
    """Few rows and many, short caches and long ones, rows that see nothing, a row behind the last sequence."""
    import torch
    gen = generator(len(new) + dim)
    c = Cache(B, gen, form, dtype, hq, hkv, dim, lens, 24, tokens=tokens)
    n, off = sum(new), offsets(new)
    q = rand(gen, dtype, n + 2, hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kvq_extend(c.cfg, c.packed, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, len(new), n + 2), faults=faults)
    assert int(faults[0]) == 0 and bool((out[n:] == 7.0).all())
    pools = c.pools()
    for b in ([0, len(new) - 1] if len(new) > 20 else range(len(new))):
        s = slice(off[b], off[b + 1])
        if new[b]:
            check_attention(host(out[s]), host(q[s]), *c.rows(b, lens[b], pools=pools), dtype, what=(b, new[b], lens[b]))
            assert not out[s][:max(0, new[b] - lens[b])].any()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("room", [0, 4096])
def test_rows_do_not_feel_what_they_do_not_see(B, form, dtype, dim, room):  # noqa: F811
    """Blocks of NaN at later tokens: earlier rows keep their bits; rows that see them are NaN in the block's 32 features (values) or all over (keys); and pages that the table does
    not name are no keys."""
    import torch
    gen = generator(3)
    lens, new = [200, 90], [150, 90]
    c = Cache(B, gen, form, dtype, 4, 2, dim, lens, 16, tokens=room)
    off, ws = ints(offsets(new)), workspace_for(B, c.cfg, 2, 240)
    q = rand(gen, dtype, 240, 4, dim)
    clean, dirty = torch.empty_like(q), torch.empty_like(q)
    B.flame_kvq_extend(c.cfg, c.packed, q, off, ints(lens), clean, ws)
    last = q[[149, 239]].contiguous()
    for at in (50, 77, 130, 199):
        page, slot, row = c.table_host[0, at // 16], at % 16, max(0, at - 50)
        for scales, where in ((c.vs, "v"), (c.ks, "k")):
            was = int(scales[page, slot, 1, dim // 32 - 1])
            scales[page, slot, 1, dim // 32 - 1] = 255
            B.flame_kvq_extend(c.cfg, c.packed, q, off, ints(lens), dirty, ws)
            assert torch.equal(dirty[:row], clean[:row]) and torch.equal(dirty[150:], clean[150:]), (at, where)
            assert torch.equal(dirty[:, :2], clean[:, :2])
            if where == "v":
                assert bool(dirty[row:150, 2:, dim - 32:].isnan().all()) and torch.equal(dirty[..., :dim - 32], clean[..., :dim - 32])
            else:
                assert bool(dirty[row:150, 2:].isnan().all())
            single = torch.empty_like(last)
            B.flame_kvq_decode(c.cfg, c.packed, last, ints(lens), single, ws)
            assert bool(single[0, 2:, dim - 32:].isnan().all()) and bool(single[:, :2].isfinite().all()) and bool(single[1].isfinite().all())
            scales[page, slot, 1, dim // 32 - 1] = was
    B.flame_kvq_extend(c.cfg, c.packed, q, off, ints(lens), dirty, ws)
    assert torch.equal(dirty, clean)
    # a page that is none
    c.table_host[0, 3] = 1 << 20
    c.table.copy_(ints(c.table_host))
    faults = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.flame_kvq_extend(c.cfg, c.packed, q, off, ints(lens), dirty, ws, faults=faults)
    seen = np.ones(200, bool)
    seen[48:64] = False
    c.table_host[0, 3] = 0
    check_attention(host(dirty[:150]), host(q[:150]), *c.rows(0, 200), dtype, seen=seen)
    assert int(faults[0]) == 1 and torch.equal(dirty[150:], clean[150:])
    B.flame_kvq_decode(c.cfg, c.packed, last, ints([200, 90]), single, ws)
    check_attention(host(single[:1]), host(last[:1]), *c.rows(0, 200), dtype, seen=seen)


@pytest.mark.parametrize("form", FORMS)
def test_offsets_and_lengths_that_are_none(B, form):  # noqa: F811
    import torch
    gen = generator(8)
    c = Cache(B, gen, form, "bf16", 4, 2, 64, [60, 40, 20], 16)
    q = rand(gen, "bf16", 30, 4, 64)
    for off, lens, fault, good in (([0, 10, 5, 30], [60, 40, 20], 4, 1), ([0, 10, 20, 40], [60, 40, 20], 4, 2), ([-5, 10, 20, 30], [60, 40, 20], 4, 0), ([0, 10, 20, 30], [60, -3, 1 << 30], 2, 1)):
        for room in (c.table, ints(np.concatenate([c.table_host, np.full((3, 200), -7, np.int32)], 1))):
            cache = B.pack_kvq_cache(c.cfg, form, c.k, c.v, c.ks, c.vs, room)
            out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
            B.flame_kvq_extend(c.cfg, cache, q, ints(off), ints(lens), out, workspace_for(B, c.cfg, 3, 30), faults=faults)
            assert int(faults[0]) & fault
            for b in range(good):
                s = slice(off[b], off[b + 1])
                check_attention(host(out[s]), host(q[s]), *c.rows(b, lens[b]), "bf16", what=(off, b))


# ---------------------------------------------------------------------------------------------- shared histories
def shared_workspace(B, cfg, n_groups, n_seqs, n_tokens=None):  # noqa: F811
    import torch
    return torch.full((B.flame_kv_shared_workspace_bytes(cfg, n_groups, n_seqs, n_tokens),), 0xff, dtype=torch.uint8, device=DEV)


# groups of (shared tokens, [(tokens in all, new ones, where it leaves the history (None: at its end))])
SHARED = {
    "one": [(100, [(101, 1, None)] * 5)],
    "several": [(70, [(71, 1, None), (90, 1, None)]), (0, [(5, 1, None), (1, 1, None)]), (333, [(400, 1, None)]), (48, [(48 + i, 1, None) for i in range(1, 20)])],
    "pieces": [(200, [(240, 7, None), (201, 1, None), (260, 60, None)]), (33, [(40, 3, None)]), (64, [(200, 100, None), (64, 1, None)])],
    "within": [(150, [(40, 10, None), (150, 150, None), (0, 2, None), (10, 20, None), (160, 30, None)]), (20, [(3, 1, None), (90, 2, None)])],
    "forks": [(300, [(320, 2, None), (310, 5, 100), (120, 4, 0), (250, 1, 299)])],
    "long": [(2500, [(2500 + 7 * i, 1 + i % 3, None) for i in range(1, 12)]), (1100, [(1101, 1, None)])],
    "many": [(30 + g, [(31 + g + i, 1, None) for i in range(1 + g % 3)]) for g in range(90)],
}


def shared_case(B, gen, form, dtype, hq, hkv, dim, groups, page=16, tokens=0, seed=0, head_major=False):  # noqa: F811
    lens, new, prefix, lists, first = [], [], [], [], [0]
    for p, seqs in groups:
        lists.append(list(range(len(lens), len(lens) + len(seqs))))
        for i, (n, m, leaves) in enumerate(seqs):
            lens.append(n), new.append(m), prefix.append(p if leaves is None else leaves)
        first.append(len(lens))
    ps = [p for p, _ in groups]
    c = Cache(B, gen, form, dtype, hq, hkv, dim, lens, page, head_major, seed, tokens, lists, ps)
    # a sequence that leaves the history has pages of its own from there on
    extra = [(b, prefix[b] // page, -(-lens[b] // page)) for g, p in zip(lists, ps) for b in g if prefix[b] < p]
    taken = set(c.table_host[c.table_host >= 0].ravel().tolist())
    spare = [x for x in range(c.n_pages) if x not in taken]
    for b, lo, hi in extra:
        for i in range(lo, hi):
            if c.table_host[b, i] < 0:
                c.table_host[b, i] = spare[(b + i) % len(spare)]        # (pages may be any: they are read alone)
    c.table.copy_(ints(c.table_host))
    return c, lens, new, prefix, lists, first


def check_shared(B, c, q, out, lens, new, prefix, lists, dtype, single, every=1):  # noqa: F811
    off, pools = offsets([1] * len(lens) if single else new), c.pools()
    for g in lists:
        for b in g[::every]:
            s = slice(off[b], off[b + 1])
            if off[b + 1] > off[b]:
                check_attention(host(out[s]), host(q[s]), *c.rows(b, lens[b], prefix[b], g[0], pools), dtype, what=(b, lens[b], prefix[b]))


@pytest.mark.parametrize("form", [None, "f8", "f4"])
@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 64), ("bf16", 4, 4, 128), ("f16", 6, 2, 128), ("f16", 3, 3, 32), ("bf16", 32, 1, 32), ("f16", 4, 4, 64), ("f32", 4, 2, 64), ("f32", 2, 2, 128), ("f32", 3, 1, 32)])
@pytest.mark.parametrize("name", SHARED)
def test_shared(B, form, dtype, hq, hkv, dim, name):  # noqa: F811
    import torch
    gen = generator(dim)
    c, lens, new, prefix, lists, first = shared_case(B, gen, form, dtype, hq, hkv, dim, SHARED[name], tokens=4096 if name in ("long", "pieces") else 0, head_major=dim == 64)
    for single in (True, False):
        n = len(lens) if single else sum(new)
        q = rand(gen, dtype, n + (0 if single else 2), hq, dim)
        out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
        ws = shared_workspace(B, c.cfg, len(first) - 1, len(lens), len(q))
        call(B, c, "shared", q, None if single else ints(offsets(new)), ints(lens), ints(first), ints(prefix), out, ws, faults=faults)
        assert int(faults[0]) == 0 and bool((out[n:] == 7.0).all())
        check_shared(B, c, q, out, lens, new, prefix, lists, dtype, single, 7 if name == "many" else 1)
        again = torch.empty_like(out)
        call(B, c, "shared", q, None if single else ints(offsets(new)), ints(lens), ints(first), ints(prefix), again, ws.random_(0, 256))
        assert torch.equal(again[:n], out[:n])                          # the same call, the same bits


@pytest.mark.parametrize("form", [None, "f8"])
def test_shared_rows_do_not_feel_what_they_do_not_see(B, form):  # noqa: F811
    """NaN at a token of the history: rows before it, sequences that left before it and other groups keep their bits."""
    import torch
    gen = generator(11)
    c, lens, new, prefix, lists, first = shared_case(B, gen, form, "bf16", 4, 2, 64, [(120, [(130, 3, None), (125, 80, None), (140, 2, 60)]), (50, [(60, 2, None)])])
    q = rand(gen, "bf16", sum(new), 4, 64)
    clean, dirty = torch.empty_like(q), torch.empty_like(q)
    ws, off = shared_workspace(B, c.cfg, 2, 4, len(q)), offsets(new)
    call(B, c, "shared", q, ints(off), ints(lens), ints(first), ints(prefix), clean, ws)
    for at in (60, 100, 119):
        page, slot = c.table_host[0, at // 16], at % 16
        keep = (c.v if form is None else c.vs)[page, slot].clone()
        (c.v if form is None else c.vs)[page, slot, 1] = math.nan if form is None else 255
        call(B, c, "shared", q, ints(off), ints(lens), ints(first), ints(prefix), dirty, ws)
        (c.v if form is None else c.vs)[page, slot] = keep
        before = at - 45                                                # rows of the second sequence: positions 45..124
        assert bool(dirty[:3, 2:].isnan().all()) and torch.equal(dirty[:3, :2], clean[:3, :2])
        assert torch.equal(dirty[3:3 + before], clean[3:3 + before]) and bool(dirty[3 + before:83, 2:].isnan().all())
        assert torch.equal(dirty[83:], clean[83:])


def test_shared_reports_groups_that_are_none(B):  # noqa: F811
    """Wrong group offsets and shared lengths: faults, no access out of range, and sequences outside of every group see their own tokens alone."""
    import torch
    gen = generator(12)
    c, lens, new, prefix, lists, first = shared_case(B, gen, None, "bf16", 4, 2, 64, [(64, [(70, 1, None), (80, 1, None)]), (32, [(40, 1, None), (33, 1, None)])])
    q = rand(gen, "bf16", 4, 4, 64)
    pools = c.pools()

    def run(group_offsets, prefix_lens):
        out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
        call(B, c, "shared", q, None, ints(lens), ints(group_offsets), ints(prefix_lens), out, shared_workspace(B, c.cfg, 8, 4), faults=faults)
        return int(faults[0]), out

    def check(out, b, trunk, first_seq, own_from):
        k, v = c.rows(b, lens[b], trunk, first_seq, pools)
        seen = np.ones(lens[b], bool)
        seen[trunk:own_from] = False
        check_attention(host(out[b:b + 1]), host(q[b:b + 1]), k, v, "bf16", seen=seen, what=(b, trunk))

    fault, out = run([0, 2, 4], prefix)
    assert fault == 0
    for b in range(4):
        check(out, b, prefix[b], 0 if b < 2 else 2, prefix[b])
    for groups in ([0, 2], [0, 2, 3], [0, 2, 9], [2, 4], [-1, 2, 4], [0, 4, 2], [0]):
        fault, out = run(groups, prefix)
        assert fault & 4, groups
        for b in range(4):
            if groups[0] == 0 and len(groups) > 1 and groups[1] == 2 and b < 2:
                check(out, b, 64, 0, 64)
    fault, out = run([2, 4], prefix)
    check(out, 0, 0, 0, 64), check(out, 1, 0, 1, 64), check(out, 2, 32, 2, 32)
    fault, out = run([0, 2, 4], [64, 80, 32, 32])                       # the second says that it shares more than there is
    assert fault == 2
    check(out, 1, 64, 0, 80)
    fault, out = run([0, 2, 4], [64, -5, 32, 1 << 30])                  # (taken as sharing nothing, the second has no pages for its first tokens)
    assert fault == 3


# ---------------------------------------------------------------------------------------------- a run of them together
@pytest.mark.parametrize("form", FORMS)
def test_a_history_and_its_candidates(B, form):  # noqa: F811
    """A user's history appended in pieces and attended over, read back, then candidates behind it: each a sequence of one token that shares the history; the last piece captured into a
    graph that follows the device arrays, replayed with other work in between."""
    import torch
    gen = generator(21)
    dtype, hq, hkv, dim, page = "bf16", 4, 2, 64, 16
    cfg = B.make_kv_config(dtype, hq, hkv, dim)
    pool = B.make_kvq_pool(cfg, form, 40, page)
    table = np.full((9, 10), -7, np.int32)
    table[0, :7] = [5, 9, 2, 30, 11, 12, 13]
    for b in range(1, 9):
        table[b, 6] = 13 + b                                            # the page that holds its candidate; the history ends within it
    cache = B.pack_kvq_cache(cfg, form, *pool, ints(table))
    rotation = B.make_kv_rotation(B.flame_kv_rotation_frequencies(dim))
    rows = rand(gen, dtype, 100, hq + 2 * hkv, dim)
    ws = workspace_for(B, cfg, 1, 60)
    history = 0
    for m in (60, 1, 39):
        part = rows[history:history + m]
        history += m
        q, out = torch.empty(m, hq, dim, device=DEV, dtype=torch_type(dtype)), torch.empty(m, hq, dim, device=DEV, dtype=torch_type(dtype))
        B.flame_kvq_append(cfg, cache, part[:, hq:hq + hkv], part[:, hq + hkv:], ints([0, m]), ints([history]), q=part[:, :hq], q_out=q, rotation=rotation)
        B.flame_kvq_extend(cfg, cache, q, ints([0, m]), ints([history]), out, ws)
        k, v = (torch.empty(history, hkv, dim, device=DEV, dtype=torch_type(dtype)) for _ in range(2))
        B.flame_kvq_read(cfg, cache, ints([0, history]), ints([history]), k, v)
        check_attention(host(out), host(q), host(k), host(v), dtype, what=m)
    # eight candidates: positions 100, each in its own copy of the history's last page's place
    new = rand(gen, dtype, 8, hq + 2 * hkv, dim)
    cand = B.pack_kvq_cache(cfg, form, *pool, ints(table[1:]))
    lens = ints([101] * 8)
    q, out = torch.empty(8, hq, dim, device=DEV, dtype=torch_type(dtype)), torch.empty(9, hq, dim, device=DEV, dtype=torch_type(dtype))
    # the group's first sequence is the history itself, with a query of its own
    everyone = ints([100] + [101] * 8)
    group, prefix, wss = ints([0, 9]), ints([100] * 9), shared_workspace(B, cfg, 1, 9)
    off = ints(np.arange(9))

    def step():
        B.flame_kvq_append(cfg, cand, new[:, hq:hq + hkv], new[:, hq + hkv:], off, lens, q=new[:, :hq], q_out=q, rotation=rotation)
        B.flame_kvq_shared(cfg, cache, torch_cat[:9], None, everyone, group, prefix, out, wss)

    torch_cat = torch.zeros(9, hq, dim, device=DEV, dtype=torch_type(dtype))

    def check():
        values = [kv_oracle.stored_values(kv_oracle.unpack(p.cpu().numpy(), form), s.cpu().numpy(), form) for p, s in ((pool[0], pool[2]), (pool[1], pool[3]))]
        assert np.array_equal(values[0][table[0, np.arange(100) // page], np.arange(100) % page], host(k))
        for b in range(9):
            kk, vv = host(k), host(v)
            if b:
                kk, vv = (np.concatenate([x, y[table[b, 6], 4][None]]) for x, y in ((kk, values[0]), (vv, values[1])))
            check_attention(host(out[b:b + 1]), host(torch_cat[b:b + 1]), kk, vv, dtype, what=b)

    torch_cat.copy_(rand(gen, dtype, 9, hq, dim))
    step()
    check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        torch_cat.copy_(rand(gen, dtype, 9, hq, dim))
        new.copy_(rand(gen, dtype, 8, hq + 2 * hkv, dim))
        wss.fill_(255)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        check()
        eager = out.clone()
        step()
        assert torch.equal(eager, out)


@pytest.mark.parametrize("form", [None, "f8"])
def test_two_calls_at_once(B, form):  # noqa: F811
    """Two streams, a workspace each, over one cache: the bits of one call after the other."""
    import torch
    gen = generator(31)
    c, lens, new, prefix, lists, first = shared_case(B, gen, form, "bf16", 8, 2, 64, SHARED["long"], tokens=4096)
    qs = [rand(gen, "bf16", sum(new), 8, 64) for _ in range(2)]
    want = [torch.empty_like(qs[0]) for _ in range(2)]
    args = ints(offsets(new)), ints(lens), ints(first), ints(prefix)
    spaces = [shared_workspace(B, c.cfg, len(first) - 1, len(lens), sum(new)) for _ in range(2)]
    for q, o, ws in zip(qs, want, spaces):
        call(B, c, "shared", q, *args, o, ws)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [torch.zeros_like(qs[0]) for _ in range(2)]
        torch.cuda.synchronize()
        for q, o, ws, s in zip(qs, got, spaces, streams):
            call(B, c, "shared", q, *args, o, ws, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---------------------------------------------------------------------------------------------- what else the calls allow
@pytest.mark.parametrize("form", [None, "f8", "f4"])
@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 2, 1, 64), ("f16", 4, 4, 32), ("f32", 3, 1, 32)])
def test_shared_of_more_groups_than_lanes_over_long_histories(B, form, dtype, hq, hkv, dim):  # noqa: F811
    """Seventy groups whose histories are cut into parts (not of equal length: that takes a lane for each group)."""
    import torch
    gen = generator(70 + dim)
    groups = [(900 + 17 * g, [(901 + 17 * g + 3 * i, 1 + (g + i) % 2, None) for i in range(1 + g % 3)]) for g in range(70)]
    c, lens, new, prefix, lists, first = shared_case(B, gen, form, dtype, hq, hkv, dim, groups, page=64, tokens=4096)
    q = rand(gen, dtype, sum(new), hq, dim)
    out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = shared_workspace(B, c.cfg, 70, len(lens), sum(new))
    call(B, c, "shared", q, ints(offsets(new)), ints(lens), ints(first), ints(prefix), out, ws, faults=faults)
    assert int(faults[0]) == 0
    check_shared(B, c, q, out, lens, new, prefix, lists[::9] + lists[-1:], dtype, False)


@pytest.mark.parametrize("form", FORMS)
def test_pools_beyond_32_bits(B, form):  # noqa: F811
    """Pages that begin 3 GiB apart: append, read, extend, decode and shared attention."""
    import torch
    gen, page, far, dim = generator(41), 16, 3 << 30, 64
    row = dim if form == "f8" else dim // 2
    cfg = B.make_kv_config("bf16", 4, 2, dim)
    pools, scales = [torch.empty(2 * far + page * 2 * row, dtype=torch.uint8, device=DEV) for _ in range(2)], []
    unit = 32 if form == "f8" else 16
    views = [p.as_strided((3, page, 2, row), (far, 2 * row, row, 1)) for p in pools]
    for _ in range(2):
        s = torch.empty(2 * far // unit + page * 4, dtype=torch.uint8, device=DEV)
        scales.append(s.as_strided((3, page, 2, 2), (far // unit, 2 * row // unit, row // unit, 1)))
    cache = B.pack_kvq_cache(cfg, form, *views, *scales, ints([[2, 0, 1], [2, 1, 0]]))
    k, v, q = rand(gen, "bf16", 40, 2, dim), rand(gen, "bf16", 40, 2, dim), rand(gen, "bf16", 40, 4, dim)
    B.flame_kvq_append(cfg, cache, k, v, ints([0, 40]), ints([40]))
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    B.flame_kvq_read(cfg, cache, ints([0, 40]), ints([40]), rk, rv)
    assert np.array_equal(host(rk), kv_oracle.quantise(host(k), form, "bf16")[2]) and np.array_equal(host(rv), kv_oracle.quantise(host(v), form, "bf16")[2])
    out = torch.empty_like(q)
    B.flame_kvq_extend(cfg, cache, q, ints([0, 40]), ints([40]), out, workspace_for(B, cfg, 1, 40))
    check_attention(host(out), host(q), host(rk), host(rv), "bf16")
    single = torch.empty_like(q[:1])
    B.flame_kvq_decode(cfg, cache, q[:1], ints([40]), single, workspace_for(B, cfg, 1))
    check_attention(host(single), host(q[:1]), host(rk), host(rv), "bf16")
    two = torch.empty_like(q[:2])                                       # the second leaves the first one's page 2 for page 1, which holds tokens 32..39
    B.flame_kvq_shared(cfg, cache, q[:2], None, ints([40, 24]), ints([0, 2]), ints([16, 16]), two, shared_workspace(B, cfg, 1, 2))
    check_attention(host(two[:1]), host(q[:1]), host(rk), host(rv), "bf16")
    rows = list(range(16)) + list(range(32, 40))
    check_attention(host(two[1:]), host(q[1:2]), host(rk)[rows], host(rv)[rows], "bf16")


@pytest.mark.parametrize("form", [None, "f8"])
@pytest.mark.parametrize("n_seqs", [5, 90])
def test_padded_batches_and_wrong_offsets(B, form, n_seqs):  # noqa: F811
    """Rows ahead of the first sequence and behind the last are left as they are; offsets that are none make no access out of range and are reported, and of up to 64 sequences those before them
    have their results, by every call."""
    import torch
    gen = generator(n_seqs)
    groups = [(70, [(71 + i, 1 + i % 3, None) for i in range(2)]), (40, [(45 + i, 2, None) for i in range(n_seqs - 2)])]
    c, lens, new, prefix, lists, first = shared_case(B, gen, form, "bf16", 4, 2, 64, groups, tokens=2048)
    off = 3 + offsets(new)
    n = int(off[-1]) + 4
    q = rand(gen, "bf16", n, 4, 64)
    pools = c.pools()

    def run(off):
        out, faults = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device=DEV)
        call(B, c, "shared", q, ints(off), ints(lens), ints(first), ints(prefix), out, shared_workspace(B, c.cfg, 2, n_seqs, n), faults=faults)
        return out, int(faults[0])

    def check(out, off, b):
        s = slice(off[b], off[b + 1])
        check_attention(host(out[s]), host(q[s]), *c.rows(b, lens[b], prefix[b], 0 if b < 2 else 2, pools), "bf16", what=b)

    out, fault = run(off)
    assert fault == 0 and bool((out[:3] == 7.0).all()) and bool((out[-4:] == 7.0).all())
    for b in (0, 1, 2, n_seqs - 1):
        check(out, off, b)
    for at, value in ((3, 4), (3, -1), (n_seqs, 1 << 30), (1, -(1 << 31)), (n_seqs, -7), (0, -2), (2, 1 << 30)):
        wrong = off.copy()
        wrong[at] = value
        out, fault = run(wrong)
        assert fault & 4, (at, value)
        if n_seqs <= 64:
            bad = next((b for b in range(n_seqs) if wrong[b] < 0 or wrong[b + 1] < wrong[b]), n_seqs)
            for b in range(bad):
                if wrong[b + 1] <= n:
                    check(out, wrong, b) if wrong[b + 1] - wrong[b] == new[b] else None
            after = int(max(wrong[:bad + 1].max(), 0)) if bad else 0
            assert bool((out[after:] == 7.0).all()), (at, value)
    if form == "f8":
        rk, rv = (torch.full((n, 2, 64), 7.0, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        B.flame_kvq_read(c.cfg, c.packed, ints(off), ints(np.minimum(lens, 16)), rk, rv)
        assert bool((rk[:3] == 7.0).all()) and bool((rk[-4:] == 7.0).all())
        for b in (0, 2):                                                # (of groups' first sequences the rows of the table name the first tokens too)
            page = c.table_host[b, 0]
            t = np.arange(min(lens[b], 16) - new[b], min(lens[b], 16))
            assert np.array_equal(host(rk)[off[b]:off[b + 1]], pools[0][page, t])


def test_append_far_positions(B):  # noqa: F811
    """A cache that spans 2^31 - 2^16 positions over a few pages: keys and queries there, by the same angles as in the cache of the element type."""
    import torch
    gen, page, width = generator(51), 65536, 32767
    cfg = B.make_kv_config("f32", 2, 1, 64)
    pool = B.make_kvq_pool(cfg, "f8", 2, page)
    cache = B.pack_kvq_cache(cfg, "f8", *pool, torch.ones(2, width, dtype=torch.int32, device=DEV))
    lens = np.array([page * width, (1 << 30) + 12345], np.int64)
    q, k = rand(gen, "f32", 4, 2, 64), rand(gen, "f32", 4, 1, 64)
    f = B.flame_kv_rotation_frequencies(64)
    out = torch.empty_like(q)
    B.flame_kvq_append(cfg, cache, k, k, ints([0, 2, 4]), ints(lens), q=q, q_out=out, rotation=B.make_kv_rotation(f))
    plain = B.pack_kv_cache(cfg, torch.zeros(2, page, 1, 64, device=DEV), torch.zeros(2, page, 1, 64, device=DEV), torch.ones(2, width, dtype=torch.int32, device=DEV))
    want = torch.empty_like(q)
    B.flame_kv_append(cfg, plain, k, k, ints([0, 2, 4]), ints(lens), q=q, q_out=want, rotation=B.make_kv_rotation(f))
    position = np.concatenate([[x - 2, x - 1] for x in lens])
    turned = kv_oracle.rotate(host(q), position, f, False)
    assert np.abs(host(out) - turned).max() <= 2.0 ** -24 * np.abs(turned).max() + 2 * np.abs(host(q)).max() * 2.0 ** -21
    assert np.abs(host(out) - host(want)).max() <= 2 * (2.0 ** -24 * np.abs(turned).max() + 2 * np.abs(host(q)).max() * 2.0 ** -21)
    back_k, back_v = torch.empty_like(k), torch.empty_like(k)
    B.flame_kvq_read(cfg, cache, ints([0, 2, 4]), ints(lens), back_k, back_v)
    assert np.array_equal(host(back_v), kv_oracle.quantise(host(k), "f8", "f32")[2])
    key = kv_oracle.rotate(host(k), position, f, False)
    assert (np.abs(host(back_k) - key) <= 2.0 ** -4 * np.abs(key) + 2.0 ** -9 * np.abs(key).max() / 464 + 2 * np.abs(host(k)).max() * 2.0 ** -21 * (1 + 2.0 ** -4)).all()


def test_two_graphs_with_one_workspace(B):  # noqa: F811
    """Graphs of a shared and of a decoding call that use the same workspace, replayed in turn with eager calls between them, lengths changing on the device."""
    import torch
    gen = generator(61)
    c, lens, new, prefix, lists, first = shared_case(B, gen, "f8", "bf16", 8, 2, 64, [(1500, [(1501 + 9 * i, 1, None) for i in range(6)])], tokens=2048)
    q, one = rand(gen, "bf16", 6, 8, 64), rand(gen, "bf16", 1, 8, 64)
    ws = shared_workspace(B, c.cfg, 1, 6)
    assert ws.numel() >= B.flame_kv_workspace_bytes(c.cfg, 1)
    lens_t, first_t, prefix_t = ints(lens), ints(first), ints(prefix)
    out, single = torch.empty_like(q), torch.empty_like(one)

    def both():
        call(B, c, "shared", q, None, lens_t, first_t, prefix_t, out, ws)

    def decode():
        B.flame_kvq_decode(c.cfg, c.packed, one, lens_t[:1], single, ws)

    both(), decode()
    graphs = []
    for f in (both, decode):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    for i in range(4):
        now = [n - 5 * i for n in lens]
        lens_t.copy_(ints(now))
        prefix_t.copy_(ints([max(0, p - 300 * i) if b else p for b, p in enumerate(prefix)]))
        q.copy_(rand(gen, "bf16", 6, 8, 64)), one.copy_(rand(gen, "bf16", 1, 8, 64))
        graphs[0].replay(), graphs[1].replay()
        torch.cuda.synchronize()
        got, alone = out.clone(), single.clone()
        ws.fill_(255), out.zero_(), single.zero_()
        both(), decode()
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(single, alone)
        pools = c.pools()
        check_attention(host(alone), host(one), *c.rows(0, now[0], pools=pools), "bf16", what=i)
        if i == 0:
            for b in range(6):
                check_attention(host(got[b:b + 1]), host(q[b:b + 1]), *c.rows(b, now[b], prefix[b], 0, pools), "bf16", what=(i, b))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("shared", [False, True])
def test_few_rows_do_not_feel_what_they_do_not_see(B, form, dtype, dim, shared):  # noqa: F811
    """A few new rows over a cache with room for many tokens (split over the keys): a NaN block among the newest tokens is seen by the rows from its token on, in its 32 features of the values."""
    import torch
    gen = generator(5 + dim)
    lens, new = [200, 90, 12], [11, 3, 12]
    c = Cache(B, gen, form, dtype, 4, 2, dim, lens, 16, tokens=4096)
    off = ints(offsets(new))
    q = rand(gen, dtype, 26, 4, dim)
    clean, dirty = torch.empty_like(q), torch.empty_like(q)

    def run(out):
        if shared:
            B.flame_kvq_shared(c.cfg, c.packed, q, off, ints(lens), ints([0, 1, 2, 3]), ints([150, 40, 0]), out, shared_workspace(B, c.cfg, 3, 3, 26))
        else:
            B.flame_kvq_extend(c.cfg, c.packed, q, off, ints(lens), out, workspace_for(B, c.cfg, 3, 26))

    run(clean)
    pools = c.pools()
    for b, (n, m) in enumerate(zip(lens, new)):
        s = slice(sum(new[:b]), sum(new[:b + 1]))
        check_attention(host(clean[s]), host(q[s]), *c.rows(b, n, pools=pools), dtype, what=b)
    for at in (189, 190, 195, 199):
        page, slot, row = c.table_host[0, at // 16], at % 16, at - 189
        for block in range(dim // 32):
            for scales, where in ((c.vs, "v"), (c.ks, "k")):
                was = int(scales[page, slot, 1, block])
                scales[page, slot, 1, block] = 255
                run(dirty)
                scales[page, slot, 1, block] = was
                assert torch.equal(dirty[:row], clean[:row]) and torch.equal(dirty[11:], clean[11:]) and torch.equal(dirty[:, :2], clean[:, :2]), (at, where)
                mine = slice(32 * block, 32 * block + 32) if where == "v" else slice(0, dim)
                assert bool(dirty[row:11, 2:, mine].isnan().all())
                others = [i for i in range(dim) if not mine.start <= i < mine.stop]
                assert torch.equal(dirty[:, :, others], clean[:, :, others])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hq,hkv,dim", [(8, 2, 64), (4, 1, 32), (32, 8, 128)])
def test_batches_padded_with_sequences(B, form, hq, hkv, dim):  # noqa: F811
    """A batch held ready for 400 sequences of which 150 are there, with empty ones among them and rows behind the last: append, read, decode and shared attention do what they do for those alone."""
    import torch
    gen = generator(dim + 1)
    new = [(1, 0, 2, 1, 0)[i % 5] for i in range(150)] + [0] * 250
    lens = [m + i % 23 for i, m in enumerate(new[:150])] + [0] * 250
    c = Cache(B, gen, form, "bf16", hq, hkv, dim, lens, 16)
    n, off = sum(new), offsets(new)
    rows = rand(gen, "bf16", n + 70, hq + 2 * hkv, dim)
    q_out = torch.full((n + 70, hq, dim), 7.0, device=DEV, dtype=torch.bfloat16)
    faults = torch.zeros(1, dtype=torch.int32, device=DEV)
    rotation = B.make_kv_rotation(B.flame_kv_rotation_frequencies(dim))
    B.flame_kvq_append(c.cfg, c.packed, rows[:, hq:hq + hkv], rows[:, hq + hkv:], ints(off), ints(lens), q=rows[:, :hq], q_out=q_out, rotation=rotation, faults=faults)
    rk, rv = (torch.full((n + 70, hkv, dim), 7.0, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    B.flame_kvq_read(c.cfg, c.packed, ints(off), ints(lens), rk, rv, faults=faults)
    assert int(faults[0]) == 0 and bool((q_out[n:] == 7.0).all()) and bool((rk[n:] == 7.0).all())
    pools = c.pools()
    seq = np.repeat(np.arange(400), new)
    position = np.concatenate([np.arange(a - m, a) for a, m in zip(lens, new)])
    where = c.table_host[seq, position // 16], position % 16
    assert np.array_equal(host(rv)[:n], kv_oracle.quantise(host(rows[:n, hq + hkv:]), form, "bf16")[2]) and np.array_equal(pools[1][where], host(rv)[:n])
    assert np.array_equal(pools[0][where], host(rk)[:n])
    turned = kv_oracle.rotate(host(rows[:n, :hq]), position, B.flame_kv_rotation_frequencies(dim), False)
    assert np.abs(host(q_out)[:n] - turned).max() <= 2.0 ** -8 * np.abs(turned).max() + 2.0 ** -19 * np.abs(host(rows)).max()
    # single tokens of all 400, and the same in groups
    q = rand(gen, "bf16", 400, hq, dim)
    out, shared = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    B.flame_kvq_decode(c.cfg, c.packed, q, ints(lens), out, workspace_for(B, c.cfg, 400), faults=faults)
    first = list(range(0, 401, 8)) + [400] * 30
    B.flame_kvq_shared(c.cfg, c.packed, q, None, ints(lens), ints(first), ints([0] * 400), shared, shared_workspace(B, c.cfg, len(first) - 1, 400), faults=faults)
    assert int(faults[0]) == 0 and not out[150:].any() and not shared[150:].any()
    for b in range(0, 150, 11):
        check_attention(host(out[b:b + 1]), host(q[b:b + 1]), *c.rows(b, lens[b], pools=pools), "bf16", what=b)
        check_attention(host(shared[b:b + 1]), host(q[b:b + 1]), *c.rows(b, lens[b], pools=pools), "bf16", what=b)


@pytest.mark.parametrize("form", [None, "f8", "f4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_shared_rows_without_a_logit_above_minus_infinity(B, form, dtype, dim):  # noqa: F811
    """Every logit is -infinity: zeros whatever the values hold, over the history and over own tokens, few (one part) and many (several); codes, of which none is infinite, take the
    infinity from the queries."""
    import torch
    gen = generator(dim)
    groups = [(600, [(601, 1, None), (604, 3, None), (2100, 2, None), (600, 40, None)]), (0, [(9, 1, None), (900, 5, None)])]
    for tokens in (0, 4096):
        c, lens, new, prefix, lists, first = shared_case(B, gen, form, dtype, 4, 2, dim, groups, tokens=tokens)
        if form is None:
            c.k[..., 0] = -math.inf
            c.v[..., 3], c.v[..., 4], c.v[..., dim - 1] = math.inf, math.nan, -math.inf
        else:
            c.k[..., 0] = 0xb8 if form == "f8" else c.k[..., 0] & 0xf0 | 0x0a       # -1
            c.vs[..., 0] = 255
        for single in (True, False):
            q = torch.zeros(len(lens) if single else sum(new), 4, dim, device=DEV, dtype=torch_type(dtype))
            q[..., 0] = 1.0 if form is None else math.inf
            out = torch.full_like(q, 7.0)
            call(B, c, "shared", q, None if single else ints(offsets(new)), ints(lens), ints(first), ints(prefix), out, shared_workspace(B, c.cfg, len(first) - 1, len(lens), len(q)))
            assert not bool(out.any()), (tokens, single, [b for b, x in enumerate(out.flatten(1).any(1).tolist()) if x])


MANY_ROWS = [("f8", "bf16", 2, 1, 32, 32, 130, 2101, 1), ("f4", "f16", 6, 3, 32, 0, 70, 4203, 3), ("f8", "f32", 3, 3, 64, 0, 200, 8301, 2), ("f4", "bf16", 5, 5, 32, 16, 300, 70001, 1),
             ("f8", "f16", 4, 1, 32, 0, 1000, 140001, 3), ("f4", "f32", 1, 1, 32, 0, 129, 66001, 0), ("f8", "bf16", 1, 1, 32, 0, 64, 270001, 2), ("f8", "f32", 8, 2, 128, 64, 17, 20003, 5)]


@pytest.mark.parametrize("form,dtype,hq,hkv,dim,rot,n_seqs,n,ahead", MANY_ROWS)
def test_append_and_read_of_many_rows(B, form, dtype, hq, hkv, dim, rot, n_seqs, n, ahead):  # noqa: F811
    """Batches large enough that a wavefront takes several tokens (append up to four, read up to 64) and that rows go past the caches (from 16 MB): ragged sequences, runs of more empty ones than
    lanes, rows ahead of the first and behind the last, and tokens below position 0, whose queries are not written."""
    import torch
    gen, rng = generator(n), np.random.default_rng(n)
    share = rng.exponential(1.0, n_seqs)
    share[rng.random(n_seqs) < 0.2] = 0
    if n_seqs > 128:
        share[10:90] = 0
    share[[0, -1]] = 0, 1.0
    new = np.floor(share / share.sum() * (n - 10)).astype(np.int64)
    new[1] += n - int(new.sum())
    before = rng.integers(0, 20, n_seqs)
    before[1] = -7                                                      # seven of its new tokens are at positions below 0
    lens = new + before
    off, page = offsets(new) + ahead, 16
    used = -(-lens // page)
    order = rng.permutation(int(used.sum()) + 2)
    table = np.full((n_seqs, int(used.max())), -7, np.int32)
    for b, first in enumerate(np.cumsum(used) - used):
        table[b, :used[b]] = order[first:first + used[b]]
    cfg = B.make_kv_config(dtype, hq, hkv, dim)
    pool = B.make_kvq_pool(cfg, form, len(order), page)
    cache = B.pack_kvq_cache(cfg, form, *pool, ints(table))
    rows = rand(gen, dtype, ahead + n + 3, hq + 2 * hkv, dim)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    q_out, faults = torch.full((len(rows), hq, dim), 7.0, device=DEV, dtype=torch_type(dtype)), torch.zeros(2, dtype=torch.int32, device=DEV)
    f = B.flame_kv_rotation_frequencies(rot) if rot else np.zeros(0)
    B.flame_kvq_append(cfg, cache, k, v, ints(off), ints(lens), q=q, q_out=q_out, rotation=B.make_kv_rotation(f) if rot else None, faults=faults[:1])
    seq = np.repeat(np.arange(n_seqs), new)
    position = np.arange(n) + ahead - off[seq + 1] + lens[seq]
    there = position >= 0
    assert int(faults[0]) == 2 and int((~there).sum()) == 7
    row = np.flatnonzero(there) + ahead
    page_of, slot = table[seq[there], position[there] // page], position[there] % page
    empty = np.ones((len(order), page), bool)
    empty[page_of, slot] = False
    held = []
    for data, codes_t, scales_t in ((k, pool[0], pool[2]), (v, pool[1], pool[3])):
        got, got_scales = kv_oracle.unpack(codes_t.cpu().numpy(), form)[page_of, slot], scales_t.cpu().numpy()[page_of, slot]
        x = host(data)[row]
        held.append(kv_oracle.stored_values(got, got_scales, form))
        if data is v or not rot:
            codes, scales, _ = kv_oracle.quantise(x, form, dtype)
            assert np.array_equal(got, codes) and np.array_equal(got_scales, scales)
        else:
            relative, least, limit = HALF[form]
            turned, pair = kv_oracle.rotate(x, position[there], f, False), np.abs(x).max(-1, keepdims=True) * 2 * 2.0 ** -21
            scale = np.repeat((np.abs(turned).reshape(*turned.shape[:-1], -1, 32).max(-1) + pair) * 2 / limit, 32, -1)
            assert (np.abs(held[-1] - turned) <= pair * (1 + relative) + np.maximum(relative * np.abs(turned), least * scale)).all()
        assert not codes_t.cpu().numpy()[empty].any() and not scales_t.cpu().numpy()[empty].any()
    want = kv_oracle.rotate(host(q)[row], position[there], f, False)
    wide = np.abs(host(q)[row]).max(-1, keepdims=True) * 2
    assert (np.abs(host(q_out)[row] - want) <= HALF_STEP[dtype] * np.abs(want) + (wide * 2.0 ** -21 + (2.0 ** -25 if dtype == "f16" else 0) if rot else 0)).all() if rot else np.array_equal(host(q_out)[row], host(q)[row])
    others = np.ones(len(rows), bool)
    others[row] = False
    others = torch.tensor(others, device=DEV)
    assert bool((q_out[others] == 7.0).all()), torch.argwhere(others & (q_out != 7.0).flatten(1).any(1)).flatten()[:10].tolist()
    back = [torch.full((len(rows), hkv, dim), 7.0, device=DEV, dtype=torch_type(dtype)) for _ in range(2)]
    B.flame_kvq_read(cfg, cache, ints(off), ints(lens), *back, faults=faults[1:])
    assert int(faults[1]) == 2
    for x, values in zip(back, held):
        assert np.array_equal(host(x)[row], values) and bool((x[others] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_values_below_the_normal_range(B, form, dtype):  # noqa: F811
    """Blocks of subnormal values, alone and beside larger ones: rounded as all others, codes and scales bit for bit."""
    import torch
    tiny = np.concatenate([np.arange(0, 160) * 2.0 ** -133, [2.0 ** -127, 2.0 ** -126, 1.5 * 2.0 ** -127, 2.0 ** -125]])
    tiny = np.concatenate([tiny, -tiny])
    rng = np.random.default_rng(3)
    x = rng.choice(tiny, (64, 1, 128))
    x[32:, :, ::32] = 2.0 ** rng.integers(-126, -115, (32, 1, 4))
    x = torch.tensor(x).to(torch_type(dtype)).to(DEV)
    n = len(x)
    cfg = B.make_kv_config(dtype, 1, 1, 128)
    pool = B.make_kvq_pool(cfg, form, 1, n)
    cache = B.pack_kvq_cache(cfg, form, *pool, ints([[0]]))
    B.flame_kvq_append(cfg, cache, x, x, ints([0, n]), ints([n]))
    back, back_v = torch.empty_like(x), torch.empty_like(x)
    B.flame_kvq_read(cfg, cache, ints([0, n]), ints([n]), back, back_v)
    codes, scales, values = kv_oracle.quantise(host(x), form, dtype)
    got = kv_oracle.unpack(pool[0][0].cpu().numpy(), form)
    assert np.array_equal(pool[2][0].cpu().numpy(), scales)
    assert np.array_equal(got, codes) and np.array_equal(host(back), values) and np.array_equal(host(back_v), values)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_nan_values_of_keys_whose_logits_are_minus_infinity(B, dtype, dim):  # noqa: F811
    """Keys 0..699 have logits of -infinity, and one of them a value that is NaN: rows with a logit above that are NaN in its feature, by every call however the keys are cut, and those without one are zeros."""
    import torch

    from test_gpu_kv import spread
    gen, n, at = generator(dim), 1500, 10
    cfg = B.make_kv_config(dtype, 8, 2, dim)
    k, v = rand(gen, dtype, 4096, 2, dim), rand(gen, dtype, 4096, 2, dim)
    k[:700, :, 0] = -math.inf
    v[at, :, 3] = math.nan

    def check(out, positions, what):
        seen, nothing = torch.tensor(positions >= 700, device=DEV), torch.tensor(positions < 700, device=DEV)
        assert bool(out[seen][..., 3].isnan().all()) and bool(out[seen][..., 4:].isfinite().all()) and not bool(out[nothing].any()), what

    def queries(tokens):
        q = rand(gen, dtype, tokens, 8, dim)
        q[..., 0] = 1.0
        return q

    for size in (0, 1, 2):
        q = queries(n)
        out = torch.full_like(q, 7.0)
        B.flame_kv_prompt(cfg, q, k[:n], v[:n], ints(offsets([n] + spread(size, dtype, 2))), out)
        check(out, np.arange(n), ("prompt", size))
    for seqs, new, pages in ((1, 100, 256), (8, 300, 256), (8, 3, 256), (8, 1, 256), (2, 900, 100), (1, 900, 256), (1, 20, 256), (2, 40, 94)):
        cache = B.pack_kv_cache(cfg, k.reshape(256, 16, 2, dim), v.reshape(256, 16, 2, dim), ints(np.tile(np.arange(pages), (seqs, 1))))
        q, lens = queries(seqs * new), ints([n] * seqs)
        positions = np.tile(np.arange(n - new, n), seqs)
        out = torch.full_like(q, 7.0)
        B.flame_kv_extend(cfg, cache, q, ints(offsets([new] * seqs)), lens, out, workspace_for(B, cfg, seqs, seqs * new))
        check(out, positions, ("extend", seqs, new))
        if new == 1:
            out.fill_(7.0)
            B.flame_kv_decode(cfg, cache, q, lens, out, workspace_for(B, cfg, seqs))
            check(out, positions, "decode")
        for prefix in (0, 690, 1000, 1300):
            out.fill_(7.0)
            B.flame_kv_shared(cfg, cache, q, ints(offsets([new] * seqs)), lens, ints([0, seqs]), ints([prefix] * seqs), out, shared_workspace(B, cfg, 1, seqs, len(q)))
            check(out, positions, ("shared", seqs, new, pages, prefix))
