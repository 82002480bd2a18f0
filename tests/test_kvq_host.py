"""The cache of 8 or 4 bits and shared histories without a GPU: exported symbols, refusals of the C entries and of the binding, and the oracle of the codes against closed forms."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from oracle import kv_oracle
from paper_2509_22681_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_the_header():
    with open(os.path.join(ROOT, "include", "flame_kvq.h")) as f:
        declared = set(re.findall(r"^int\s*(flame_kvq_[a-z_]+)\(", f.read(), re.M))
    assert declared == set(B.KVQ_EXPORTS)
    for name in declared:
        assert hasattr(B._lib, name), name


# Arguments that pass every check, with addresses that nothing reads: only refused calls are made here.
A = 1 << 20


def call(op, **change):
    d = dict(dtype=1, hq=8, hkv=2, dim=64, scale=0.0, row_stride=512, head_stride=64, data=A, n_seqs=3, n_tokens=10, pool=A, form=1, scales=A, head=64, slot=128, page=2048, n_pages=4, page_size=16,
             table=A, pages_per_seq=8, offsets=A, kv_lens=A, workspace=A, bytes=1 << 62, rot_dim=64, frequencies=np.ones(64), q=True, n_groups=2, groups=A, prefix=A)
    d.update(change)
    cfg = None if d.get("cfg", 1) is None else C.byref(B.flame_kv_config(d["dtype"], d["hq"], d["hkv"], d["dim"], d["scale"]))
    rows = C.byref(B.flame_kv_rows(d["data"], d["row_stride"], d["head_stride"])) if d.get("rows", 1) else None
    where = d["n_pages"], d["page_size"], d["table"], 8, d["pages_per_seq"]
    cache = C.byref(B.flame_kvq_cache(d["form"], d["pool"], d["pool"], d["scales"], d["scales"], d["page"], d["slot"], d["head"], *where)) if d.get("cache", 1) else None
    plain = C.byref(B.flame_kv_cache(d["pool"], d["pool"], d["page"], d["slot"], d["head"], *where)) if d.get("cache", 1) else None
    f = d["frequencies"]
    rot = C.byref(B.flame_kv_rotation(d["rot_dim"], 0, None if f is None else f.ctypes.data_as(C.POINTER(C.c_double))))
    groups = C.byref(B.flame_kv_groups(d["groups"], d["prefix"], d["n_groups"])) if d.get("group", 1) else None
    n_seqs, n_tokens, off, lens = d["n_seqs"], d["n_tokens"], d["offsets"], d["kv_lens"]
    if op == "append":
        return B._lib.flame_kvq_append(cfg, cache, rows, rows, rows, rows if d["q"] else None, rot, off, lens, n_seqs, n_tokens, None, None)
    if op == "read":
        return B._lib.flame_kvq_read(cfg, cache, off, lens, n_seqs, n_tokens, rows, rows, None, None)
    if op == "extend":
        return B._lib.flame_kvq_extend(cfg, cache, rows, off, lens, n_seqs, n_tokens, rows, d["workspace"], d["bytes"], None, None)
    if op == "decode":
        return B._lib.flame_kvq_decode(cfg, cache, rows, lens, n_seqs, rows, d["workspace"], d["bytes"], None, None)
    if op == "shared_q":
        return B._lib.flame_kvq_shared(cfg, cache, rows, off, lens, groups, n_seqs, n_tokens, rows, d["workspace"], d["bytes"], None, None)
    return B._lib.flame_kv_shared(cfg, plain, rows, off, lens, groups, n_seqs, n_tokens, rows, d["workspace"], d["bytes"], None, None)


QUANTISED = ("append", "read", "extend", "decode", "shared_q")
ALL = QUANTISED + ("shared",)
SHARED = ("shared_q", "shared")
INVALID, CAPACITY, UNSUPPORTED = -1, -2, -5
REFUSED = [(ALL, dict(cfg=None), INVALID), (ALL, dict(dtype=3), INVALID), (ALL, dict(hq=7), INVALID), (ALL, dict(dim=48), UNSUPPORTED), (ALL, dict(dim=256), UNSUPPORTED), (ALL, dict(hq=8192), UNSUPPORTED),
           (ALL, dict(scale=-1.0), INVALID), (ALL, dict(n_seqs=-1), INVALID), (ALL, dict(rows=0), INVALID), (ALL, dict(data=None), INVALID), (ALL, dict(data=A + 8), INVALID),
           (ALL, dict(row_stride=516), INVALID), (ALL, dict(kv_lens=None), INVALID), (ALL, dict(cache=0), INVALID), (ALL, dict(pool=None), INVALID), (ALL, dict(pool=A + 8), INVALID),
           (QUANTISED, dict(scales=None), INVALID), (QUANTISED, dict(scales=A + 2), INVALID), (QUANTISED, dict(form=0), INVALID), (QUANTISED, dict(form=3), INVALID),
           (QUANTISED, dict(slot=96), INVALID), (QUANTISED, dict(head=32), INVALID), (QUANTISED, dict(page=2000), INVALID), (QUANTISED, dict(page=-2048), INVALID),
           (QUANTISED, dict(form=2, slot=48), INVALID), (ALL, dict(n_pages=0), INVALID), (ALL, dict(page_size=0), INVALID), (ALL, dict(page_size=65537), INVALID),
           (ALL, dict(pages_per_seq=0), INVALID), (ALL, dict(pages_per_seq=1 << 28), INVALID), (ALL, dict(table=None), INVALID),
           (("append", "read", "extend", "shared", "shared_q"), dict(n_tokens=-1), INVALID), (("append", "read", "extend", "shared", "shared_q"), dict(n_tokens=1 << 23), INVALID),
           (("append", "read", "extend", "shared", "shared_q"), dict(n_tokens=1 << 61), INVALID), (("append", "read", "extend"), dict(offsets=None), INVALID),
           (SHARED, dict(offsets=None), INVALID),                       # ten rows of three sequences
           (SHARED, dict(hq=1, hkv=1, n_tokens=1 << 24), INVALID), (SHARED, dict(group=0), INVALID), (SHARED, dict(n_groups=-1), INVALID), (SHARED, dict(n_groups=1 << 21), INVALID), (SHARED, dict(groups=None), INVALID), (SHARED, dict(prefix=None), INVALID),
           (("append",), dict(rot_dim=8), INVALID), (("append",), dict(rot_dim=80), INVALID), (("append",), dict(frequencies=None), INVALID), (("append",), dict(q=False), INVALID)]


@pytest.mark.parametrize("ops,change,code", REFUSED)
def test_refusals_of_the_c_entries(ops, change, code):
    for op in ops:
        assert call(op, **change) == code, (op, change)
        assert B._lib.flame_kv_last_error(), (op, change)


def test_a_workspace_that_is_too_small_is_refused():
    cfg = B.make_kv_config("bf16", 8, 2, 64)
    for op, need in (("extend", B.flame_kv_workspace_bytes(cfg, 1, 1)), ("decode", B.flame_kv_workspace_bytes(cfg, 1, 1)), ("shared", B.flame_kv_shared_workspace_bytes(cfg, 2, 3, 10)),
                     ("shared_q", B.flame_kv_shared_workspace_bytes(cfg, 2, 3, 10))):
        if need > 0:
            assert call(op, workspace=None) == INVALID and call(op, workspace=A + 4) == INVALID and call(op, bytes=need // 64) == CAPACITY, op
        assert call(op, bytes=-1) == CAPACITY, op


def test_empty_calls_enqueue_nothing():
    for op in ALL:
        assert call(op, n_seqs=0, rows=0, cache=0) == 0, op
    for op in ("append", "read", "extend") + SHARED:
        assert call(op, n_tokens=0, rows=0, cache=0) == 0, op


def test_workspace_refusals():
    cfg = B.make_kv_config("bf16", 8, 2, 64)
    for bad in (lambda: B.flame_kv_shared_workspace_bytes(B.make_kv_config("bf16", 8, 3, 64), 1, 1), lambda: B.flame_kv_shared_workspace_bytes(cfg, -1, 1),
                lambda: B.flame_kv_shared_workspace_bytes(cfg, 1, -1), lambda: B.flame_kv_shared_workspace_bytes(cfg, 1, 1, -1), lambda: B.flame_kv_shared_workspace_bytes(cfg, 1, 1, 1 << 61)):
        with pytest.raises(B.FlameGRError) as e:
            bad()
        assert e.value.code == INVALID
    assert B.flame_kv_shared_workspace_bytes(cfg, 0, 0) >= 0
    sizes = [[B.flame_kv_shared_workspace_bytes(cfg, g, s, t) for s, t in ((1, 1), (5, 40), (64, 64), (64, 4096), (500, 5000))] for g in (0, 1, 8, 100)]
    assert all(a <= b for row in sizes for a, b in zip(row, row[1:])) and all(a <= b for u, v in zip(sizes, sizes[1:]) for a, b in zip(u, v))


def test_refusals_of_the_binding():
    cfg = B.make_kv_config("bf16", 8, 2, 64)
    pool, scales, table = torch.zeros(4, 16, 2, 64, dtype=torch.uint8), torch.zeros(4, 16, 2, 2, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.int32)
    half = torch.zeros(4, 16, 2, 32, dtype=torch.uint8)
    for bad in (lambda: B.pack_kvq_cache(cfg, "f7", pool, pool, scales, scales, table), lambda: B.pack_kvq_cache(cfg, "f8", half, half, scales, scales, table),
                lambda: B.pack_kvq_cache(cfg, "f4", pool, pool, scales, scales, table), lambda: B.pack_kvq_cache(cfg, "f8", pool.char(), pool.char(), scales, scales, table),
                lambda: B.pack_kvq_cache(cfg, "f8", pool, pool[:3], scales, scales, table), lambda: B.pack_kvq_cache(cfg, "f8", pool, pool, scales[..., :1], scales, table),
                lambda: B.pack_kvq_cache(cfg, "f8", pool, pool, scales, scales.float(), table), lambda: B.pack_kvq_cache(cfg, "f8", pool, pool, scales, scales, table.long()),
                lambda: B.pack_kvq_cache(cfg, "f8", pool, pool, scales, scales, table[0]), lambda: B.pack_kvq_cache(cfg, "f8", pool, pool, scales, scales, table),   # (host memory)
                lambda: B.pack_kvq_cache(B.make_kv_config(7, 8, 2, 64), "f8", pool, pool, scales, scales, table)):
        with pytest.raises(ValueError):
            bad()


def test_oracle_of_the_codes():
    """Against the formats' tables, and nearest values by trying all of them."""
    f4 = kv_oracle.code_values("f4")
    assert f4.tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    f8 = kv_oracle.code_values("f8")
    bits = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(f8, bits) and f8[-1] == 448
    rng = np.random.default_rng(1)
    for form, table, limit in (("f8", f8, 464.0), ("f4", f4, 7.0)):
        for dtype in ("bf16", "f16"):
            x = rng.standard_normal((40, 64)) * 2.0 ** rng.integers(-20, 12, (40, 1))
            x[0] = 0
            x[1, :32] = np.arange(32) / 16
            codes, scales, values = kv_oracle.quantise(x, form, dtype)
            assert np.array_equal(kv_oracle.stored_values(codes, scales, form), values)
            for i in range(40):
                for j in range(2):
                    block, s = x[i, 32 * j:32 * j + 32], 2.0 ** (scales[i, j] - 127.0)
                    top = np.abs(block).max()
                    least = {"f8": -15, "f4": -23}[form] if dtype == "f16" else -100
                    assert top <= limit * s and (top >= limit * s / 2 or scales[i, j] - 127 == least or top == 0)
                    for a, b in zip(block, values[i, 32 * j:32 * j + 32]):
                        assert abs(abs(a) - abs(b)) == np.abs(table * s - abs(a)).min() and (a == 0 or b == 0 or (a < 0) == (b < 0))
        broken = np.ones((1, 64))
        broken[0, 40] = np.inf
        codes, scales, values = kv_oracle.quantise(broken, form, "f32")
        assert scales[0, 1] == 255 and np.isnan(values[0, 32:]).all() and (values[0, :32] == 1).all()


def test_unpacked_codes():
    pool = np.arange(256, dtype=np.uint8).reshape(1, 256)
    assert np.array_equal(kv_oracle.unpack(pool, "f8"), pool)
    codes = kv_oracle.unpack(pool, "f4")
    assert codes.shape == (1, 512) and (codes[0, 0::2] == np.arange(256) % 16).all() and (codes[0, 1::2] == np.arange(256) // 16).all()


class Route(C.Structure):
    _fields_ = [("split", C.c_bool), ("wavefronts", C.c_int32), ("splits", C.c_int32), ("workspace", C.c_int64)]


class SharedRoute(C.Structure):
    _fields_ = [("wavefronts", C.c_int32), ("splits", C.c_int32), ("budget", C.c_int32), ("slots", C.c_int64), ("part_rows", C.c_int64), ("cuts_at", C.c_int64), ("own_at", C.c_int64),
                ("split_at", C.c_int64), ("workspace", C.c_int64)]


# KvRoute kvq_route(const flame_kv_config &, int32_t n_seqs, int64_t n_rows, bool decode, int64_t capacity) and
# KvSharedRoute kv_shared_route(const flame_kv_config &, int32_t n_groups, int64_t n_rows, int64_t capacity) of csrc/kv.h
kvq_route = B._lib["_ZN5flame9kvq_routeERK15flame_kv_configilbl"]
kvq_route.restype, kvq_route.argtypes = Route, [C.POINTER(B.flame_kv_config), C.c_int32, C.c_int64, C.c_bool, C.c_int64]
kv_shared_route = B._lib["_ZN5flame15kv_shared_routeERK15flame_kv_configill"]
kv_shared_route.restype, kv_shared_route.argtypes = SharedRoute, [C.POINTER(B.flame_kv_config), C.c_int32, C.c_int64, C.c_int64]
ROOM = [1, 1023, 1024, 1025, 5000, 16384, 1 << 20, (1 << 31) - 65536]
SHAPES = [("bf16", 32, 8, 128), ("f16", 8, 2, 64), ("f32", 32, 8, 128), ("bf16", 1, 1, 32), ("f32", 6, 2, 64), ("f16", 40, 1, 32), ("bf16", 400, 400, 64), ("f32", 4096, 1, 128)]


@pytest.mark.parametrize("dtype,hq,hkv,dim", SHAPES)
def test_a_workspace_serves_every_smaller_batch(dtype, hq, hkv, dim):
    cfg, rng = B.make_kv_config(dtype, hq, hkv, dim), np.random.default_rng(hq)
    most = [min(1 << 22, ((1 << 23) - 1) // hq), min((1 << 25) // hq, (1 << 24) - 1)]
    counts = [sorted({min(n, m) for n in [1, 2, 5, 8, 16, 33, 64, 65, 128, 129, 200, 400, 401, 1000, 4096, 1 << 17, m] + rng.integers(1, 3000, 8).tolist()}) for m in most]
    needed, held, shared = {}, {}, {}
    for s in counts[0]:
        for t in counts[1]:
            needed[s, t] = max(kvq_route(cfg, s, t, False, c).workspace for c in ROOM)
            held[s, t] = B.flame_kv_workspace_bytes(cfg, s, t)
    for t in counts[1]:
        shared[t] = 0
        for g in [0] + counts[0]:
            for c in ROOM:
                r = kv_shared_route(cfg, g, t, c)
                rows = 128 // r.wavefronts
                assert (r.slots * hkv * max(r.splits, 1) + 1024) * 256 < 1 << 32 and r.part_rows >= (0 if g == 0 else t * hq)
                # the parts that the row tiles may leave: of equal length as many as there are slots, else a plane for each of `splits`
                if g:
                    assert r.part_rows >= (r.slots * hkv * rows if r.splits == 0 else r.splits * t * hq)
                    assert r.slots >= t * (hq // hkv) // rows + g and (r.splits or (g <= 64 and 1 <= r.budget <= r.slots))
                assert r.cuts_at >= r.part_rows * (dim + 2) * 4 and r.own_at >= r.cuts_at + 512 and r.split_at >= r.own_at + t * hq * (dim + 2) * 4 and r.split_at % 16 == r.own_at % 16 == 0
                shared[t] = max(shared[t], r.workspace)
    for s_most in counts[0]:
        for t_most in counts[1]:
            assert held[s_most, t_most] >= max(needed[s, t] for s, t in needed if s <= s_most and t <= t_most), (s_most, t_most)
    for t_most in counts[1]:
        assert B.flame_kv_shared_workspace_bytes(cfg, 1, 1, t_most) >= max(n for t, n in shared.items() if t <= t_most), t_most
