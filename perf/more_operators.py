"""The operators on a cache of 8 or 4 bits, and on histories that several sequences share, whose speed is measured, over the range that their users call them in.

A case is one of four:

  append   flame_kvq_append: keys and values of new tokens, quantised as they are written, keys and queries rotated on the way; and flame_kvq_read of all that the
           sequences hold then, as whoever takes the cache elsewhere does;
  read     flame_kvq_read: keys and values of whole sequences back as rows of the element type;
  attend   flame_kvq_extend, or flame_kvq_decode with one new token a sequence: causal attention over a quantised cache;
  shared   flame_kv_shared or flame_kvq_shared: the same for groups of sequences that begin with the same tokens, which are read once for all of them.

The form of a cache is "f8" (e4m3), "f4" (e2m1), both with a power of two for each 32 features, or "plain" (the element type).  Sequences have `lo` to `hi` tokens
(uniform, the last of them `hi`) of which `new_lo` to `new_hi` are new; in shared cases these are their own tokens, and each of the `groups` has `p_lo` to `p_hi` before
them.  Lengths follow from the case alone, values from the seed: queries, keys and values arrive as slices of the rows of one projection, N(0, 1), queries N(0, 2^2), so
that logits spread over several units.  The pages of a sequence lie anywhere in the pool, and the pages of a shared history are in the tables of all its sequences.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BITS = {"f8": 8, "f4": 4}


def _heads(q, kv, dim, dtype="bf16"):
    return dict(q_heads=q, kv_heads=kv, dim=dim, dtype=dtype)


def _lengths(seqs, lo, hi, new_lo=1, new_hi=1, page=16, draw=0):
    return dict(seqs=seqs, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, page=page, draw=draw)


def _history(groups=0, p_lo=0, p_hi=0):
    return dict(groups=groups, p_lo=p_lo, p_hi=p_hi)


def _rotary(rotary=0, interleaved=False):
    return dict(rotary=rotary, interleaved=interleaved)


def listed():
    return [
        # one new action of each of a batch of users: the smallest call that writes
        dict(name="append_step_f8", kind="append", form="f8", **_rotary(64), **_heads(8, 2, 64), **_lengths(48, 200, 1500)),
        # whole prompts of a model without rotation (its positions are a bias) into 4 bits
        dict(name="append_prompts_f4", kind="append", form="f4", **_rotary(), **_heads(32, 8, 128), **_lengths(12, 100, 3500, 100, 3500, 64)),
        # pieces of histories, neighbours as pairs in half of the features, pages of an odd size
        dict(name="append_pieces_f8", kind="append", form="f8", **_rotary(32, True), **_heads(8, 8, 64, "f16"), **_lengths(24, 300, 3000, 100, 500, 24)),
        # one user's history out of the cache: latency counts
        dict(name="read_one_f8", kind="read", form="f8", **_heads(8, 8, 64, "f16"), **_lengths(1, 2573, 2573)),
        # a ragged batch of histories
        dict(name="read_batch_f4", kind="read", form="f4", **_heads(32, 8, 128), **_lengths(40, 500, 9000, page=32)),
        # one user's next token: latency counts
        dict(name="decode_one_f8", kind="attend", form="f8", **_heads(8, 8, 64, "f16"), **_lengths(1, 2573, 2573)),
        # an ordinary ragged batch in service
        dict(name="decode_batch_f8", kind="attend", form="f8", **_heads(32, 8, 128), **_lengths(64, 100, 8192)),
        # few sequences, very long caches in 4 bits
        dict(name="decode_long_f4", kind="attend", form="f4", **_heads(32, 4, 128), **_lengths(3, 60000, 131072, page=64)),
        # prompts taken in pieces, most of them in the cache already: the most work
        dict(name="extend_chunk_f8", kind="attend", form="f8", **_heads(32, 8, 128), **_lengths(6, 4000, 16384, 400, 400)),
        # one user's candidates: each is a token of its own behind the user's history
        dict(name="shared_candidates", kind="shared", form="plain", **_heads(8, 8, 64, "f16"), **_history(1, 2000, 2000), **_lengths(128, 1, 1)),
        # users with several continuations each
        dict(name="shared_batch", kind="shared", form="plain", **_heads(32, 8, 128), **_history(8, 2000, 12000), **_lengths(96, 20, 800)),
        # long common histories in 8 bits, a few new tokens of every sequence
        dict(name="shared_long_f8", kind="shared", form="f8", **_heads(32, 4, 128), **_history(2, 40000, 65536), **_lengths(100, 10, 2000, 1, 4)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "read", "attend", "attend", "shared", "shared"])
    while True:
        q, kv, dim = rng.choice([(8, 8, 64), (8, 2, 64), (16, 16, 32), (8, 1, 64), (32, 8, 128), (16, 2, 128), (6, 2, 128), (16, 16, 128), (32, 4, 128)])
        c = dict(kind=kind, form=rng.choice(["f8", "f4"]), **_heads(q, kv, dim, rng.choice(["bf16", "bf16", "f16", "f32"])))
        page, seed = rng.choice([8, 16, 16, 24, 32, 64, 100, 256]), rng.randrange(1 << 16)
        if kind == "append":
            hi = _log_int(rng, 64, 8192)
            new = rng.choice([1, 1, _log_int(rng, 2, hi), hi])
            # A value in 4 bits, or in 8 where the results are fp32, jumps by more than results may be off where rotations that differ in their last place
            # fall on either side of the middle between two codes.  Rotated keys are drawn where no such jump is that large.
            turns = c["form"] == "f8" and c["dtype"] != "f32"
            c.update(**_rotary(rng.choice([dim, dim, dim // 2, 0]) if turns else 0, rng.random() < 0.5),
                     **_lengths(_log_int(rng, 1, 256), max(1, hi // 8), hi, max(1, new // rng.choice([1, 4])), new, page, seed))
        elif kind == "read":
            hi = _log_int(rng, 1, 16384)
            c.update(**_lengths(_log_int(rng, 1, 256), max(1, int(hi * rng.choice([0.01, 0.5, 1.0]))), hi, page=page, draw=seed))
        elif kind == "attend":
            hi = _log_int(rng, 64, 131072)
            new = rng.choice([1, 1, _log_int(rng, 2, min(hi, 1024))])
            c.update(**_lengths(_log_int(rng, 1, 256), max(1, hi // rng.choice([1, 2, 16])), hi, max(1, new // rng.choice([1, 4])), new, page, seed))
        else:
            p, hi = _log_int(rng, 64, 65536), _log_int(rng, 1, 4096)
            new, groups = rng.choice([1, 1, _log_int(rng, 1, min(hi, 16))]), _log_int(rng, 1, 16)
            c.update(form=rng.choice(["plain", "plain", "f8", "f4"]), **_history(groups, max(1, p // rng.choice([1, 2, 8])), p),
                     **_lengths(groups * _log_int(rng, 1, 128), max(1, hi // rng.choice([1, 4, 16])), hi, max(1, new // rng.choice([1, 4])), new, page, seed))
        w, heaviest = work(c), 4.0e10 if c["dtype"] == "f32" else 3.0e11
        n, m, p = _counts(c)
        # nothing larger than the largest listed call, nor a cache, padded to its longest sequence, or scores that the plain form cannot spread out
        padded = c["seqs"] * (c["hi"] if kind != "attend" or c["new_hi"] == 1 else 0) * kv * dim
        scores = 0 if kind != "shared" else max(p) * c["seqs"] // c["groups"] * int(m.max()) * q
        if w["flops"] <= heaviest and w["bytes"] <= 5.0e8 and padded <= 1 << 28 and scores <= 1 << 29 and (n.sum() + p.sum()) * kv * dim <= 1 << 28 and c["seqs"] <= 1024:
            return c


def _counts(case):
    """Tokens of the sequences behind what they share, how many of them are new, and the shared ones of each group."""
    rng = np.random.default_rng(case["draw"])
    n = rng.integers(case["lo"], case["hi"] + 1, case["seqs"])
    n[-1] = case["hi"]
    m = np.minimum(n, rng.integers(case["new_lo"], case["new_hi"] + 1, case["seqs"]))
    p = rng.integers(case["p_lo"], case["p_hi"] + 1, case["groups"]) if case.get("groups") else np.zeros(0, np.int64)
    p[-1:] = case.get("p_hi", 0)
    return n, m, p


def _groups(case):
    """Where the groups begin among the sequences."""
    return np.linspace(0, case["seqs"], case["groups"] + 1).astype(np.int64)


def work(case):
    n, m, p = (x.astype(np.float64) for x in _counts(case))
    size = 4 if case["dtype"] == "f32" else 2
    held = size if case["form"] == "plain" else BITS[case["form"]] / 8 + 1 / 32
    q, kv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    tables = 4.0 * ((n / case["page"]).sum() + (p / case["page"]).sum()) + 8.0 * case["seqs"]
    read = (n.sum() * 2 * kv * dim) * (held + size)
    if case["kind"] == "append":
        return {"bytes": float(m.sum() * dim * (2 * kv * (size + held) + 2 * q * size) + read + tables), "flops": float(m.sum() * (q + kv) * case["rotary"] / 2 * 6)}
    if case["kind"] == "read":
        return {"bytes": float(read + tables), "flops": 0.0}
    pairs = (m * n - m * (m - 1) / 2).sum()
    if case["kind"] == "shared":
        first = _groups(case)
        pairs += sum(p[g] * m[first[g]:first[g + 1]].sum() for g in range(case["groups"]))
    return {"bytes": float(m.sum() * 2 * q * dim * size + (n.sum() + p.sum()) * 2 * kv * dim * held + tables), "flops": float(4 * dim * q * pairs)}


def _frequencies(rotary):
    return 10000.0 ** (-np.arange(0, rotary, 2) / max(rotary, 1))


# ----------------------------------------------------------------------------------------------
# what the cache holds
# ----------------------------------------------------------------------------------------------
def _encode(x, form, dtype):
    """Codes and scales (bytes) of x [..., dim] in fp32: per 32 features the least power of two by which none of them rounds to more than the largest code."""
    blocks = x.unflatten(-1, (-1, 32))
    # nothing that would read back as an infinity, nor finer than the element type
    least, most = {"f8": (-15, 61440.0), "f4": (-23, 49152.0)}[form] if dtype == "f16" else {"f8": (-117, 240 * 2.0 ** 120), "f4": (-125, 1.5 * 2.0 ** 127)}[form]
    blocks = blocks.clamp(-most, most)
    mantissa, exponent = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    if form == "f8":
        exponent = exponent - 9 + (mantissa > 464 / 512).int()
    else:
        exponent = exponent - 3 + (mantissa >= 7 / 8).int()
    exponent = exponent.clamp(min=least)
    y = torch.ldexp(blocks, -exponent)
    if form == "f8":
        codes = y.flatten(-2).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        y = y.flatten(-2)
        a = y.abs()
        step = 0.5 + 0.5 * (a >= 2).float() + (a >= 4).float()
        a = torch.round(a / step) * step
        code = (torch.bucketize(a, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)) + 8 * torch.signbit(y).int()).to(torch.uint8)
        codes = code[..., 0::2] | code[..., 1::2] << 4
    return codes, (exponent.squeeze(-1) + 127).to(torch.uint8)


def _values(codes, scales, form):
    """fp32 values of codes [..., stored bytes] with scales [..., blocks]."""
    if form == "f8":
        y = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
        y = table[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(-2)
    return (y.unflatten(-1, (-1, 32)) * torch.exp2(scales.float() - 127)[..., None]).flatten(-2)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype, q, kv, dim = TYPES[case["dtype"]], case["q_heads"], case["kv_heads"], case["dim"]
    n, m, p = _counts(case)
    seqs, tokens, page = case["seqs"], int(m.sum()), case["page"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32 if case["dtype"] == "f32" else torch.float16).to(dtype)

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)

    state = {"case": dict(case), "m": [int(x) for x in m]}
    if case["kind"] != "read":
        rows = normal(tokens, q + 2 * kv, dim)
        rows[:, :q] *= 2
        state.update(q=rows[:, :q], k=rows[:, q:q + kv], v=rows[:, q + kv:], offsets=ints(np.concatenate([[0], np.cumsum(m)])),
                     out=torch.empty(tokens, q, dim, device=DEVICE, dtype=dtype))
    # the pages: those of the groups' histories as far as they are full, then each sequence's own
    first = _groups(case) if len(p) else np.zeros(1, np.int64)
    before = np.zeros(seqs, np.int64)
    group = np.searchsorted(first, np.arange(seqs), side="right") - 1
    if len(p):
        before = p[group]
    n = n + before
    full = before // page
    trunk = p // page
    used = -(-n // page) - full
    pages = int(used.sum() + trunk.sum()) + 3
    order = np.random.default_rng(seed).permutation(pages)
    table = np.zeros((seqs, int((used + full).max())), np.int32)
    starts, own_starts = np.cumsum(trunk) - trunk, int(trunk.sum()) + np.cumsum(used) - used
    for b in range(seqs):
        if len(p):
            table[b, :full[b]] = order[starts[group[b]]:starts[group[b]] + full[b]]
        table[b, full[b]:full[b] + used[b]] = order[own_starts[b]:own_starts[b] + used[b]]
    state.update(n=[int(x) for x in n], lens=ints(n), table=ints(table))
    if len(p):
        state.update(p=[int(x) for x in p], first=[int(x) for x in first], group_offsets=ints(first), prefix_lens=ints(before))
    for x in ("k", "v"):
        values = normal(pages, page, kv, dim)
        if case["form"] == "plain":
            state[x + "_pool"] = values
        else:
            state[x + "_pool"], state[x + "_scales"] = _encode(values.float(), case["form"], case["dtype"])
    if case["kind"] in ("append", "read"):
        state["all_offsets"] = ints(np.concatenate([[0], np.cumsum(n)]))
        state["k_all"], state["v_all"] = (torch.empty(int(n.sum()), kv, dim, device=DEVICE, dtype=dtype) for _ in range(2))
    return state


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["kind"] == "append":
        return _plain_append(state, case)
    if case["kind"] == "read":
        return _plain_read(state, case)
    return _plain_attention(state, case)


def _own(state):
    from paper_2509_22681_amd import binding as B
    case = state["case"]
    if "config" not in state:           # what a program makes once: the shape, the pool with its table, the frequencies, the workspace
        cfg = state["config"] = B.make_kv_config(case["dtype"], case["q_heads"], case["kv_heads"], case["dim"])
        if case["form"] == "plain":
            state["cache"] = B.pack_kv_cache(cfg, state["k_pool"], state["v_pool"], state["table"])
        else:
            state["cache"] = B.pack_kvq_cache(cfg, case["form"], state["k_pool"], state["v_pool"], state["k_scales"], state["v_scales"], state["table"])
        if case["kind"] == "append":
            state["rotation"] = B.make_kv_rotation(_frequencies(case["rotary"]), interleaved=case["interleaved"]) if case["rotary"] else None
        if case["kind"] == "attend":
            state["workspace"] = torch.empty(B.flame_kv_workspace_bytes(cfg, case["seqs"], sum(state["m"])), device=DEVICE, dtype=torch.uint8)
        if case["kind"] == "shared":
            state["workspace"] = torch.empty(B.flame_kv_shared_workspace_bytes(cfg, case["groups"], case["seqs"], sum(state["m"])), device=DEVICE, dtype=torch.uint8)
    cfg, cache = state["config"], state["cache"]
    if case["kind"] == "append":
        B.flame_kvq_append(cfg, cache, state["k"], state["v"], state["offsets"], state["lens"], q=state["q"], q_out=state["out"], rotation=state["rotation"])
    if case["kind"] in ("append", "read"):
        B.flame_kvq_read(cfg, cache, state["all_offsets"], state["lens"], state["k_all"], state["v_all"])
        return {"k": state["k_all"], "v": state["v_all"], **({"q": state["out"]} if case["kind"] == "append" else {})}
    single = case["new_hi"] == 1
    if case["kind"] == "attend" and single:
        B.flame_kvq_decode(cfg, cache, state["q"], state["lens"], state["out"], state["workspace"])
    elif case["kind"] == "attend":
        B.flame_kvq_extend(cfg, cache, state["q"], state["offsets"], state["lens"], state["out"], state["workspace"])
    else:
        call = B.flame_kv_shared if case["form"] == "plain" else B.flame_kvq_shared
        call(cfg, cache, state["q"], None if single else state["offsets"], state["lens"], state["group_offsets"], state["prefix_lens"], state["out"], state["workspace"])
    return state["out"]


# ----------------------------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------------------------
def _rotated(x, positions, case):
    r = case["rotary"]
    x = x.float()
    if not r:
        return x
    # the angles of far positions need 64 bits
    angle = positions.double()[:, None] * torch.from_numpy(_frequencies(r)).to(DEVICE)
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    y = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def _where(state, case, offsets):
    """Sequence and position of every row of sequences whose newest tokens are at offsets[b]..offsets[b + 1], and the page and slot of it."""
    off = offsets.long()
    token = torch.arange(int(sum(state["m"])) if offsets is not state.get("all_offsets") else len(state["k_all"]), device=DEVICE)
    seq = torch.bucketize(token, off[1:], right=True)
    position = state["lens"].long()[seq] - off[seq + 1] + token
    return position, state["table"].long()[seq, position // case["page"]], position % case["page"]


def _plain_append(state, case):
    position, page, slot = _where(state, case, state["offsets"])
    for x, rows in (("k", _rotated(state["k"], position, case)), ("v", state["v"].float())):
        codes, scales = _encode(rows, case["form"], case["dtype"])
        state[x + "_pool"][page, slot] = codes
        state[x + "_scales"][page, slot] = scales
    return {**_plain_read(state, case), "q": _rotated(state["q"], position, case).to(TYPES[case["dtype"]])}


def _plain_read(state, case):
    _, page, slot = _where(state, case, state["all_offsets"])
    return {x: _values(state[x + "_pool"][page, slot], state[x + "_scales"][page, slot], case["form"]).to(TYPES[case["dtype"]]) for x in ("k", "v")}


def _tokens(state, case, seqs, at):
    """fp32 keys and values of tokens `at` [len(seqs), n] of sequences `seqs`, as [sequence, head, token, feature]."""
    page, slot = state["table"].long()[seqs[:, None], at // case["page"]], at % case["page"]
    for x in ("k", "v"):
        rows = state[x + "_pool"][page, slot]
        rows = rows.float() if case["form"] == "plain" else _values(rows, state[x + "_scales"][page, slot], case["form"])
        yield rows.transpose(1, 2).contiguous()


def _plain_attention(state, case):
    """A group of sequences at a time: scores of all their rows with what they share, and of each one's rows with its own tokens, in one softmax.  Without a shared history,
    single tokens are one group, and longer pieces one for each sequence, as many rows at a time as their scores have room for."""
    kv, dim, dtype = case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    heads = case["q_heads"] // kv
    out = torch.empty_like(state["out"])
    single = case["new_hi"] == 1
    first = state.get("first") or ([0, case["seqs"]] if single else list(range(case["seqs"] + 1)))
    start = np.concatenate([[0], np.cumsum(state["m"])])
    for g, (b0, b1) in enumerate(zip(first[:-1], first[1:])):
        if b0 == b1:
            continue
        p = state["p"][g] if "p" in state else 0
        n, m = np.array(state["n"][b0:b1]), np.array(state["m"][b0:b1])
        last, most = int(n.max()) - p, int(m.max())
        seqs = torch.arange(b0, b1, device=DEVICE)
        lens, rows = torch.from_numpy(n).to(DEVICE), torch.from_numpy(m).to(DEVICE)
        behind = (p + torch.arange(last, device=DEVICE))[None, :]
        own_k, own_v = _tokens(state, case, seqs, torch.minimum(behind, lens[:, None] - 1))
        own_k = own_k.transpose(2, 3).contiguous()
        if p:
            k, v = (x[0] for x in _tokens(state, case, seqs[:1], torch.arange(p, device=DEVICE)[None, :]))
            k = k.transpose(1, 2).contiguous()
        step = max(1, (1 << 29) // (case["q_heads"] * (b1 - b0) * (last + p)))
        for i in range(0, most, step):
            # rows i, i + 1.. of every sequence (those behind its last one repeat that), as [sequence, row]
            row = torch.minimum(torch.arange(i, min(most, i + step), device=DEVICE)[None, :], rows[:, None] - 1)
            at = torch.from_numpy(start[b0:b1]).to(DEVICE)[:, None] + row
            q = state["q"][at].float() / math.sqrt(dim)
            q = q.unflatten(2, (kv, heads)).permute(0, 2, 1, 3, 4)                           # [sequence, key head, row, head, feature]
            s = torch.bmm(q.flatten(2, 3).flatten(0, 1), own_k.flatten(0, 1)).unflatten(0, (b1 - b0, kv)).unflatten(2, q.shape[2:4])
            hidden = behind[:, None, :] > (lens - rows)[:, None, None] + row[:, :, None]
            s.masked_fill_(hidden[:, None, :, None, :], -math.inf)
            top = s.amax(-1, keepdim=True)
            if p:
                z = torch.bmm(q.transpose(0, 1).flatten(1, 3), k).unflatten(1, (b1 - b0, *q.shape[2:4])).transpose(0, 1)
                top = torch.maximum(top, z.amax(-1, keepdim=True))
                z = (z - top).exp_()
            s = s.sub_(top).exp_()
            total = s.sum(-1, keepdim=True)
            o = torch.bmm(s.flatten(2, 3).flatten(0, 1), own_v.flatten(0, 1)).unflatten(0, (b1 - b0, kv)).unflatten(2, q.shape[2:4])
            if p:
                total = total + z.sum(-1, keepdim=True)
                o = o + torch.bmm(z.transpose(0, 1).flatten(1, 3), v).unflatten(1, (b1 - b0, *q.shape[2:4])).transpose(0, 1)
            out[at] = (o / total).permute(0, 2, 1, 3, 4).flatten(2, 3).to(dtype)
    return out


# ----------------------------------------------------------------------------------------------
# the definition in 64 bits: codes bit by bit, tokens one sequence and head at a time
# ----------------------------------------------------------------------------------------------
def _code_values(form):
    """The value of every code, from its bits: sign, exponent, fraction."""
    bits, fraction, bias = (8, 3, 7) if form == "f8" else (4, 1, 1)
    got = []
    for code in range(1 << bits):
        e, f = code >> fraction & (1 << bits - 1 - fraction) - 1, code & (1 << fraction) - 1
        x = math.ldexp(f, 1 - bias - fraction) if e == 0 else math.ldexp((1 << fraction) + f, e - bias - fraction)
        got.append(math.nan if form == "f8" and code & 127 == 127 else -x if code >> bits - 1 else x)
    return np.array(got)


def _exact_values(state, case, x):
    """The pool of keys or values in 64 bits, [tokens, heads, features]."""
    pool = state[x + "_pool"].flatten(0, 1)
    if case["form"] == "plain":
        return pool.double()
    codes = pool.long() if case["form"] == "f8" else torch.stack([pool.long() % 16, torch.div(pool.long(), 16, rounding_mode="floor")], -1).flatten(-2)
    scale = torch.pow(torch.tensor(2.0, device=DEVICE, dtype=torch.float64), state[x + "_scales"].flatten(0, 1).double() - 127)
    return torch.from_numpy(_code_values(case["form"])).to(DEVICE)[codes] * scale.repeat_interleave(32, -1)


def _exact_quantised(x, case):
    """Values that a cache holds of x [tokens, heads, features] in 64 bits."""
    form = case["form"]
    values = _code_values(form)
    values = np.sort(values[(values >= 0) & np.isfinite(values)])
    values = np.unique(values)
    middle = (values[1:] + values[:-1]) / 2
    # beyond the largest code the next one would be a step further; a middle goes to the even code
    beyond = values[-1] + (values[-1] - values[-2]) / 2
    even = np.arange(len(values)) % 2 == 0
    least = (-15 if form == "f8" else -23) if case["dtype"] == "f16" else (-117 if form == "f8" else -125)
    blocks = x.unflatten(-1, (-1, 32))
    most = blocks.abs().amax(-1)
    e = torch.ceil(torch.log2(most / beyond)).clamp(min=least)
    e = torch.where(most * torch.exp2(-e + 1) < beyond, e - 1, e)
    over = most * torch.exp2(-e)
    e = torch.where(over > beyond if even[-1] else over >= beyond, e + 1, e).clamp(min=least)
    y = blocks * torch.exp2(-e)[..., None]
    table = torch.from_numpy(values).to(DEVICE)
    up = torch.searchsorted(torch.from_numpy(middle).to(DEVICE), y.abs().contiguous())     # of a middle the lower neighbour
    tie = y.abs() == torch.from_numpy(np.append(middle, np.inf)).to(DEVICE)[up]
    up = torch.where(tie & (up % 2 == 1), up + 1, up)
    return (torch.sign(y) * table[up] * torch.exp2(e)[..., None]).flatten(-2)


def _exact_turned(x, position, case):
    r = case["rotary"]
    x = x.double().clone()
    if r:
        turn = torch.from_numpy(np.exp(1j * position[:, None] * _frequencies(r)[None, :])).to(DEVICE)[:, None, :]
        head = x[..., :r].unflatten(-1, (r // 2, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
        turned = torch.view_as_real(torch.complex(head[..., 0].contiguous(), head[..., 1].contiguous()) * turn)
        x[..., :r] = (turned if case["interleaved"] else turned.transpose(-1, -2)).flatten(-2)
    return x


def exact(case, seed):
    state = prepare(case, seed)
    table, page, n = state["table"].cpu().numpy().astype(np.int64), case["page"], state["n"]

    def rows(b, first, last):
        t = np.arange(first, last)
        return torch.from_numpy(table[b, t // page] * page + t % page).to(DEVICE)

    k, v = _exact_values(state, case, "k"), _exact_values(state, case, "v")
    if case["kind"] in ("append", "read"):
        found = {}
        if case["kind"] == "append":
            m = state["m"]
            position = np.concatenate([np.arange(a - c, a) for a, c in zip(n, m)])
            at = torch.cat([rows(b, a - c, a) for b, (a, c) in enumerate(zip(n, m))])
            k[at] = _exact_quantised(_exact_turned(state["k"], position, case), case)
            v[at] = _exact_quantised(state["v"].double(), case)
            found["q"] = _exact_turned(state["q"], position, case)
        everything = torch.cat([rows(b, 0, a) for b, a in enumerate(n)])
        return {"k": k[everything], "v": v[everything], **found}
    out = torch.zeros(state["out"].shape, device=DEVICE, dtype=torch.float64)
    group, at = case["q_heads"] // case["kv_heads"], 0
    for b, (a, c) in enumerate(zip(n, state["m"])):
        mine = rows(b, 0, a)
        if "p" in state:
            g = int(np.searchsorted(state["first"], b, side="right")) - 1
            mine = torch.cat([rows(state["first"][g], 0, state["p"][g]), mine[state["p"][g]:]])
        keys, values = k[mine].transpose(0, 1).contiguous(), v[mine].transpose(0, 1).contiguous()
        for h in range(case["kv_heads"]):
            q = state["q"][at:at + c, h * group:(h + 1) * group].double().flatten(0, 1)
            last = (a - c + torch.arange(c, device=DEVICE)).repeat_interleave(group)
            z = q @ keys[h].T * case["dim"] ** -0.5
            z = torch.where(torch.arange(a, device=DEVICE)[None, :] <= last[:, None], z, torch.full_like(z, -math.inf))
            out[at:at + c, h * group:(h + 1) * group] = (torch.exp(z - torch.logsumexp(z, 1)[:, None]) @ values[h]).unflatten(0, (c, group))
        at += c
    return out
