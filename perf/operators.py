"""Timed workloads of the caches held in 4 bits: block tables, rows to and from 4 bits, decode attention.

Three kinds of work, in the order in which a serving program comes to them:

  tables   blocks of a paged cache for the requests of a batch, and the slots of their tokens, from lengths on the GPU
  store    key and value rows into a 4-bit cache, by the index lists of the routing or by slots, and their values back
  decode   one decode step's attention over caches held in 4 bits: contiguous, with per-sequence capacities, or paged

A row of d elements in 4 bits is d / 2 bytes of codes (E2M1: magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; element 2 i in
the low half of byte i) and a scale byte for every 32 elements (2^(byte - 127), 255: the block is NaN).  The scale of a block
is the smallest power of two, 2^-126 at least, that is no less than a seventh of the block's largest magnitude; elements
are rounded to the nearest code, ties to the even one.
"""
import math

import torch

DEV = "cuda"
THETA = 500000.0          # base of the rotary frequencies
own = False               # whether `run` calls the library, or computes the operators from elementary operations

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BORDERS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)        # between two magnitudes; on a border the even code wins


def _tables(name, **kw):
    c = dict(name=name, kind="tables", batch=1, hkv=8, n=8192, lengths="unequal", block_rows=64, fresh=True, scarce=False)
    c.update(kw)
    return c


def _store(name, **kw):
    c = dict(name=name, kind="store", how="lists", dtype="bf16", d=128, hkv=8, n=8192, batch=1, retain=0.10, approx=0.10, block_rows=64)
    c.update(kw)
    return c


def _decode(name, **kw):
    c = dict(name=name, kind="decode", dtype="bf16", d=128, hkv=8, group=4, n=8192, batch=1, lengths="equal", retain=0.10, approx=0.10,
             layout="blocks", block_rows=64, rope=False, step=False)
    c.update(kw)
    return c


def listed():
    return [
        # a decode step of 64 requests in flight: each grows by a token, and now and then one needs another block
        _tables("tables_step_64", batch=64, n=16000, fresh=False),
        # an ordinary batch of prompts, small blocks, and a pool that does not suffice for all of them
        _tables("tables_prompts_37", batch=37, hkv=2, n=5003, block_rows=16, scarce=True),
        # the largest: 256 prompts admitted at once
        _tables("tables_prompts_256", batch=256, n=8192, block_rows=16),
        # the new tokens of a decode step into a paged cache: latency
        _store("store_step_16", how="step", batch=16, n=32768),
        # one layer of the long prompt after its routing: the packed cache in 4 bits
        _store("store_lists_32k", n=32768),
        # a batch of prompts kept whole, all rows into their blocks
        _store("store_prompts_8", how="prompts", batch=8),
        # a small fp32 layer of an odd length
        _store("store_lists_5k_f32", dtype="f32", d=64, hkv=1, n=5001, retain=0.25, approx=0.25),
        # interactive use: one routed sequence, one step, latency is everything
        _decode("decode_1x8k", retain=0.15, approx=0.15),
        # serving: the repository's decode configuration, with the append
        _decode("decode_step_16x32k", n=32768, batch=16, step=True),
        # the largest: whole caches of long prompts, paged, nothing evicted
        _decode("decode_16x32k_whole", n=32768, batch=16, retain=1.0, approx=0.0, layout="paged"),
        # post-RoPE caches of prompts of unequal length
        _decode("decode_24_rope_unequal", n=16000, batch=24, lengths="unequal", layout="sequences", rope=True),
        # fp32 queries, 64 dims, an odd number of query heads and of tokens
        _decode("decode_3x2k_f32", dtype="f32", d=64, hkv=2, group=7, n=2049, batch=3, retain=0.3, approx=0.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(w["bytes"] for w in map(work, listed()))
    while True:
        c = _draw_once(rng)
        if work(c)["bytes"] <= most:
            return c


def _draw_once(rng):
    kind = rng.choices(("tables", "store", "decode"), (2, 2, 4))[0]
    hkv = rng.choice((1, 2, 4, 8, 8))
    dtype, d = ("f32" if rng.random() < 0.2 else "bf16"), rng.choice((64, 128, 128))
    block_rows = rng.choice((16, 32, 64, 64, 128))
    if kind == "tables":
        c = _tables("", batch=_log_int(rng, 1, 256), hkv=hkv, n=_log_int(rng, 2, 16000), lengths=rng.choice(("equal", "unequal")), block_rows=block_rows,
                    fresh=rng.random() < 0.6, scarce=rng.random() < 0.3)
    elif kind == "store":
        how = rng.choice(("lists", "lists", "step", "prompts"))
        c = _store("", how=how, dtype=dtype, d=d, hkv=hkv, n=_log_int(rng, 40, 8192 if how == "prompts" else 65536),
                   batch=1 if how == "lists" else _log_int(rng, 1, 64 if how == "step" else 8),
                   retain=round(rng.uniform(0.02, 0.5), 3), approx=round(rng.uniform(0.0, 0.5), 3), block_rows=block_rows)
    else:
        whole = rng.random() < 0.3
        layout = rng.choice(("blocks", "sequences", "paged"))
        c = _decode("", dtype=dtype, d=d, hkv=hkv, group=rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 8, 16)), n=_log_int(rng, 16, 32768), batch=_log_int(rng, 1, 48),
                    lengths=rng.choice(("equal", "unequal")), retain=1.0 if whole else round(rng.uniform(0.04, 0.5), 3),
                    approx=0.0 if whole else round(rng.uniform(0.04, 0.5), 3), layout=layout, block_rows=block_rows, rope=rng.random() < 0.3,
                    step=rng.random() < 0.3)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------
def _lengths(c):
    """Tokens of the sequences of a case, the longest n."""
    B, n = c["batch"], c["n"]
    if c.get("lengths", "equal") == "equal":
        return [n] * B
    # 1/4 .. 1 of n, in an order that is not sorted
    return [max(1, n - (n - n // 4) * ((5 * b + 3) % B if B % 5 else (3 * b + 1) % B) // B - b % 7) for b in range(B)]


def _rows(c, n):
    """Retained and approximated rows of a sequence of n tokens; at least one is retained."""
    return max(1, math.floor(c["retain"] * n + 1e-9)), math.floor(c["approx"] * n + 1e-9)


def _growth(c, b, n):
    """Tokens that a request already has blocks for, of n."""
    return 0 if c["fresh"] else n - 1


def _wanted_blocks(c):
    R, H = c["block_rows"], c["hkv"]
    return [H * (-(-n // R) - -(-_growth(c, b, n) // R)) for b, n in enumerate(_lengths(c))]


def _torch_dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def _inv_freq(d):
    return THETA ** (-torch.arange(0, d, 2, dtype=torch.float64, device=DEV) / d)


# ---------------------------------------------------------------------------
# the 4-bit format, in 32 bits
# ---------------------------------------------------------------------------
def _quantise(x):
    """Rows x [..., d] -> (magnitude codes with sign bit, uint8 [..., d], scale bytes [..., d / 32])."""
    blocks = x.float().unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    bad = ~torch.isfinite(blocks).all(-1)
    # the exponent of the largest magnitude, one more if its mantissa is above 1.75, less 2
    byte = ((top.view(torch.int32) + 0x1FFFFF) >> 23).sub_(2).clamp_(min=1)
    byte = torch.where(bad, 255, byte)
    unit = (torch.where(bad, 0, 254 - byte) << 23).view(torch.float32)       # one over the scale, by its bits: exp2 is not exact everywhere
    y = torch.nan_to_num(blocks, 0.0, 0.0, 0.0).abs_().mul_(unit[..., None])
    code = torch.zeros_like(y, dtype=torch.uint8)
    for i, border in enumerate(BORDERS):
        code += (y > border) if i % 2 == 0 else (y >= border)
    code += 8 * torch.signbit(blocks)
    return code.flatten(-2), byte.to(torch.uint8)


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unit(byte):
    """Scale bytes (1 and more) as 32-bit numbers."""
    return torch.where(byte == 255, float("nan"), (byte.int() << 23).view(torch.float32))


def _pairs():
    """The two values of every byte of codes, [256, 2]."""
    one = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=DEV)
    return torch.stack((one.repeat(16), one.repeat_interleave(16)), -1)


def _values(packed, byte, pairs):
    """Packed codes [..., d / 2] and scale bytes [..., d / 32] -> fp32 values [..., d]."""
    x = pairs[packed.int()].flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * _unit(byte)[..., None]).flatten(-2)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _keys_values(H, n, d, g, rope=False):
    """Keys and values [H, n, d] of one sequence: 5 % of the keys four times as long as the others, values of unequal size."""
    k = torch.randn(H, n, d, generator=g, device=DEV)
    k *= torch.where(torch.rand(H, n, 1, generator=g, device=DEV) < 0.05, 4.0, 1.0)
    v = torch.randn(H, n, d, generator=g, device=DEV) * 10.0 ** (-torch.rand(H, n, 1, generator=g, device=DEV))
    if rope:
        # the channels of turned keys are of unequal size: some pairs stand out
        k *= 1.0 + 3.0 * (torch.rand(H, 1, d, generator=g, device=DEV) < 0.06)
    return k, v


def _prepare_tables(c, seed):
    g = _generator(seed)
    lens, B, H, R = _lengths(c), c["batch"], c["hkv"], c["block_rows"]
    held = [_growth(c, b, n) for b, n in enumerate(lens)]
    # another seed has other lengths, of the same number of tokens
    order = torch.randperm(B, generator=g, device=DEV).tolist()
    lens, held = [lens[i] for i in order], [held[i] for i in order]
    per_seq = -(-c["n"] // R) + 2
    wanted = sum(_wanted_blocks(c))
    free = max(1, wanted * 2 // 3 if c["scarce"] else wanted + 3)
    taken = 0 if c["fresh"] else H * sum(-(-n // R) for n in held)
    ids = torch.randperm(free + taken, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(B, H, per_seq, dtype=torch.int32, device=DEV)
    if not c["fresh"]:                       # the blocks that the requests hold
        at = 0
        for b, n in enumerate(held):
            k = -(-n // R)
            table[b, :, :k] = ids[free + at:free + at + H * k].view(H, k)
            at += H * k
    s = dict(case=c, held=None if c["fresh"] else _i32(held), length=_i32(lens), free=ids[:free].contiguous(), table=table,
             n_slots=sum(lens) - sum(held), live=torch.zeros(B, dtype=torch.int32, device=DEV), counts=torch.zeros(3, dtype=torch.int32, device=DEV))
    s["slots"] = torch.zeros(H, s["n_slots"], dtype=torch.int64, device=DEV)
    if own:
        from paper_2605_23258_amd import binding as vb
        s["blocks"] = vb.make_blocks(s["length"], H, R, per_seq, s["free"], held=s["held"])
    return s


def _prepare_store(c, seed):
    g, dt = _generator(seed), _torch_dtype(c)
    H, d, n, R, B = c["hkv"], c["d"], c["n"], c["block_rows"], c["batch"]
    s = dict(case=c, pairs=_pairs())
    byte = lambda *shape: torch.zeros(*shape, dtype=torch.uint8, device=DEV)
    if c["how"] == "lists":
        k, v = _keys_values(H, n, d, g)
        n_r, n_a = _rows(c, n)
        # the lists of a routing: disjoint ascending token indices
        pick = torch.rand(H, n, generator=g, device=DEV).argsort(-1)
        s.update(k=k.to(dt), v=v.to(dt), idx_retain=pick[:, :n_r].sort(-1).values.to(torch.int32).contiguous(),
                 idx_approx=pick[:, n_r:n_r + n_a].sort(-1).values.to(torch.int32).contiguous(), n_r=n_r, n_a=n_a)
        for x, rows in (("k_ret", n_r), ("v_ret", n_r), ("k_apx", max(n_a, 1))):
            s[x], s[x + "_scale"], s[x + "_values"] = byte(H, rows, d // 2), byte(H, rows, d // 32), torch.zeros(H, rows, d, dtype=dt, device=DEV)
        T = n
    else:
        lens = [1] * B if c["how"] == "step" else _lengths(dict(c, lengths="unequal"))
        T, per_seq = sum(lens), -(-n // R)
        k, v = _keys_values(H, T, d, g)
        n_blocks = B * H * per_seq
        table = torch.randperm(n_blocks, generator=g, device=DEV).view(B, H, per_seq)
        slots = []
        for b, m in enumerate(lens):
            at = torch.arange(m, device=DEV) if c["how"] == "prompts" else torch.tensor([(n * (b + 1)) // (B + 1)], device=DEV)
            slots.append(table[b, :, at // R] * R + at % R)
        slots = torch.cat(slots, -1)
        slots[:, T - T // 50:] = -1                      # the last tokens are padding
        s.update(k=k.to(dt), v=v.to(dt), slots=slots.contiguous(), rows=n_blocks * R)
        for x in ("k_pool", "v_pool"):
            s[x], s[x + "_scale"], s[x + "_values"] = byte(n_blocks * R, d // 2), byte(n_blocks * R, d // 32), torch.zeros(H, T, d, dtype=dt, device=DEV)
    if own:
        from paper_2605_23258_amd import binding as vb
        s["shape"] = vb.Shape(n_q_heads=H, n_kv_heads=H, head_dim=d, seq_len=T, window=1, pool_kernel=1,
                              dtype=vb.VECTOR_BF16 if c["dtype"] == "bf16" else vb.VECTOR_F32)
    return s


def _segment(H, rows, d, g, rope=False):
    """Packed key and value rows [H, rows, ..] of a sequence, codes and scales."""
    out = []
    for x in _keys_values(H, rows, d, g, rope):
        code, scale = _quantise(x.bfloat16())
        out += [_pack(code), scale]
    return out


def _prepare_decode(c, seed):
    g, dt = _generator(seed), _torch_dtype(c)
    H, G, d, B, R = c["hkv"], c["group"], c["d"], c["batch"], c["block_rows"]
    lens = _lengths(c)
    rets, apxs = zip(*(_rows(c, n) for n in lens))
    room = 64                                            # rows free for the tokens to come
    caps = [r + room for r in rets] if c["layout"] == "sequences" else [max(rets) + room] * B
    n_as = list(apxs) if c["layout"] == "sequences" else [max(apxs)] * B
    byte = lambda *shape: torch.zeros(*shape, dtype=torch.uint8, device=DEV)
    s = dict(case=c, pairs=_pairs(), rets=rets, caps=caps, n_as=n_as, live=_i32(rets), length=_i32(rets), scale=1.0 / math.sqrt(d))
    ret0, apx0 = [H * sum(caps[:b]) for b in range(B)], [H * sum(n_as[:b]) for b in range(B)]
    if c["layout"] == "paged":
        per_seq = -(-caps[0] // R)
        n_blocks = B * H * per_seq
        s["table"] = torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32).view(B, H, per_seq)
        rows = n_blocks * R
    else:
        rows = H * sum(caps)
    pools = {"k_ret": byte(rows, d // 2), "k_ret_scale": byte(rows, d // 32), "v_ret": byte(rows, d // 2), "v_ret_scale": byte(rows, d // 32),
             "k_apx": byte(max(H * sum(n_as), 1), d // 2), "k_apx_scale": byte(max(H * sum(n_as), 1), d // 32)}
    for b in range(B):
        seg = _segment(H, rets[b], d, g, c["rope"])
        for x, part in zip(("k_ret", "k_ret_scale", "v_ret", "v_ret_scale"), seg):
            if c["layout"] == "paged":
                at = torch.arange(rets[b], device=DEV)
                pools[x][s["table"][b].long()[:, at // R] * R + at % R] = part
            else:
                pools[x][ret0[b]:ret0[b] + H * caps[b]].view(H, caps[b], -1)[:, :rets[b]] = part
        if n_as[b]:
            seg = _segment(H, n_as[b], d, g, c["rope"])
            for x, part in zip(("k_apx", "k_apx_scale"), seg):
                pools[x][apx0[b]:apx0[b] + H * n_as[b]] = part.flatten(0, 1)
    s.update(pools)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device=DEV)
    s["W"] = (rnd(H, d, d) / math.sqrt(d)).to(dt)
    s["q"] = rnd(B, H * G, d).to(dt)
    s["k_new"], s["v_new"] = rnd(B, H, d).to(dt), rnd(B, H, d).to(dt)
    s["out"] = torch.zeros(B, H * G, d, dtype=dt, device=DEV)
    s["start"] = (ret0, apx0)
    if c["rope"] and max(n_as):
        # the tokens' own positions: ascending in a row, with gaps
        gaps = torch.randint(1, 10, (H * sum(n_as),), generator=g, device=DEV).cumsum(0)
        s["positions"] = (gaps % 100003).to(torch.int32)
    if c["step"]:
        # where the new rows lie: [H, B] rows of the pools
        at = []
        for b in range(B):
            h = torch.arange(H, device=DEV)
            at.append(s["table"][b, :, rets[b] // R].long() * R + rets[b] % R if c["layout"] == "paged" else ret0[b] + h * caps[b] + rets[b])
        s["new_rows"] = torch.stack(at).contiguous()     # [B, H]
        s["k_row"], s["v_row"] = torch.zeros(B, H, d, dtype=dt, device=DEV), torch.zeros(B, H, d, dtype=dt, device=DEV)
    if own:
        from paper_2605_23258_amd import binding as vb
        cache = vb.CacheFp4()
        cache.batch, cache.n_q_heads, cache.n_kv_heads, cache.head_dim = B, H * G, H, d
        cache.dtype = vb.VECTOR_BF16 if c["dtype"] == "bf16" else vb.VECTOR_F32
        cache.cap_retain, cache.n_approx = max(caps), max(n_as)
        cache.len_retain, cache.W = s["live"].data_ptr(), s["W"].data_ptr()
        for x in pools:
            setattr(cache, x, s[x].data_ptr())
        if c["layout"] == "sequences":
            s["arrays"] = [_i32(caps), _i32(n_as), _i64(ret0), _i64(apx0)]
            cache.cap_retain_seq, cache.n_approx_seq, cache.ret_row_start, cache.apx_row_start = (t.data_ptr() for t in s["arrays"])
        if c["layout"] == "paged":
            cache.ret_block_table, cache.ret_block_rows, cache.ret_blocks_per_seq, cache.n_blocks = s["table"].data_ptr(), R, s["table"].shape[2], rows // R
        s["cache"] = cache
        s["rope"], s["keep"] = vb.make_rope(_inv_freq(d).cpu().numpy(), s["positions"]) if "positions" in s else (None, None)
        s["ws"] = torch.empty(vb.vector_decode_fp4_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    return s


def prepare(case, seed):
    return {"tables": _prepare_tables, "store": _prepare_store, "decode": _prepare_decode}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_tables(s):
    """Requests are admitted in order while the free blocks last (one that needs none always); an admitted one gets its new blocks,
    KV head after KV head, from the front of the free list, and its new tokens get the slots of their rows."""
    c = s["case"]
    H, R = c["hkv"], c["block_rows"]
    length, free, table = s["length"].long(), s["free"].long(), s["table"]
    B, per_seq = table.shape[0], table.shape[2]
    held = torch.zeros_like(length) if s["held"] is None else s["held"].long()
    before, after = (held + R - 1) // R, (length + R - 1) // R
    need = (after - before) * H
    upto = need.cumsum(0)
    admitted = (need == 0) | (upto <= free.numel())
    live = torch.where(admitted, length, held)
    # entries of the table
    col = torch.arange(per_seq, device=DEV)[None, None, :]
    fresh = admitted[:, None, None] & (col >= before[:, None, None]) & (col < after[:, None, None])
    at = (upto - need)[:, None, None] + torch.arange(H, device=DEV)[None, :, None] * (after - before)[:, None, None] + col - before[:, None, None]
    ids = free[torch.where(fresh, at, 0)].to(torch.int32)
    table = torch.where(fresh, ids, torch.zeros_like(table) if s["held"] is None else table)
    # slots of the new tokens, request after request
    grown = length - held
    start = grown.cumsum(0) - grown
    b = torch.repeat_interleave(torch.arange(B, device=DEV), grown, output_size=s["n_slots"])
    pos = held[b] + torch.arange(s["n_slots"], device=DEV) - start[b]
    ok = admitted[b]
    block = table[b, :, torch.where(ok, pos, 0) // R].t().long()
    slots = torch.where(ok[None], block * R + (pos % R)[None], -1)
    counts = torch.stack((torch.where(admitted, need, 0).sum(), upto[-1], grown.sum())).to(torch.int32)
    return {"table": table, "live": live.to(torch.int32), "slots": slots, "counts": counts}


def _round_trip(x, dt, pairs):
    code, scale = _quantise(x)
    return _values(_pack(code), scale, pairs).to(dt)


def _plain_store(s):
    c, dt = s["case"], _torch_dtype(s["case"])
    if c["how"] == "lists":
        rows = lambda x, idx: torch.gather(x, 1, idx.long()[..., None].expand(-1, -1, c["d"]))
        out = {"k_ret": _round_trip(rows(s["k"], s["idx_retain"]), dt, s["pairs"]), "v_ret": _round_trip(rows(s["v"], s["idx_retain"]), dt, s["pairs"])}
        if s["n_a"]:
            out["k_apx"] = _round_trip(rows(s["k"], s["idx_approx"]), dt, s["pairs"])
        return out
    there = (s["slots"] >= 0)[..., None]
    return {x: torch.where(there, _round_trip(s[x], dt, s["pairs"]), 0.0) for x in ("k", "v")}


def _plain_decode(s):
    c = s["case"]
    H, G, d, B, R, dt = c["hkv"], c["group"], c["d"], c["batch"], c["block_rows"], _torch_dtype(c)
    ret0, apx0 = s["start"]
    out = torch.empty(B, H, G, d, device=DEV)
    new = {x: _round_trip(s[x], torch.float32, s["pairs"]) for x in ("k_new", "v_new")} if c["step"] else None
    for b in range(B):
        r, cap, n_a = s["rets"][b], s["caps"][b], s["n_as"][b]
        if c["layout"] == "paged":
            at = torch.arange(r, device=DEV)
            rows = s["table"][b].long()[:, at // R] * R + at % R
            k, v = (_values(s[x][rows], s[x + "_scale"][rows], s["pairs"]) for x in ("k_ret", "v_ret"))
        else:
            part = lambda x: s[x][ret0[b]:ret0[b] + H * cap].view(H, cap, -1)[:, :r]
            k, v = (_values(part(x), part(x + "_scale"), s["pairs"]) for x in ("k_ret", "v_ret"))
        if c["step"]:
            k, v = torch.cat((k, new["k_new"][b][:, None]), 1), torch.cat((v, new["v_new"][b][:, None]), 1)
        if n_a:
            part = lambda x: s[x][apx0[b]:apx0[b] + H * n_a].view(H, n_a, -1)
            ka = _values(part("k_apx"), part("k_apx_scale"), s["pairs"])
            k = torch.cat((k, ka), 1)
            if c["rope"]:
                pos = s["positions"][apx0[b]:apx0[b] + H * n_a].view(H, n_a, 1).double()
                angle = pos * _inv_freq(d)
                cs, sn = torch.cos(angle).float(), torch.sin(angle).float()
                x, y = ka[..., :d // 2], ka[..., d // 2:]
                ka = torch.cat((x * cs + y * sn, y * cs - x * sn), -1)
            v = torch.cat((v, torch.bmm(ka, s["W"].float())), 1)
        q = s["q"][b].view(H, G, d).float()
        logits = torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]
        p = torch.exp(logits - logits.amax(-1, keepdim=True))
        out[b] = torch.bmm(p, v) / p.sum(-1, keepdim=True)
    res = {"out": out.view(B, H * G, d).to(dt)}
    if c["step"]:
        res.update(length=s["length"] + 1, k_row=new["k_new"].to(dt), v_row=new["v_new"].to(dt))
    return res


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _own_tables(s):
    from paper_2605_23258_amd import binding as vb
    vb.vector_block_tables(s["blocks"], s["table"], s["live"], s["slots"], s["counts"])
    return {x: s[x] for x in ("table", "live", "slots", "counts")}


def _own_store(s):
    from paper_2605_23258_amd import binding as vb
    c, d = s["case"], s["case"]["d"]
    dtype = vb.VECTOR_BF16 if c["dtype"] == "bf16" else vb.VECTOR_F32
    if c["how"] == "lists":
        vb.vector_compact_fp4(s["shape"], s["k"], s["v"], s["idx_retain"], s["idx_approx"] if s["n_a"] else None, s["n_r"], s["n_a"],
                              s["k_ret"], s["k_ret_scale"], s["v_ret"], s["v_ret_scale"], s["k_apx"], s["k_apx_scale"], s["n_r"])
        names = ("k_ret", "v_ret", "k_apx") if s["n_a"] else ("k_ret", "v_ret")
        for x in names:
            rows = s[x + "_values"].numel() // d
            vb.vector_load_fp4(rows, d, dtype, s[x], s[x + "_scale"], rows, None, s[x + "_values"])
        return {x: s[x + "_values"] for x in names}
    vb.vector_store_fp4(s["shape"], s["k"], s["v"], s["slots"], s["rows"], s["k_pool"], s["k_pool_scale"], s["v_pool"], s["v_pool_scale"])
    for x in ("k_pool", "v_pool"):
        vb.vector_load_fp4(s["slots"].numel(), d, dtype, s[x], s[x + "_scale"], s["rows"], s["slots"], s[x + "_values"])
    return {"k": s["k_pool_values"], "v": s["v_pool_values"]}


def _own_decode(s):
    from paper_2605_23258_amd import binding as vb
    c = s["case"]
    if not c["step"]:
        vb.vector_decode_attn_fp4(s["cache"], s["q"], s["scale"], s["out"], s["ws"], rope=s["rope"])
        return {"out": s["out"]}
    s["live"].copy_(s["length"])                         # every pass is the same step
    vb.vector_decode_step_fp4(s["cache"], s["q"], s["k_new"], s["v_new"], s["scale"], s["out"], s["ws"], rope=s["rope"])
    rows, dtype = s["new_rows"], vb.VECTOR_BF16 if c["dtype"] == "bf16" else vb.VECTOR_F32
    n_rows = s["k_ret"].shape[0]
    vb.vector_load_fp4(rows.numel(), c["d"], dtype, s["k_ret"], s["k_ret_scale"], n_rows, rows, s["k_row"])
    vb.vector_load_fp4(rows.numel(), c["d"], dtype, s["v_ret"], s["v_ret_scale"], n_rows, rows, s["v_row"])
    return {"out": s["out"], "length": s["live"], "k_row": s["k_row"], "v_row": s["v_row"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"tables": _own_tables, "store": _own_store, "decode": _own_decode}[kind](state)
    return {"tables": _plain_tables, "store": _plain_store, "decode": _plain_decode}[kind](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    H = c["hkv"]
    lens = _lengths(c)
    B = len(lens)
    if c["kind"] == "tables":
        R = c["block_rows"]
        new = sum(n - _growth(c, b, n) for b, n in enumerate(lens))
        blocks = sum(_wanted_blocks(c))
        entries = B * H * (-(-c["n"] // R) + 2) if c["fresh"] else blocks
        return {"bytes": 4 * (3 * B + blocks + entries + 3) + 8 * H * new, "flops": B + H * new}
    esz, d = (2 if c["dtype"] == "bf16" else 4), c["d"]
    row, packed = d * esz, d // 2 + d // 32
    if c["kind"] == "store":
        if c["how"] == "lists":
            n_r, n_a = _rows(c, c["n"])
            rows, index = H * (2 * n_r + n_a), 4 * H * (n_r + n_a)
        else:
            tokens = B if c["how"] == "step" else sum(_lengths(dict(c, lengths="unequal")))
            rows, index = 2 * H * tokens, 8 * H * tokens
        # rows in, codes and scales out and back in, values out
        return {"bytes": rows * (2 * row + 2 * packed) + index, "flops": 4 * rows * d}
    rets, apxs = zip(*(_rows(c, n) for n in lens))
    if c["layout"] != "sequences":
        apxs = [max(apxs)] * B
    P, A, Hq = sum(rets), sum(apxs), H * c["group"]
    bytes_ = H * (2 * P + A) * packed + 2 * B * Hq * row + (H * d * row if A else 0)
    if c["step"]:
        bytes_ += H * B * (4 * row + 4 * packed)
    return {"bytes": bytes_, "flops": Hq * ((P + A) * 4 * d + (B * 2 * d * d if A else 0))}


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _power(e):
    """2^e as 64-bit numbers, by their bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """Rows x [..., d] rounded to 4 bits, as 64-bit values."""
    blocks = x.double().unflatten(-1, (-1, 32))
    mantissa, exponent = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    # top = mantissa 2^exponent <= 7 * 2^e: e = exponent - 3 where mantissa <= 7 / 8, else exponent - 2
    e = torch.where(mantissa <= 0.875, exponent - 3, exponent - 2).clamp(min=-126)
    e = torch.where(mantissa == 0.0, torch.full_like(e, -126), e)
    unit = _power(e)
    y = blocks.abs() / unit
    # below 2 the codes lie 0.5 apart, below 4 1, then 2; round() takes ties to the even one
    step = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0)).double()
    y = (torch.round(y / step) * step).clamp(max=6.0)
    return (torch.copysign(y, blocks) * unit).flatten(-2)


def _exact_unpacked(packed, byte):
    nibbles = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    exponent, fraction = ((nibbles >> 1) & 3).double(), (nibbles & 1).double()
    size = torch.where(exponent == 0, 0.5 * fraction, (1.0 + 0.5 * fraction) * _power(exponent - 1.0))
    x = torch.where(nibbles >= 8, -size, size).unflatten(-1, (-1, 32)) * _power(byte.long() - 127)[..., None]
    return x.flatten(-2)


def _exact_decode(s):
    c = s["case"]
    H, G, d, B, R = c["hkv"], c["group"], c["d"], c["batch"], c["block_rows"]
    ret0, apx0 = s["start"]
    out = torch.empty(B, H, G, d, dtype=torch.float64, device=DEV)
    new = {x: _exact_rows(s[x]) for x in ("k_new", "v_new")}
    for b in range(B):
        r, cap, n_a = s["rets"][b], s["caps"][b], s["n_as"][b]
        for h in range(H):
            at = torch.arange(r, device=DEV)
            rows = s["table"][b, h].long()[at // R] * R + at % R if c["layout"] == "paged" else ret0[b] + h * cap + at
            k, v = (_exact_unpacked(s[x][rows], s[x + "_scale"][rows]) for x in ("k_ret", "v_ret"))
            if c["step"]:
                k, v = torch.cat((k, new["k_new"][b, h][None])), torch.cat((v, new["v_new"][b, h][None]))
            if n_a:
                at = apx0[b] + h * n_a + torch.arange(n_a, device=DEV)
                ka = _exact_unpacked(s["k_apx"][at], s["k_apx_scale"][at])
                k = torch.cat((k, ka))
                if c["rope"]:
                    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), -s["positions"][at].double()[:, None] * _inv_freq(d))
                    z = torch.complex(ka[:, :d // 2].contiguous(), ka[:, d // 2:].contiguous()) * turn
                    ka = torch.cat((z.real, z.imag), -1)
                v = torch.cat((v, torch.mm(ka, s["W"][h].double())))
            q = s["q"][b].view(H, G, d)[h].double()
            out[b, h] = torch.mm(torch.softmax(torch.mm(q, k.t().contiguous()) * s["scale"], -1), v)
    res = {"out": out.view(B, H * G, d)}
    if c["step"]:
        res.update(length=None, k_row=new["k_new"], v_row=new["v_new"])
    return res


def exact(case, seed):
    if case["kind"] == "tables":
        return None                                      # whole numbers, which the plain form has
    s = prepare(case, seed)
    if case["kind"] == "decode":
        return _exact_decode(s)
    if case["how"] == "lists":
        rows = lambda x, idx: torch.stack([x[h][idx[h].long()] for h in range(case["hkv"])])
        out = {"k_ret": _exact_rows(rows(s["k"], s["idx_retain"])), "v_ret": _exact_rows(rows(s["v"], s["idx_retain"]))}
        if s["n_a"]:
            out["k_apx"] = _exact_rows(rows(s["k"], s["idx_approx"]))
        return out
    gone = (s["slots"] < 0)[..., None]
    return {x: _exact_rows(s[x]).masked_fill(gone, 0.0) for x in ("k", "v")}
