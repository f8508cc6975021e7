"""The operators of a context cache held in 4 bits, measured over the sizes a serving program calls them in.

  append   the new keys/values of a step into the 4-bit cache, and what it then holds of them read back
           (relay_attn_cache_append_fp4, relay_attn_cache_read_fp4)
  read     rows of the 4-bit cache as bfloat16, straight into a system cache (relay_attn_cache_read_fp4)
  decode   one new token per request over [shared system prompt ; 4-bit context] (relay_attn_decode_fp4)
  prompt   several new tokens per request, causal inside the 4-bit context (relay_attn_prefill_fp4)
  tables   block tables, lengths, bounds of the new tokens and their slots from request lengths
           (relay_attn_update_tables)

The format: the d values of a (position, kv head) lie in blocks of 32 that share a power of two, 2^e, and hold one of
0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign.  With a the block's largest magnitude, e is floor(log2 a) - 2, and one more where
a >= 1.75 * 2^floor(log2 a), within -127 .. 125; values round to the nearest (ties to the code that is even) and
saturate at 6; an infinity or a NaN counts as the largest magnitude.  A cache is [num_blocks][kv heads] of
block_size * 17 d / 32 bytes: the codes [block_size][d / 2], the even channel in the low half of a byte and the sign on top
of each half, and behind them e + 127 as [d / 32][block_size] bytes.

Lengths are spread evenly over the case's range and dealt to the requests in an order that depends on the seed, so that
the work of a case does not.  Values are N(0, 1) in bfloat16; physical cache blocks are a random permutation of a
pool with spare blocks.
"""
import math
import random

import torch

own = False

UNUSED_BLOCK = 0x7FFFFFF0       # block-table slots behind a request's last block: never followed
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# What a case holds beside its own entries.
DEFAULTS = {
    "kind": "decode", "batch": 1, "q_heads": 32, "kv_heads": 32, "head_dim": 128, "sys_len": 0,
    "ctx_lo": 0, "ctx_hi": 0,    # context in front of the step's new tokens
    "new_lo": 1, "new_hi": 1,    # new tokens per request
    "block_size": 16,
    "slack": 0,                  # block-table columns beyond the longest request
    "bound": "batch",            # max_context_len: the batch's longest, or "table" (left 0: the capacity)
    "slots": False,              # the rows of append and read named by a slot map instead of tables and lengths
    "fp32_out": False, "lse": False,
    "ended": 0, "back": 0,       # tables: every so manieth request ends / gives back its last tokens (0: none)
    "scarce": False,             # tables: fewer free blocks than the step asks for
}


def listed():
    return [
        # The cache write of a generation step of a grouped-query 8B model: the smallest, launches and latency.
        dict(DEFAULTS, name="append_step", kind="append", batch=32, kv_heads=8, ctx_lo=130, ctx_hi=380, slack=4),
        # The cache write of a burst of prompts on a 13B model, by the slots that the block tables were built with.
        dict(DEFAULTS, name="append_prompts_13b", kind="append", batch=16, q_heads=40, kv_heads=40, ctx_hi=77,
             new_lo=64, new_hi=512, slots=True),
        # A few drafted tokens of requests with 64-wide heads looked at again.
        dict(DEFAULTS, name="read_turns_d64", kind="read", batch=24, kv_heads=8, head_dim=64, ctx_lo=31, ctx_hi=900,
             new_lo=1, new_hi=9, block_size=32, slots=True),
        # A long context that becomes a shared system prompt.
        dict(DEFAULTS, name="read_promote", kind="read", batch=1, kv_heads=8, new_lo=8192, new_hi=8192),
        # One interactive user of a small deployment: the smallest attention call.
        dict(DEFAULTS, name="decode_one", batch=1, kv_heads=8, sys_len=512, ctx_lo=90, ctx_hi=90),
        # A wide batch on a grouped-query 8B model behind a long system prompt.
        dict(DEFAULTS, name="decode_8b_gqa", batch=128, kv_heads=8, sys_len=8192, ctx_lo=63, ctx_hi=1023),
        # Long conversations on the same model: very unequal contexts, the launch bounded by the table capacity only;
        # fp32 output and log-sum-exp for a further merge.
        dict(DEFAULTS, name="decode_long_context", batch=12, kv_heads=8, sys_len=777, ctx_lo=1500, ctx_hi=15000,
             slack=88, bound="table", fp32_out=True, lse=True),
        # A full machine of chats on a 13B model: the context cache is what a step reads.
        dict(DEFAULTS, name="decode_13b_chats", batch=64, q_heads=40, kv_heads=40, sys_len=1024, ctx_lo=300,
             ctx_hi=2500),
        # Drafted tokens to be verified: a few per request over a cached context, 64-wide heads.
        dict(DEFAULTS, name="prompt_drafts_d64", kind="prompt", batch=32, kv_heads=8, head_dim=64, sys_len=600,
             ctx_lo=200, ctx_hi=2100, new_lo=2, new_hi=8, lse=True),
        # A burst of new conversations on a 13B model behind a long system prompt.
        dict(DEFAULTS, name="prompt_13b", kind="prompt", batch=16, q_heads=40, kv_heads=40, sys_len=4096, new_lo=64,
             new_hi=512),
        # The block tables of a generation step: one token each.
        dict(DEFAULTS, name="tables_step", kind="tables", batch=64, ctx_lo=100, ctx_hi=900, slack=8),
        # A busy scheduler: prompts come, drafts are taken back, requests end, and the pool runs dry.
        dict(DEFAULTS, name="tables_busy", kind="tables", batch=1500, ctx_lo=0, ctx_hi=4000, new_lo=1, new_hi=700,
             ended=7, back=3, scarce=True, slack=3),
    ]


# Head layouts met in the tests and the benchmark, and their 64-wide relatives.
_HEADS = ((32, 32, 128), (32, 8, 128), (40, 40, 128), (52, 52, 128), (28, 4, 128), (8, 8, 128),
          (16, 16, 64), (32, 8, 64), (4, 4, 64))


def draw(rng):
    """A case of the ranges the listed ones stand for; no larger than the largest of its kind."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(("append", "read", "decode", "decode", "decode", "prompt", "prompt", "tables"))
        hq, hkv, d = rng.choice(_HEADS)
        case = dict(DEFAULTS, kind=kind, q_heads=hq, kv_heads=hkv, head_dim=d, block_size=rng.choice((8, 16, 16, 32, 64)),
                    slack=rng.choice((0, 3, 40)), batch=log_int(1, {"tables": 2000, "prompt": 48}.get(kind, 256)))
        case["ctx_hi"] = log_int(1, 16384) if rng.random() < 0.85 else 0
        if kind in ("append", "read", "prompt", "tables") and rng.random() < 0.8:
            case["new_hi"] = log_int(1, 1024)
            case["new_lo"] = max(1, int(case["new_hi"] * rng.uniform(0.1, 1.0)))
        case["ctx_lo"] = int(case["ctx_hi"] * rng.uniform(0.0, 1.0))
        if kind in ("append", "read"):
            case["slots"] = rng.random() < 0.5
        if kind in ("decode", "prompt"):
            case.update(sys_len=log_int(100, 16384) if rng.random() < 0.85 else 0, bound=rng.choice(("batch", "table")),
                        fp32_out=rng.random() < 0.25, lse=rng.random() < 0.25)
        if kind == "tables":
            case.update(ended=rng.choice((0, 2, 9)), back=rng.choice((0, 3, 5)), scarce=rng.random() < 0.3)
        most = [work(c) for c in listed() if c["kind"] == kind]
        if all(work(case)[k] <= max(w[k] for w in most) for k in ("bytes", "flops")):
            return case


def _spread(lo, hi, n):
    """n whole numbers spread evenly over lo .. hi, the largest of them hi."""
    return [hi - (hi - lo) * (n - 1 - i) // max(n - 1, 1) for i in range(n)]


def _requests(case):
    """Per request, before the seed's shuffle: its length before and behind the step, and its number of new tokens."""
    c, n = case, case["batch"]
    ctx = _spread(c["ctx_lo"], c["ctx_hi"], n)
    random.Random(n).shuffle(ctx)          # pairs short and long ones; the same for every seed
    got = []
    for i, (old, m) in enumerate(zip(ctx, _spread(c["new_lo"], c["new_hi"], n))):
        if c["ended"] and i % c["ended"] == c["ended"] - 1:
            got.append((old, 0, 0))
        elif c["back"] and i % c["back"] == c["back"] - 1:
            got.append((old, max(0, old - m), 0))
        else:
            got.append((old, old + m, m))
    return got


def _blocks(length, block_size):
    return -(-length // block_size)


def work(case):
    """Bytes and operations of one pass: every input once and every output once."""
    c = case
    hq, hkv, d, bs = c["q_heads"], c["kv_heads"], c["head_dim"], c["block_size"]
    requests = _requests(c)
    tokens = sum(m for _, _, m in requests)
    full, small = 2 * hkv * d * 2, 2 * hkv * d * 17 // 32       # bytes of a position's keys and values
    if c["kind"] == "append":                                    # in, into the cache, out of it again
        return {"bytes": tokens * (2 * full + 2 * small), "flops": tokens * hkv * d * 8}
    if c["kind"] == "read":
        return {"bytes": tokens * (full + small), "flops": tokens * hkv * d * 2}
    if c["kind"] == "tables":
        moved = sum(abs(_blocks(new, bs) - _blocks(old, bs)) for old, new, _ in requests)
        return {"bytes": 16 * len(requests) + 8 * moved + 4 * tokens, "flops": 3 * len(requests)}
    nbytes = tokens * hq * d * (2 + (4 if c["fp32_out"] else 2)) + (4 * tokens * hq if c["lse"] else 0)
    nbytes += full * c["sys_len"] + small * sum(new for _, new, _ in requests)
    pairs = sum(m * (c["sys_len"] + old) + m * (m + 1) // 2 for old, _, m in requests)
    return {"bytes": nbytes, "flops": 4 * d * hq * pairs}


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)


def _codes(x):
    """The 4-bit codes and the scale bytes of x [..., d] in bfloat16."""
    blocks = x.unflatten(-1, (-1, 32))
    bits = blocks.view(torch.int16).to(torch.int32)
    mag = bits & 0x7FFF
    top = mag.amax(-1)
    byte = ((top >> 7) + ((top & 0x7F) >= 0x60) - 2).clamp(0, 252)
    # |x| in units of 2^(byte - 127); both powers of two are whole, and the product is exact
    unit = ((254 - byte).clamp(min=1) << 23).view(torch.float32)
    y = torch.where(mag > 0x7F80, math.inf, blocks.float().abs()) * unit[..., None]
    code = sum((y > t).to(torch.int32) for t in (0.25, 1.25, 2.5, 5.0)) + sum((y >= t).to(torch.int32) for t in (0.75, 1.75, 3.5))
    return (code | torch.where(bits < 0, 8, 0)).flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def _parts(cache, bs, d):
    """A cache's codes [num_blocks, kv heads, block_size, d / 2] and scale bytes [num_blocks, kv heads, d / 32, block_size]."""
    at = bs * d // 2
    return cache[..., :at].unflatten(-1, (bs, d // 2)), cache[..., at:].unflatten(-1, (d // 32, bs))


def _values(packed, scale, magnitudes):
    """The values, in 32 bits, that codes [..., d / 2] and scale bytes [..., d / 32] stand for."""
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    v = magnitudes[code.to(torch.int32)].unflatten(-1, (-1, 32))
    byte = scale.to(torch.int32)
    unit = (byte.clamp(min=1) << 23).view(torch.float32) * torch.where(byte == 0, 0.5, 1.0)
    return (v * unit[..., None]).flatten(-2)


def prepare(case, seed):
    """What the serving program holds before the call: caches, block tables and lengths of the batch, queries or new
    keys/values, output buffers, and what a call of the library needs beside them."""
    c = case
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hq, hkv, d, n, bs = c["q_heads"], c["kv_heads"], c["head_dim"], c["batch"], c["block_size"]
    requests = _requests(c)
    rng.shuffle(requests)
    old, lens, new = (list(x) for x in zip(*requests))
    tokens = sum(new)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    tables_hold = old if c["kind"] == "tables" else lens
    blocks = [_blocks(length, bs) for length in tables_hold]
    spare = sum(blocks) // 10 + 1
    if c["kind"] == "tables":              # what the step asks for, or a good half of it
        wanted = sum(max(0, _blocks(b, bs) - _blocks(a, bs)) for a, b in zip(old, lens))
        spare = wanted * 6 // 10 if c["scarce"] else wanted + wanted // 4 + 1
    pool = sum(blocks) + spare
    ids = list(range(pool))
    rng.shuffle(ids)
    width = max(_blocks(max(a, b), bs) for a, b in zip(old, lens)) + c["slack"]
    rows, at = [], 0
    for used in blocks:
        rows.append(ids[at:at + used] + [UNUSED_BLOCK] * (width - used))
        at += used
    state = dict(c, tokens=tokens, max_new=max(new), tables=i32(rows), lens=i32(lens), max_len=max(lens),
                 magnitudes=torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device="cuda"))
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    if c["kind"] == "tables":
        state.update(old=i32(old), free=i32(ids[at:] + [UNUSED_BLOCK] * at), pool=i32([spare, 0]), pool_out=i32([0, 0]),
                     granted=i32([0] * n), starts=i32([0] * (n + 1)), slots_out=i32([0] * tokens))
        if own:
            import paper_2402_14808_amd as ra
            state["params"] = ra.make_table_params(state["tables"], num_blocks=pool, block_size=bs)
        return state
    state["starts"] = i32(starts)
    token = torch.arange(tokens, device="cuda")
    owner = torch.searchsorted(state["starts"][1:].contiguous(), token, right=True)
    pos = state["lens"][owner] - state["starts"][owner + 1] + token
    state["slot_map"] = (state["tables"][owner, pos // bs] * bs + pos % bs).to(torch.int32) if c["slots"] else None
    shape = (pool, hkv, bs * d * 17 // 32)
    state["k_cache"], state["v_cache"] = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    for cache in (state["k_cache"], state["v_cache"]):
        codes, scales = _parts(cache, bs, d)
        step = max(1, (1 << 27) // (hkv * bs * d))
        for first in range(0, pool, step):
            part = slice(first, min(pool, first + step))
            code, byte = _codes(_normal(gen, part.stop - first, hkv, bs, d))
            codes[part] = code[..., 0::2] | code[..., 1::2] << 4
            scales[part] = byte.transpose(-1, -2)
    if c["kind"] in ("append", "read"):
        state["k_new"], state["v_new"] = _normal(gen, tokens, hkv, d), _normal(gen, tokens, hkv, d)
        state["k_out"], state["v_out"] = torch.zeros_like(state["k_new"]), torch.zeros_like(state["v_new"])
        q = out = state["k_new"]
    else:
        # (token rows padded by 384 bytes over a multiple of 1024, the layout recommended for system caches)
        stride = -(-(hkv * d - 192) // 512) * 512 + 192
        for name in ("k_sys", "v_sys"):
            flat = torch.zeros(max(1, c["sys_len"]) * stride, dtype=torch.bfloat16, device="cuda")
            state[name] = flat.as_strided((c["sys_len"], hkv, d), (stride, d, 1))
            state[name].copy_(_normal(gen, c["sys_len"], hkv, d))
        q = state["q"] = _normal(gen, tokens, hq, d)
        out = state["out"] = torch.empty(tokens, hq, d, device="cuda", dtype=torch.float32 if c["fp32_out"] else torch.bfloat16)
        state["lse_out"] = torch.empty(tokens, hq, device="cuda") if c["lse"] else None
    if own:
        import paper_2402_14808_amd as ra
        state["params"] = ra.make_params(q, out, state.get("k_sys"), state["k_cache"], state["tables"], batch=n,
                                         softmax_scale=1.0 / math.sqrt(d), max_context_len=max(lens) if c["bound"] == "batch" else 0)
        if c["kind"] in ("decode", "prompt"):
            nbytes = ra.relay_attn_workspace_bytes(state["params"], tokens)
            state["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return state


def _run_own(s):
    import paper_2402_14808_amd as ra
    if s["kind"] == "tables":
        ra.relay_attn_update_tables(s["params"], s["old"], s["lens"], s["pool"], s["pool_out"], s["free"], s["tables"], s["granted"],
                                    s["starts"], s["slots_out"])
        return s["tables"], s["granted"], s["starts"], s["slots_out"], s["pool_out"], s["free"]
    p, caches = s["params"], (s["k_cache"], s["v_cache"])
    if s["kind"] in ("append", "read"):
        where = (s["starts"], s["tokens"], *caches, s["tables"], s["lens"])
        if s["kind"] == "append":
            ra.relay_attn_cache_append_fp4(p, s["k_new"], s["v_new"], *where, slot_map=s["slot_map"])
        ra.relay_attn_cache_read_fp4(p, s["k_out"], s["v_out"], *where, slot_map=s["slot_map"])
        return s["k_out"], s["v_out"]
    paged = (*caches, s["tables"], s["lens"], s["out"], s["lse_out"], s["workspace"])
    if s["kind"] == "decode":
        ra.relay_attn_decode_fp4(p, s["q"], s["k_sys"], s["v_sys"], *paged)
    else:
        ra.relay_attn_prefill_fp4(p, s["q"], s["starts"], s["tokens"], s["max_new"], s["k_sys"], s["v_sys"], *paged)
    return s["out"], s["lse_out"]


def _place(s):
    """Block and offset of each packed new token, from the slot map or from lengths and tables."""
    bs = s["block_size"]
    if s["slot_map"] is not None:
        slot = s["slot_map"].long()
        return slot // bs, slot % bs
    token = torch.arange(s["tokens"], device="cuda")
    owner = torch.searchsorted(s["starts"][1:].contiguous(), token, right=True)
    pos = s["lens"][owner] - s["starts"][owner + 1] + token
    return s["tables"][owner, pos // bs].long(), pos % bs


def _run_rows(s):
    """append and read: the new rows rounded and packed into the caches; what the caches hold of them."""
    bs, d = s["block_size"], s["head_dim"]
    block, off = _place(s)
    def through(cache, fresh):
        codes, scales = _parts(cache, bs, d)
        if s["kind"] == "append":
            code, byte = _codes(fresh)
            codes[block, :, off] = code[..., 0::2] | code[..., 1::2] << 4
            scales[block, :, :, off] = byte
        return _values(codes[block, :, off], scales[block, :, :, off], s["magnitudes"]).to(torch.bfloat16)
    return through(s["k_cache"], s["k_new"]), through(s["v_cache"], s["v_new"])


def _run_tables(s):
    """Requests in order: ends and shrinking requests put their blocks on top of the pool's stack, growing ones take from
    the top, as long as the pool holds everything asked for so far."""
    bs, n = s["block_size"], s["batch"]
    width, pool = s["tables"].shape[1], s["free"].shape[0]
    old, new, held = s["old"].long(), s["lens"].long(), s["pool"][0].long()
    had, want = (old + bs - 1) // bs, (new + bs - 1) // bs
    need, back = (want - had).clamp(min=0), (had - want).clamp(min=0)
    top = held + back.sum()
    through = need.cumsum(0)
    served = (need == 0) | (through <= top)
    taken = torch.where(served, need, 0)
    granted = torch.where(served, new, old)
    # the stack with the released blocks on top: release k lies at held + k, allocation k takes top - 1 - k
    column = torch.arange(width, device="cuda")
    leaving = (column >= want[:, None]) & (column < had[:, None])
    stack = torch.cat((s["free"], s["free"].new_full((1,), -1))).long()
    rank = (back.cumsum(0) - back)[:, None] + column - want[:, None]
    stack_ext = torch.full((pool + int(s["batch"]) * width + 1,), -1, dtype=torch.long, device="cuda")
    stack_ext[:pool] = s["free"].long()
    stack_ext[torch.where(leaving, held + rank, pool + n * width)] = s["tables"].long()
    coming = (column >= had[:, None]) & (column < (had + taken)[:, None])
    k = (taken.cumsum(0) - taken)[:, None] + column - had[:, None]
    tables = torch.where(coming, stack_ext[(top - 1 - k).clamp(min=0)], s["tables"].long()).to(torch.int32)
    left = top - taken.sum()
    place = torch.arange(pool, device="cuda")
    free = torch.where((place >= held) & (place < left), stack_ext[:pool], stack[:pool]).to(torch.int32)
    more = (new - old).clamp(min=0)
    starts = torch.cat((more.new_zeros(1), more.cumsum(0)))
    token = torch.arange(s["tokens"], device="cuda")
    owner = torch.searchsorted(starts[1:].contiguous(), token, right=True)
    pos = old[owner] + token - starts[owner]
    slots = torch.where(served[owner], tables[owner, pos // bs].long() * bs + pos % bs, -1)
    s["tables"].copy_(tables)
    s["free"].copy_(free)
    pool_out = torch.stack((left, (~served).sum()))
    return s["tables"], *(x.to(torch.int32) for x in (granted, starts, slots, pool_out)), s["free"]


def _run_attention(s):
    """Attention over [system ; context] with every request padded to the longest, in 32 bits."""
    bs, d, hkv, n, m = s["block_size"], s["head_dim"], s["kv_heads"], s["batch"], s["max_new"]
    group = s["q_heads"] // hkv
    used = -(-s["max_len"] // bs)
    first, count = s["starts"][:-1].long(), s["starts"].diff().long()
    step = torch.arange(m, device="cuda")
    row = (first[:, None] + step).clamp(max=s["tokens"] - 1)                     # [n, m]
    q = s["q"][row].float().unflatten(2, (hkv, group)).permute(0, 2, 1, 3, 4).reshape(n, hkv, m * group, d)
    scale = 1.0 / math.sqrt(d)
    blocks = s["tables"][:, :used].long()
    blocks = torch.where(torch.arange(used, device="cuda") * bs < s["lens"][:, None], blocks, 0)

    def gathered(cache):
        codes, scales = _parts(cache, bs, d)
        v = _values(codes[blocks], scales[blocks].transpose(-1, -2), s["magnitudes"])
        return v.permute(0, 2, 1, 3, 4).flatten(2, 3)                           # [n, kv heads, used * bs, d]

    k_sys, v_sys = (x.float().permute(1, 0, 2).contiguous() for x in (s["k_sys"], s["v_sys"]))
    scores_sys = torch.matmul(q.transpose(0, 1).reshape(hkv, -1, d), k_sys.transpose(1, 2).contiguous())
    scores_sys = scores_sys.unflatten(1, (n, m * group)).transpose(0, 1)
    scores_ctx = torch.matmul(q, gathered(s["k_cache"]).transpose(2, 3).contiguous())
    last = (s["lens"].long() - count)[:, None] + step                            # the last position that a new token sees
    seen = torch.arange(used * bs, device="cuda") <= last.repeat_interleave(group, 1)[..., None]
    scores = torch.cat((scores_sys, scores_ctx.masked_fill_(~seen[:, None], -math.inf)), -1).mul_(scale)
    del scores_sys, scores_ctx
    top = scores.amax(-1, keepdim=True)
    weight = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight[..., s["sys_len"]:], torch.where(seen[:, None, -1:].transpose(2, 3), gathered(s["v_cache"]), 0.0))
    out += torch.matmul(weight[..., :s["sys_len"]].transpose(0, 1).reshape(hkv, n * m * group, -1), v_sys).unflatten(1, (n, m * group)).transpose(0, 1)
    out = out / torch.where(total == 0, 1.0, total)
    lse = (top + total.log())[..., 0]
    mine = step < count[:, None]
    out = out.unflatten(2, (m, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)[mine]
    lse = lse.unflatten(2, (m, group)).permute(0, 2, 1, 3).flatten(2, 3)[mine]
    return out.to(torch.float32 if s["fp32_out"] else torch.bfloat16), lse if s["lse"] else None


def run(state):
    """One operator of one layer's step."""
    if own:
        return _run_own(state)
    if state["kind"] == "tables":
        return _run_tables(state)
    return _run_rows(state) if state["kind"] in ("append", "read") else _run_attention(state)


def _held(cache, block, off, bs, d):
    """The values of rows (block, off) [...] of a cache in 64 bits, [..., kv heads, d]."""
    at = bs * d // 2
    lane = torch.arange(d, device="cuda")
    byte = cache[block][..., :at].reshape(*block.shape, -1, bs, d // 2)
    byte = torch.gather(byte, -2, off[..., None, None, None].expand(*block.shape, byte.shape[-3], 1, d // 2))[..., 0, :]
    code = (byte[..., lane // 2].long() >> (4 * (lane % 2))) & 15
    exponent = cache[block][..., at:].reshape(*block.shape, -1, d // 32, bs)
    exponent = torch.gather(exponent, -1, off[..., None, None, None].expand(*block.shape, exponent.shape[-3], d // 32, 1))[..., 0]
    table = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    v = table[code & 7] * (1 - 2 * (code >> 3)).double()
    return v * torch.pow(2.0, exponent[..., lane // 32].double() - 127)


def _nearest(x):
    """x [..., d] as the format holds it, in 64 bits: the exponent of each block, and the nearest multiple of the step at
    each value's place (half steps go to the even one)."""
    blocks = x.double().unflatten(-1, (-1, 32))
    fraction, exponent = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    unit = torch.pow(2.0, (exponent - 3 + (fraction >= 0.875)).clamp(-127, 125).double())
    y = blocks.abs() / unit
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    return (torch.clamp(torch.round(y / step) * step, max=6) * unit * torch.sign(blocks)).flatten(-2)


def exact(case, seed):
    """What run() returns for the inputs of this seed, from the definitions in 64 bits."""
    c = case
    if c["kind"] == "tables":
        return None
    s = prepare(case, seed)
    hq, hkv, d, bs = c["q_heads"], c["kv_heads"], c["head_dim"], c["block_size"]
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    if c["kind"] == "append":
        return _nearest(s["k_new"]), _nearest(s["v_new"])
    if c["kind"] == "read":
        rows = []
        for i, length in enumerate(lens):
            pos = torch.arange(length - (starts[i + 1] - starts[i]), length, device="cuda")
            rows.append((s["tables"][i].long()[pos // bs], pos % bs))
        block, off = (torch.cat(x) for x in zip(*rows))
        return _held(s["k_cache"], block, off, bs, d), _held(s["v_cache"], block, off, bs, d)
    out = torch.zeros(s["tokens"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], hq), -math.inf, dtype=torch.float64, device="cuda")
    for i, length in enumerate(lens):
        m, rows = starts[i + 1] - starts[i], slice(starts[i], starts[i + 1])
        pos = torch.arange(length, device="cuda")
        block, off = s["tables"][i].long()[pos // bs], pos % bs
        keys, values = (torch.cat((s[a].double(), _held(s[b], block, off, bs, d)))
                        for a, b in (("k_sys", "k_cache"), ("v_sys", "v_cache")))
        if len(keys) == 0 or m == 0:
            continue
        hidden = torch.ones(m, len(keys), dtype=torch.bool, device="cuda").triu(len(keys) - m + 1)
        for g in range(hkv):
            heads = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            q, k, v = s["q"][rows, heads].double(), keys[:, g], values[:, g]
            scores = (torch.matmul(q, k.t().contiguous()) / math.sqrt(d)).masked_fill_(hidden[:, None], -math.inf)
            lse[rows, heads] = torch.logsumexp(scores, -1)
            out[rows, heads] = torch.matmul(torch.softmax(scores, -1), v)
    return out, lse if c["lse"] else None
