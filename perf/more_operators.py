"""Measurable cases of rotating appends and of the 4-bit pages: keys and values
put into a paged cache with the position rotation applied on the way
(page_append), attention over pages of 4-bit codes (page_attend) and the way back
to a K/V cache (page_read).

A 4-bit row, one position of one head, is codes c = 0 .. 15, two a byte (the even
dimension in the low half), and two bfloat16 numbers: its step and its middle.  A
code stands for middle + (c - 7.5) step.

Shapes are those of the repository's own configurations: GPT-2-shaped (12 heads
x 64, 1024 positions) and Llama-3-8B-shaped (8 KV heads x 128, up to 131072
positions, 64 sequences a decode step), with four query heads a KV head for the
latter.  Each pass works on one layer.

`own` false: the plain form, elementary torch operations in 32 bits, rounded
once at the end.  `own` true: the library's calls.
"""
import functools
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "uint4": torch.uint8}
FLOOR = 2.0 ** -100          # the smallest scale of a page, and step of a row
MOST = 2.0 ** 102            # the largest magnitude of a 4-bit row


# ------------------------------------------------------------------ cases --
def _append(name, n_req, heads, group, dim, rot, pairs, block, dtype, fmt, lo, hi, new_lo, new_hi):
    """new_lo..new_hi new positions after lo..hi cached ones; pairs: dimensions 2i and 2i + 1 turn together, else i and
    i + rot / 2, of the first rot ones."""
    return dict(name=name, op="append", n_req=n_req, heads=heads, group=group, dim=dim, rot=rot, pairs=pairs,
                block=block, dtype=dtype, fmt=fmt, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi)


def _attend(name, n_req, heads, group, dim, block, dtype, lo, hi, new_lo, new_hi, window=0, sinks=0, softcap=0.0,
            bias=False, prefix=0, causal=True, by_token=False):
    """lo..hi positions before the new ones; by_token: pages laid out [block][token][head][dim]."""
    return dict(name=name, op="attend", n_req=n_req, heads=heads, group=group, dim=dim, block=block, dtype=dtype,
                fmt="uint4", lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, window=window, sinks=sinks, softcap=softcap,
                bias=bias, prefix=prefix, causal=causal, by_token=by_token)


def _read(name, n_req, heads, dim, block, dtype, lo, hi, t0, t1):
    return dict(name=name, op="read", n_req=n_req, heads=heads, dim=dim, block=block, dtype=dtype, fmt="uint4", lo=lo,
                hi=hi, t0=t0, t1=t1)


def listed():
    return [
        # a decode step's queries and keys turned to their positions, the keys and values into 8-bit pages (latency)
        _append("append_step_llama_e4m3", 64, 8, 4, 128, 128, False, 32, "bf16", "e4m3", 1, 32000, 1, 1),
        # several drafted positions a sequence, into 4-bit pages
        _append("append_drafts_llama_uint4", 24, 8, 4, 128, 128, False, 16, "f16", "uint4", 1, 16000, 2, 7),
        # ragged GPT-2-shaped prompts, half of each head turned, neighbouring dimensions together
        _append("append_prompts_gpt2_int8", 13, 12, 1, 64, 32, True, 16, "f16", "int8", 0, 23, 1, 1000),
        # Llama-shaped prompts into 4-bit pages
        _append("append_prompts_llama_uint4", 9, 8, 4, 128, 128, False, 64, "bf16", "uint4", 0, 700, 1000, 8192),
        # one decode step of a small GPT-2-shaped batch (latency)
        _attend("step_gpt2_uint4", 8, 12, 1, 64, 16, "f16", 40, 1023, 1, 1),
        # one decode step of 64 long Llama-shaped sequences: the cache's bandwidth
        _attend("step_llama_uint4", 64, 8, 4, 128, 32, "bf16", 16000, 32767, 1, 1),
        # a single very long sequence: the work has to be split along the positions; capped scores
        _attend("step_long_uint4", 1, 8, 4, 128, 64, "bf16", 131071, 131071, 1, 1, softcap=30.0),
        # several drafted positions a sequence checked at once; sinks and a sliding window, a bias by distance
        _attend("drafts_window_uint4", 24, 8, 4, 128, 16, "f16", 3000, 16000, 2, 7, window=4096, sinks=4, bias=True,
                by_token=True),
        # ragged GPT-2-shaped prompts whose first positions see one another (prefix mask)
        _attend("prompts_gpt2_prefix_uint4", 13, 12, 1, 64, 16, "f16", 0, 0, 1, 1000, prefix=100),
        # a long Llama-shaped prompt taken in pieces: the pieces' tokens against all that is cached
        _attend("prompt_llama_piece_uint4", 2, 8, 4, 128, 64, "bf16", 12000, 12288, 4000, 4096),
        # a GPT-2-shaped batch read back for the archive
        _read("read_gpt2_uint4", 8, 12, 64, 16, "f16", 500, 1024, 4, 992),
        # Llama-shaped sequences read back for the archive
        _read("read_llama_uint4", 4, 8, 128, 32, "bf16", 9000, 32768, 4, 32736),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "read"])
    heads, dim = rng.choice([(12, 64), (8, 128), (rng.randint(1, 9), 128), (rng.randint(1, 13), 64)])
    block, dtype, group = rng.choice([16, 32, 48, 64, 128]), rng.choice(["f16", "bf16"]), rng.choice([1, 2, 3, 4, 8])
    if op == "append":
        n, hi = _log(rng, 1, 64), _log(rng, 1, 30000)
        new = rng.choice([1, _log(rng, 1, max(1, min(8192, 20000 // n)))])
        return _append("", n, heads, group, dim, 16 * rng.randint(1, dim // 16), rng.random() < 0.3, block,
                       rng.choice(["f16", "bf16", "f32"]), rng.choice(["uint4", "uint4", "e4m3", "int8"]), 0, hi,
                       0 if new > 1 else 1, new)
    if op == "read":
        n, hi = _log(rng, 1, 8), _log(rng, 64, 16384)
        t0 = rng.randint(0, hi // 4)
        return _read("", n, heads, dim, block, rng.choice(["f16", "bf16", "f32"]), hi // 3, hi, t0,
                     rng.randint(t0 + 1, hi))
    how = rng.choice(["step", "drafts", "prompts"])
    most = {"step": 400000, "drafts": 200000, "prompts": 12000}[how]       # positions of all sequences
    n = _log(rng, 1, 64 if how != "prompts" else 8)
    hi = _log(rng, 16, max(17, min(131071, most // n)))
    new = {"step": 1, "drafts": rng.randint(2, 16), "prompts": rng.randint(17, max(18, min(2048, hi)))}[how]
    window = rng.choice([0, 0, _log(rng, 16, 4096)])
    return _attend("", n, heads, group, dim, block, dtype, hi // 2, hi, 0 if how == "prompts" else 1, new, window,
                   4 if window else 0, rng.choice([0.0, 0.0, 20.0]), rng.random() < 0.3,
                   rng.choice([0, 0, rng.randint(1, 200)]), rng.random() < 0.9, rng.random() < 0.3)


# ----------------------------------------------------------------- inputs --
def _lengths(case):
    """Positions in the cache and new ones of every request, host lists (the sizes are the case's, not the seed's)."""
    g = torch.Generator().manual_seed(case["n_req"] * 7919 + case["hi"] * 31 + case["lo"])
    n = case["n_req"]
    # the lengths' first and last values are always met
    length = torch.randint(case["lo"], case["hi"] + 1, (n,), generator=g)
    length[0] = case["hi"]
    lo, hi = case.get("new_lo", 0), case.get("new_hi", 0)
    new = torch.randint(lo, hi + 1, (n,), generator=g)
    new[-1] = hi
    return length.tolist(), new.tolist()


def _blocks(tokens, block):
    return (tokens + block - 1) // block


def _table(lengths, block, n_blocks, width, g):
    """Blocks scattered over the pool: a block table whose unused entries are -1."""
    ids = torch.randperm(n_blocks, generator=g, device="cuda").to(torch.int32)
    need = torch.tensor([_blocks(t, block) for t in lengths], device="cuda")
    start = torch.cumsum(need, 0) - need
    col = torch.arange(width, device="cuda")
    at = (start[:, None] + col).clamp(max=n_blocks - 1)
    return torch.where(col < need[:, None], ids[at], torch.full_like(ids[at], -1)).contiguous()


def _pool(case, n_blocks, g):
    """Codes as quantised activations have them, with scales of their own; slots never written hold any bytes."""
    H, B, D, fmt = case["heads"], case["block"], case["dim"], case["fmt"]
    shape = (n_blocks, B, H, D) if case.get("by_token") else (n_blocks, H, B, D)
    pools, scales = [], []
    for _ in range(2):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)
        if fmt == "uint4":
            c = x.mul_(3.2).add_(7.5).round_().clamp_(0.0, 15.0).to(torch.uint8)
            c = c[..., ::2] | c[..., 1::2] << 4
            step = torch.exp(torch.randn((n_blocks, H, B), generator=g, device="cuda") * 0.3) / 3.2
            mid = torch.randn((n_blocks, H, B), generator=g, device="cuda") * 0.3
            s = torch.stack([step, mid], -1).to(torch.bfloat16)
        elif fmt == "e4m3":
            c = x.mul_(100.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
            s = torch.exp2(torch.randint(-9, -5, (n_blocks, H), generator=g, device="cuda").float())
        else:
            c = x.mul_(32.0).round_().clamp_(-127.0, 127.0).to(torch.int8)
            s = torch.exp(torch.randn((n_blocks, H), generator=g, device="cuda") * 0.3) / 32
        pools.append(c.permute(0, 2, 1, 3) if case.get("by_token") else c)
        scales.append(s)
    return pools[0], pools[1], scales[0], scales[1]


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


@functools.lru_cache(None)
def _context():
    import paper_2607_07144_gb300 as fkv
    return fkv.Context(256)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    length, new = _lengths(case)
    n, B, op = case["n_req"], case["block"], case["op"]
    state = dict(case=case, op=op, block=B)
    after = [l + v for l, v in zip(length, new)]
    width = max(1, max(_blocks(t, B) for t in after))
    n_blocks = sum(_blocks(t, B) for t in after) + 3
    table = _table(after, B, n_blocks, width, g)
    k, v, ks, vs = _pool(case, n_blocks, g)
    state.update(k=k, v=v, k_scale=ks, v_scale=vs)
    if own:
        import paper_2607_07144_gb300 as fkv
        state["pages"] = fkv.Pages(k, v, ks, vs)
    H, D, dt = case["heads"], case["dim"], DTYPES[case["dtype"]]
    if op == "read":
        shape = (1, n, H, max(case["t1"], case["hi"]), D)
        state.update(kv_len=_ints(length), table=table, t0=case["t0"], t1=case["t1"],
                     k_out=torch.zeros(shape, dtype=dt, device="cuda"), v_out=torch.zeros(shape, dtype=dt, device="cuda"))
        return state
    T, Hq = sum(new), H * case["group"]
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    if op == "append":
        req = torch.repeat_interleave(torch.arange(n, device="cuda"), _ints(new))
        p = _ints(length)[req] + torch.arange(T, device="cuda") - _ints(cu)[req]
        slots = table[req, (p // B)].long() * B + p % B
        # a fused projection's rows: queries, keys, values
        chan = torch.exp(torch.randn((1, Hq + 2 * H, D), generator=g, device="cuda") * 0.5)
        x = (torch.randn((T, Hq + 2 * H, D), generator=g, device="cuda") * chan).to(dt)
        half = case["rot"] // 2
        freq = 10000.0 ** (torch.arange(half, dtype=torch.float64, device="cuda") / -half)
        angle = torch.arange(max(after), dtype=torch.float64, device="cuda")[:, None] * freq
        state.update(slots=slots, positions=p.int(), q=x[:, :Hq], x_k=x[:, Hq:Hq + H], x_v=x[:, Hq + H:],
                     cos=torch.cos(angle).float(), sin=torch.sin(angle).float(),
                     q_out=torch.empty((T, Hq, D), dtype=dt, device="cuda"))
        return state
    q = torch.randn((T, Hq, D), generator=g, device="cuda").to(dt)
    state.update(q=q, cu=_ints(cu), kv_len=_ints(after), table=table, max_new=max(new), max_len=max(after),
                 out=torch.empty_like(q), lse=torch.empty((T, Hq), dtype=torch.float32, device="cuda"),
                 slopes=torch.exp2(-8.0 * (torch.arange(Hq, device="cuda") + 1) / Hq) if case["bias"] else None,
                 prefix=_ints([min(case["prefix"], t) for t in after]) if case["prefix"] else None)
    return state


# ------------------------------------------------------------ plain forms --
def _plain_turn(s, x):
    """x [T, heads, D] in float32, its first rot dimensions turned by the angles of the tokens' positions."""
    c, x = s["case"], x.float()
    rot, p = c["rot"], s["positions"].long()
    cos, sin = s["cos"][p][:, None], s["sin"][p][:, None]
    a, b = (x[..., :rot:2], x[..., 1:rot:2]) if c["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, z = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([y, z], -1).flatten(-2) if c["pairs"] else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_put4(codes, scale, x, slots):
    """Rows x [T, H, D] into their slots; codes and scale are updated in place."""
    B = codes.shape[2]
    x = x.float().clamp(-MOST, MOST)
    lo, hi = x.amin(-1), x.amax(-1)
    mid = (lo * 0.5 + hi * 0.5).to(torch.bfloat16).float()
    reach = torch.maximum(hi - mid, mid - lo)
    # a step that reaches the outermost value in 7.5, rounded up to bfloat16
    up = (reach * (2.0 / 15.0)).view(torch.int32) + 0xffff >> 16 << 16
    step = torch.maximum(up.view(torch.float32), mid.abs() * 2.0 ** -16).clamp(min=FLOOR)
    inv = 1.0 / step
    c = torch.round((x - mid[..., None]) * inv[..., None] + 7.5).clamp(0.0, 15.0).to(torch.uint8)
    blk, off = slots // B, slots % B
    codes[blk, :, off] = c[..., ::2] | c[..., 1::2] << 4
    scale[blk, :, off] = torch.stack([step, mid], -1).to(torch.bfloat16)


def _plain_put8(codes, scale, x, tok, new, old, blk):
    """The touched blocks [L, B, H, D] of one of the two pools, quantised; codes and scale are updated in place."""
    e4m3 = codes.dtype == torch.float8_e4m3fn
    byte = codes.view(torch.int8) if e4m3 else codes
    x = x[tok].float()
    fresh = new[:, :, None, None]
    amax = torch.where(fresh & torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax((1, 3))            # [L, H]
    if e4m3:
        # the smallest power of two that brings amax to 448 = 1.75 2^8 or less
        m, e = torch.frexp(amax)
        want = ((e - 9 + (m > 0.875)).clamp(min=-100) + 127 << 23).view(torch.float32)
    else:
        want = amax / torch.full_like(amax, 127.0)
    want = torch.where(amax > 0, want, torch.zeros_like(want)).clamp(min=FLOOR)
    has = old.any(1)[:, None]
    was = torch.where(has, scale[blk], torch.zeros_like(want))
    now = torch.maximum(was, want)
    inv = 1.0 / now
    kept = byte[blk].transpose(1, 2)                                                                    # [L, B, H, D]
    grown = (kept.contiguous().view(codes.dtype).float() * (was * inv)[:, None, :, None])
    y = torch.where(fresh, x * inv[:, None, :, None], grown)
    if e4m3:
        q = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.int8)
    else:
        q = torch.round(y).clamp(-127.0, 127.0).to(torch.int8)
    touch = (new | (old & has))[:, :, None, None]
    byte[blk] = torch.where(touch, q, kept).transpose(1, 2)
    scale[blk] = now


def _plain_append(s):
    B, slots = s["block"], s["slots"]
    s["q_out"].copy_(_plain_turn(s, s["q"]))
    x_k = _plain_turn(s, s["x_k"])
    if s["case"]["fmt"] == "uint4":
        _plain_put4(s["k"], s["k_scale"], x_k, slots)
        _plain_put4(s["v"], s["v_scale"], s["x_v"], slots)
        return [s["q_out"], s["k"], s["v"], s["k_scale"], s["v_scale"]]
    T = slots.numel()
    before = torch.cat([slots.new_full((1,), -2), slots[:-1]])
    lead = torch.nonzero((slots % B == 0) | (before != slots - 1))[:, 0]
    row = torch.arange(B, device=slots.device)
    off, blk = slots[lead] % B, slots[lead] // B
    tok = lead[:, None] + row - off[:, None]
    new = (row >= off[:, None]) & (tok < T)
    tok = tok.clamp(0, max(T - 1, 0))
    new = new & (slots[tok] == blk[:, None] * B + row)
    old = row < off[:, None]
    _plain_put8(s["k"], s["k_scale"], x_k, tok, new, old, blk)
    _plain_put8(s["v"], s["v_scale"], s["x_v"], tok, new, old, blk)
    return [s["q_out"], s["k"], s["v"], s["k_scale"], s["v_scale"]]


def _plain_rows(codes, scale, table, tokens):
    """Values [n, H, tokens, D] in float32 of the first `tokens` positions of every request."""
    B, H = codes.shape[2], codes.shape[1]
    ids = table[:, :_blocks(tokens, B)].long().clamp(min=0)
    c, f = codes[ids], scale[ids].float()                                                # [n, blocks, H, B, ...]
    x = torch.stack([c & 15, c >> 4], -1).flatten(-2).float()
    x = x.sub_(7.5).mul_(f[..., :1]).add_(f[..., 1:])
    return x.transpose(1, 2).reshape(ids.shape[0], H, -1, x.shape[-1])[:, :, :tokens]


def _plain_attend(s):
    c, q, cu, length = s["case"], s["q"], s["cu"].long(), s["kv_len"].long()
    n, H, G, D, M, N = c["n_req"], c["heads"], c["group"], c["dim"], s["max_new"], s["max_len"]
    T = q.shape[0]
    i, j = torch.arange(M, device=q.device), torch.arange(N, device=q.device)
    tok = (cu[:n, None] + i).clamp(max=T - 1)                                            # [n, M]
    p = (length - (cu[1:] - cu[:n]))[:, None] + i
    rows = q[tok].float().reshape(n, M, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, M * G, D)
    k = _plain_rows(s["k"], s["k_scale"], s["table"], N)
    x = torch.matmul(rows, k.transpose(2, 3)).reshape(n, H, M, G, N)
    del k
    x *= 1.0 / math.sqrt(D)
    if c["softcap"]:
        x = torch.tanh_(x.div_(c["softcap"])).mul_(c["softcap"])
    j, pp = j[None, None, :], p[:, :, None]
    if s["slopes"] is not None:
        x += s["slopes"].reshape(1, H, 1, G, 1) * (j - pp).float().reshape(n, 1, M, 1, N)
    seen = torch.ones((n, M, N), dtype=torch.bool, device=q.device)
    if c["causal"]:
        seen &= j <= pp
    if c["window"]:
        seen &= j > pp - c["window"]
        seen |= j < c["sinks"]
        if c["causal"]:
            seen &= j <= pp
    if s["prefix"] is not None:
        seen |= j < s["prefix"][:, None, None]
    seen &= (j < length[:, None, None]) & (pp >= 0)
    x.masked_fill_(~seen.reshape(n, 1, M, 1, N), -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    x = torch.exp_(x.sub_(m))
    total = x.sum(-1, keepdim=True)
    v = _plain_rows(s["v"], s["v_scale"], s["table"], N)
    v = torch.where((j[0, 0] < length[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = torch.matmul(x.reshape(n, H, M * G, N), v).reshape(n, H, M, G, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (m + torch.log(total))[..., 0]
    t = torch.arange(T, device=q.device)
    r = torch.searchsorted(cu, t, right=True) - 1
    o = o.permute(0, 2, 1, 3, 4).reshape(n, M, H * G, D)[r, t - cu[r]]
    lse = lse.permute(0, 2, 1, 3).reshape(n, M, H * G)[r, t - cu[r]]
    return [o.to(q.dtype), lse]


def _plain_read(s):
    t0, t1 = s["t0"], s["t1"]
    live = (torch.arange(t0, t1, device="cuda") < s["kv_len"][:, None])[:, None, :, None]
    wide = min(t1, s["table"].shape[1] * s["block"])
    k = _plain_rows(s["k"], s["k_scale"], s["table"], wide)[:, :, t0:]
    v = _plain_rows(s["v"], s["v_scale"], s["table"], wide)[:, :, t0:]
    live = live[:, :, :k.shape[2]]
    to = slice(t0, t0 + k.shape[2])
    s["k_out"][0, :, :, to] = torch.where(live, k.to(s["k_out"].dtype), s["k_out"][0, :, :, to])
    s["v_out"][0, :, :, to] = torch.where(live, v.to(s["v_out"].dtype), s["v_out"][0, :, :, to])
    return [s["k_out"], s["v_out"]]


# -------------------------------------------------------------------- run --
def run(state):
    s, op = state, state["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "read": _plain_read}[op](s)
    ctx, c = _context(), s["case"]
    if op == "append":
        ctx.page_append(s["pages"], s["x_k"], s["x_v"], s["slots"], s["positions"], s["cos"], s["sin"], q=s["q"],
                        q_out=s["q_out"], interleaved=c["pairs"])
        return [s["q_out"], s["k"], s["v"], s["k_scale"], s["v_scale"]]
    if op == "read":
        ctx.page_read(s["pages"], s["kv_len"], s["table"], s["t0"], s["t1"], 0, s["k_out"], s["v_out"])
        return [s["k_out"], s["v_out"]]
    ctx.page_attend(s["pages"], s["q"], s["cu"], s["kv_len"], s["table"], s["max_new"], s["max_len"], out=s["out"],
                    lse=s["lse"], causal=c["causal"], window=c["window"], sinks=c["sinks"], softcap=c["softcap"],
                    slopes=s["slopes"], prefix=s["prefix"])
    return [s["out"], s["lse"]]


# ------------------------------------------------------------------- work --
def _seen(case, length, new, pre):
    """(visible pairs, positions that any row sees) of one request, counted from the mask's intervals."""
    pairs, after, first = 0, length + new, length + new
    W = case["window"]
    for i in range(new):
        p = length + i
        end = p + 1 if case["causal"] else after
        lo = max(0, p - W + 1) if W else 0
        low = max(min(pre, after), min(case["sinks"], end) if W else 0)
        first = min(first, lo)
        lo = max(lo, low)
        pairs += low + max(0, end - lo)
    low = max(min(pre, after), min(case["sinks"], after) if W else 0)
    return pairs, (min(after, low) + max(0, after - max(first, low))) if new else 0


def work(case):
    length, new = _lengths(case)
    n, B, op, H, D = case["n_req"], case["block"], case["op"], case["heads"], case["dim"]
    size = torch.empty(0, dtype=DTYPES[case["dtype"]]).element_size()
    # a row's codes and numbers in the pages; 8-bit pages have a scale each
    row = D // 2 + 4 if case["fmt"] == "uint4" else D
    if op == "append":
        T, Hq = sum(new), H * case["group"]
        table = min(T, max(l + v for l, v in zip(length, new))) * case["rot"] * 4
        scales = 0 if case["fmt"] == "uint4" else 8 * H * sum(_blocks(l + v, B) - l // B for l, v in zip(length, new) if v)
        return {"bytes": T * (2 * Hq * D * size + 2 * H * (D * size + row) + 12) + table + scales,
                "flops": T * (3 * (Hq + H) * case["rot"] + 4 * H * D)}
    if op == "read":
        T = sum(max(0, min(l, case["t1"]) - case["t0"]) for l in length)
        return {"bytes": T * H * 2 * (D * size + row), "flops": T * H * D * 4}
    pairs = positions = 0
    for l, v in zip(length, new):
        a, b = _seen(case, l, v, case["prefix"])
        pairs, positions = pairs + a, positions + b
    Hq = H * case["group"]
    return {"bytes": positions * H * 2 * row + sum(new) * Hq * (2 * D * size + 4), "flops": 4 * D * pairs * Hq}


# ------------------------------------------------------------------ exact --
def _exact_e4m3(y):
    """The nearest number of 4 significant bits, exponents from -6 on, at most 448; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _exact_page_scale(amax, e4m3):
    if not e4m3:
        return (amax / 127.0).clamp(min=FLOOR)
    # the first power of two from 2^-100 on that is not below amax / 448
    powers = torch.tensor([2.0 ** i for i in range(-100, 128)], dtype=torch.float64, device="cuda")
    return powers[torch.searchsorted(powers * 448.0, amax.contiguous())]


def _exact_rows4(x):
    """(step, middle) of rows in 64 bits: the middle to 8 significant bits, the step up to as many."""
    def bits8(y, how):
        unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1e-300))) - 7)
        return how(y / unit) * unit
    lo, hi = x.min(-1).values, x.max(-1).values
    mid = bits8((lo + hi) / 2, torch.round)
    step = bits8(torch.maximum(hi - mid, mid - lo) / 7.5, torch.ceil)
    return torch.stack([torch.maximum(step, mid.abs() / 65536).clamp(min=FLOOR), mid], -1)


def _exact_append(case, s):
    B, D, rot = case["block"], case["dim"], case["rot"]
    p = s["positions"].long()
    # a rotation as a complex product
    turn = torch.complex(s["cos"].double(), s["sin"].double())[p][:, None]

    def turned(x):
        x = x.double().clone()
        i = torch.arange(rot // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + rot // 2)
        z = torch.complex(x[..., a], x[..., b]) * turn
        x[..., a], x[..., b] = z.real, z.imag
        return x
    k, v, slots = turned(s["x_k"]), s["x_v"].double(), s["slots"]
    out = [turned(s["q"]), None, None]
    if case["fmt"] == "uint4":
        for scale, x in ((s["k_scale"], k), (s["v_scale"], v)):
            f = scale.double()
            f[slots // B, :, slots % B] = _exact_rows4(x)
            out.append(f)
        return out
    e4m3, runs = case["fmt"] == "e4m3", []
    for t, x in enumerate(slots.tolist()):
        if runs and runs[-1][1] + runs[-1][2] == x and x % B:
            runs[-1][2] += 1
        else:
            runs.append([t, x, 1])
    t, x, m = torch.tensor(runs, device="cuda").T
    blk, off = x // B, x % B
    which = torch.repeat_interleave(torch.arange(len(runs), device="cuda"), m)
    for i, (codes, scale, src) in enumerate(((s["k"], s["k_scale"], k), (s["v"], s["v_scale"], v))):
        c, f = codes.double(), scale.double()
        per = torch.zeros((len(runs), case["heads"]), dtype=torch.float64, device="cuda")
        per.scatter_reduce_(0, which[:, None].expand(-1, case["heads"]), src.abs().amax(-1), "amax")
        now = torch.maximum(_exact_page_scale(per, e4m3), torch.where(off[:, None] > 0, f[blk], torch.zeros_like(per)))
        if e4m3:
            again = _exact_e4m3(c[blk] * (f[blk] / now)[:, :, None, None])
            old = torch.arange(B, device="cuda") < off[:, None]
            c[blk] = torch.where(old[:, None, :, None], again, c[blk])
            c[slots // B, :, slots % B] = _exact_e4m3(src / now[which][:, :, None])
            out[1 + i] = c
        f[blk] = now
        out.append(f)
    return out


def _exact_values(codes, scale, ids, tokens):
    """One request's values [tokens, D] of one head in 64 bits."""
    level = (torch.arange(16, dtype=torch.float64, device="cuda") * 2 - 15) / 2
    c = codes[ids].flatten(0, 1)[:tokens].long()
    f = scale[ids].flatten(0, 1)[:tokens].double()
    x = torch.empty((c.shape[0], 2 * c.shape[1]), dtype=torch.float64, device="cuda")
    x[:, 0::2], x[:, 1::2] = level[c % 16], level[c // 16]
    return f[:, 1:] + x * f[:, :1]


def _exact_attend(case, s):
    length, new = _lengths(case)
    H, G, D = case["heads"], case["group"], case["dim"]
    outs, lses = [], []
    for r, (before, m) in enumerate(zip(length, new)):
        N = before + m
        if not m:
            continue
        ids = s["table"][r, :_blocks(N, case["block"])].long()
        first = int(s["cu"][r])
        pos = torch.arange(before, N, device="cuda")[:, None]
        j = torch.arange(N, device="cuda")[None, :]
        near = torch.ones((m, N), dtype=torch.bool, device="cuda")
        if case["window"]:
            near = (j > pos - case["window"]) | (j < case["sinks"])
        if case["causal"]:
            near = near & (j <= pos)
        if s["prefix"] is not None:
            near = near | (j < s["prefix"][r])
        o, l = [], []
        for h in range(H):
            k, v = (_exact_values(c[:, h], f[:, h], ids, N) for c, f in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
            for u in range(G):
                x = (s["q"][first:first + m, h * G + u].double() @ k.T) / math.sqrt(D)
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                if s["slopes"] is not None:
                    x = x + s["slopes"][h * G + u].double() * (j - pos)
                x = x.masked_fill(~near, -math.inf)
                z = torch.logsumexp(x, 1)
                l.append(z)
                o.append(torch.exp(x - torch.where(torch.isfinite(z), z, torch.zeros_like(z))[:, None]) @ v)
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(l, 1))
    return [torch.cat(outs), torch.cat(lses)]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "append":
        return _exact_append(case, s)
    if op == "attend":
        return _exact_attend(case, s)
    t0, t1 = s["t0"], s["t1"]
    k, v = s["k_out"].double(), s["v_out"].double()
    for r, l in enumerate(s["kv_len"].tolist()):
        to = min(l, t1)
        ids = s["table"][r, :_blocks(l, case["block"])].long()
        if to > t0:
            for out, codes, scale in ((k, s["k"], s["k_scale"]), (v, s["v"], s["v_scale"])):
                for h in range(case["heads"]):
                    out[0, r, h, t0:to] = _exact_values(codes[:, h], scale[:, h], ids, l)[t0:to]
    return [k, v]
