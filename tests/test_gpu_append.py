"""Writes of 4-bit pages, and appends with rotary positions into pages of every
format, on the GPU against the float64 oracle (oracle/paged.py): codes, scales and
numbers have to be equal, and so have turned queries (each step of the definition is
one float32 operation)."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
FMT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "uint4": torch.uint8}


@pytest.fixture(scope="module")
def fkv():
    import paper_2607_07144_gb300 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def ctx(fkv):
    return fkv.Context(256)


def _cuda(x, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda() if dtype else torch.from_numpy(np.ascontiguousarray(x)).cuda()


class Pool:
    """Pages of random bytes, here and on the device."""

    def __init__(self, fkv, rng, nb, H, D, block, fmt, by_token=False):
        self.fmt, self.block = fmt, block
        self.codes, self.scale, dev = [], [], []
        for _ in range(2):
            c = rng.integers(0, 256, (nb, H, block, D // 2 if fmt == "uint4" else D), dtype=np.uint8)
            if fmt == "e4m3":
                c[(c & 127) == 127] = 1                      # no NaN codes
            if fmt == "int8":
                c[c == 128] = 127
            if fmt == "uint4":
                s = paged.to_bf16(rng.standard_normal((nb, H, block, 2)).astype(np.float32))
                s[..., 0] = np.abs(s[..., 0]) + np.float32(1)
                s = paged.to_bf16(s)
            else:
                s = np.exp2(rng.integers(-9, -5, (nb, H))).astype(np.float32)
            self.codes.append(c)
            self.scale.append(s)
            t = _cuda(c if fmt != "int8" else c.view(np.int8))
            t = t.view(FMT[fmt])
            dev.append(t.transpose(1, 2).contiguous().transpose(1, 2) if by_token else t)
        st = torch.bfloat16 if fmt == "uint4" else torch.float32
        self.pages = fkv.Pages(dev[0], dev[1], *(_cuda(s, st) for s in self.scale))

    def write(self, k, v, slots):
        for c, s, x in zip(self.codes, self.scale, (k, v)):
            if self.fmt == "uint4":
                paged.write4(c, s, x, slots)
            else:
                paged.write(c, s, x.astype(np.float64), slots, self.fmt)

    def same(self):
        p = self.pages
        for c, s, t, f in zip(self.codes, self.scale, (p.k, p.v), (p.k_scale, p.v_scale)):
            assert np.array_equal(f.float().cpu().numpy(), s)
            assert np.array_equal(t.contiguous().view(torch.uint8).cpu().numpy(), c)


def _table(n_pos, half, base=10000.0):
    angle = np.arange(n_pos)[:, None] * base ** (-np.arange(half) / half)
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def _slots(rng, lens, nb, block):
    """Slots and positions of requests (positions before, new tokens) with scattered pages; a few tokens skipped."""
    ids, at, slots, pos = rng.permutation(nb), 0, [], []
    for before, n in lens:
        p = before + np.arange(n)
        j = p // block - before // block
        slots += list(ids[at + j] * block + p % block) if n else []
        pos += list(p)
        at += (int(j[-1]) + 1) if n else 0
    assert at <= nb
    return np.array(slots, np.int64), np.array(pos, np.int32)


LENS = {"steps": [(b, 1) for b in (0, 5, 16, 47, 300, 31, 15, 1000)], "drafts": [(3, 5), (14, 4), (500, 7), (0, 0), (63, 2)],
        "prompts": [(0, 1), (7, 100), (0, 33), (1000, 130), (0, 16)], "many": [(0, 1500), (10, 700)]}


@pytest.mark.parametrize("how", list(LENS))
@pytest.mark.parametrize("D,rot,pairs,block", [(64, 64, False, 16), (64, 16, True, 48), (128, 128, False, 64),
                                               (128, 128, True, 16), (128, 48, False, 128), (64, 32, False, 32)])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8", "uint4"])
def test_append(fkv, ctx, fmt, dtype, D, rot, pairs, block, how):
    rng = np.random.default_rng(3)
    H, Hq = 2, 5
    slots, pos = _slots(rng, LENS[how], 250 if block < 64 else 40, block)
    T = len(slots)
    # the ends of two requests, as a page of 8-bit codes takes one run of slots a call
    ends = np.cumsum([n for _, n in LENS[how]]) - 1
    slots[ends[0]] = -1                                      # its query is turned all the same
    pos[ends[1]] = -1                                        # left out
    pool = Pool(fkv, rng, 250 if block < 64 else 40, H, D, block, fmt, by_token=rot == 16)
    x = torch.from_numpy((rng.standard_normal((T, Hq + 2 * H, D)) * np.exp(rng.standard_normal((T, 1, 1)) * 2))
                         .astype(np.float32)).to(DT[dtype]).cuda()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    cos, sin = _table(1200 if how != "many" else 1600, rot // 2)
    both = _cuda(np.concatenate([cos, sin], 1)) if pairs or rot == 48 else None
    dc, ds = (both[:, :rot // 2], both[:, rot // 2:]) if both is not None else (_cuda(cos), _cuda(sin))
    out = torch.full((T, Hq, D), 7.0, dtype=DT[dtype], device="cuda")
    got = ctx.page_append(pool.pages, k, v, _cuda(slots), _cuda(pos), dc, ds, q=q, q_out=out, interleaved=pairs)
    assert ctx.sync_status() == 0 and got is out
    h = x.float().cpu().numpy()
    turned = paged.turn(h[:, :Hq + H], pos, cos, sin, rot, pairs)
    want = torch.from_numpy(turned[:, :Hq]).to(DT[dtype])
    want[torch.from_numpy(pos) < 0] = 7.0
    assert torch.equal(out.cpu(), want)
    pool.write(turned[:, Hq:], h[:, Hq + H:], np.where(pos < 0, -1, slots))
    pool.same()
    # queries in place, and none at all, give the same
    ctx.page_append(pool.pages, k, v, _cuda(slots), _cuda(pos), dc, ds, interleaved=pairs)
    pool.same()
    live = torch.from_numpy(pos) >= 0
    ctx.page_append(pool.pages, k, v, _cuda(slots), _cuda(pos), dc, ds, q=q, q_out=q, interleaved=pairs)
    assert ctx.sync_status() == 0
    assert torch.equal(q.cpu()[live], want[live])


@pytest.mark.parametrize("fmt", ["e4m3", "int8", "uint4"])
@pytest.mark.parametrize("H,D,block", [(7, 64, 16), (12, 64, 16), (13, 64, 16), (11, 128, 64), (8, 128, 32)])
def test_append_of_many_tokens(fkv, ctx, fmt, H, D, block):
    """So many runs that several heads share one look-up, heads that do not divide evenly among them, pages that grow."""
    rng = np.random.default_rng(12)
    lens = [(5, 9000), (0, 17), (block - 1, 6000), (3, 1), (0, 2500)]
    nb = sum(n // block + 3 for _, n in lens)
    slots, pos = _slots(rng, lens, nb, block)
    T = len(slots)
    pool = Pool(fkv, rng, nb, H, D, block, fmt)
    x = torch.from_numpy(rng.standard_normal((T, 1 + 2 * H, D)).astype(np.float32)).bfloat16().cuda()
    x[5999] *= 100                                           # a page's scale is one row's
    cos, sin = _table(9100, D // 4)
    out = ctx.page_append(pool.pages, x[:, 1:1 + H], x[:, 1 + H:], _cuda(slots), _cuda(pos), _cuda(cos), _cuda(sin), q=x[:, :1])
    assert ctx.sync_status() == 0
    h = x.float().cpu().numpy()
    t = paged.turn(h[:, :1 + H], pos, cos, sin, D // 2)
    assert torch.equal(out.cpu(), torch.from_numpy(t[:, :1]).bfloat16())
    pool.write(t[:, 1:], h[:, 1 + H:], slots)
    pool.same()


# So many tokens that a block of threads takes a run (its rule: more than 64 (token, head, K or V) an SM, and rows
# enough in a page for a block), in runs of up to 1,024 rows: more than its threads keep.
BLOCKS = [(64, 64, False, 48), (64, 32, True, 128), (128, 128, True, 48), (128, 128, False, 1024), (128, 64, False, 128),
          (64, 48, True, 1024)]


def _by_blocks(fkv, seed, fmt, dtype, D, block):
    rng = np.random.default_rng(seed)
    H, Hq = 8, 3
    lens = [(0, 500), (37, 400), (block - 1, 300), (1000, 1), (5, 1150), (block, 37)]
    nb = sum(n // block + 3 for _, n in lens)
    slots, pos = _slots(rng, lens, nb, block)
    T = len(slots)
    assert T * H * 2 > 64 * torch.cuda.get_device_properties(0).multi_processor_count and block * (D // 16) > 128
    pool = Pool(fkv, rng, nb, H, D, block, fmt)
    x = torch.from_numpy((rng.standard_normal((T, Hq + 2 * H, D)) * np.exp(rng.standard_normal((T, 1, 1))))
                         .astype(np.float32)).to(DT[dtype])
    return H, Hq, lens, slots, pos, pool, x


def _append_by_blocks(ctx, H, Hq, slots, pos, pool, x, rot, pairs, status):
    cos, sin = _table(2300, rot // 2)
    d = x.cuda()
    out = torch.full((len(slots), Hq, x.shape[2]), 7.0, dtype=x.dtype, device="cuda")
    ctx.page_append(pool.pages, d[:, Hq:Hq + H], d[:, Hq + H:], _cuda(slots), _cuda(pos), _cuda(cos), _cuda(sin), q=d[:, :Hq],
                    q_out=out, interleaved=pairs)
    assert ctx.sync_status() == status
    h = x.float().numpy()
    turned = paged.turn(h[:, :Hq + H], pos, cos, sin, rot, pairs)
    off = (pos < 0) | (pos >= len(cos))
    want = torch.from_numpy(turned[:, :Hq]).to(x.dtype)
    want[torch.from_numpy(off)] = 7.0
    assert torch.equal(out.cpu(), want)
    pool.write(turned[:, Hq:], h[:, Hq + H:], np.where(off, -1, slots))
    pool.same()


@pytest.mark.parametrize("D,rot,pairs,block", BLOCKS)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_runs_of_a_block_of_threads(fkv, ctx, fmt, dtype, D, rot, pairs, block):
    """Runs that end early: at tokens of no slot, and of negative positions, at requests' and pages' ends."""
    H, Hq, lens, slots, pos, pool, x = _by_blocks(fkv, 13, fmt, dtype, D, block)
    ends = np.cumsum([n for _, n in lens]) - 1
    slots[ends[0]], pos[ends[1]] = -1, -1
    last = np.flatnonzero(slots % block == block - 1)
    slots[last[0]], pos[last[-1]] = -1, -1
    _append_by_blocks(ctx, H, Hq, slots, pos, pool, x, rot, pairs, 0)


@pytest.mark.parametrize("D,rot,pairs,block", BLOCKS)
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_runs_of_a_block_with_positions_and_slots_outside(fkv, ctx, fmt, D, rot, pairs, block):
    H, Hq, lens, slots, pos, pool, x = _by_blocks(fkv, 14, fmt, "bf16", D, block)
    ends = np.cumsum([n for _, n in lens]) - 1
    pos[ends[0]], pos[ends[2]], pos[ends[4]] = 2300, 2 ** 31 - 1, -5
    _append_by_blocks(ctx, H, Hq, slots, pos, pool, x, rot, pairs, -2)
    slots = slots.copy()
    slots[ends[1]], slots[ends[5]] = 1 << 40, len(pool.codes[0]) * block
    pos[ends[0]] = pos[ends[2]] = -1
    _append_by_blocks(ctx, H, Hq, slots, pos, pool, x, rot, pairs, -2)


@pytest.mark.parametrize("D,rot,pairs,block", BLOCKS)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_runs_of_a_block_with_values_that_are_no_numbers(fkv, ctx, fmt, dtype, D, rot, pairs, block):
    """NaN, infinities and values beyond the scales' range in some rows of a run, in its first ones and in its last."""
    H, Hq, lens, slots, pos, pool, x = _by_blocks(fkv, 15, fmt, dtype, D, block)
    x[3, Hq + 1, 5], x[499, Hq + H + 7, D - 1], x[700, Hq + 2, 0] = float("nan"), float("inf"), float("-inf")
    x[1300, Hq + H, 9], x[1301, Hq + H, 9], x[40, 1, 3] = float("inf"), float("nan"), float("nan")
    if dtype != "f16":
        x[1700, Hq + 3], x[2000, Hq + H + 3] = 1.5e38, -2e36
    cos, sin = _table(2300, rot // 2)
    d = x.cuda()
    ctx.page_append(pool.pages, d[:, Hq:Hq + H], d[:, Hq + H:], _cuda(slots), _cuda(pos), _cuda(cos), _cuda(sin), interleaved=pairs)
    assert ctx.sync_status() == -5
    h = x.float().numpy()
    pool.write(paged.turn(h[:, Hq:Hq + H], pos, cos, sin, rot, pairs), h[:, Hq + H:], slots)
    pool.same()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D,block,T", [(64, 16, 1), (128, 32, 5), (128, 1024, 700), (64, 48, 3000)])
def test_write_of_4_bits(fkv, ctx, D, block, T, dtype):
    rng = np.random.default_rng(4)
    H = 3
    nb = T // block + 9
    slots = rng.permutation(nb * block)[:T].astype(np.int64)
    slots[T // 2] = -1
    pool = Pool(fkv, rng, nb, H, D, block, "uint4", by_token=D == 64)
    kv = torch.from_numpy((rng.standard_normal((T, 2, H, D)) + rng.standard_normal((T, 2, H, 1)) * 3).astype(np.float32)).to(DT[dtype]).cuda()
    ctx.page_write(pool.pages, kv[:, 0], kv[:, 1], _cuda(slots))
    assert ctx.sync_status() == 0
    h = kv.float().cpu().numpy()
    pool.write(h[:, 0], h[:, 1], slots)
    pool.same()


def test_unusual_values_of_4_bits(fkv, ctx):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((12, 1, 64)).astype(np.float32)
    x[0, 0, :4] = [np.inf, -np.inf, 0.0, -0.0]
    x[1] = 0
    x[2] *= np.float32(2.0 ** -130)
    x[3] *= np.float32(2.0 ** 110)
    x[4] = 1e-42
    x[5] = -1000.25
    x[6] = 3.0e38
    x[7, 0, ::2], x[7, 0, 1::2] = 3e38, -3e38
    x[8] = 1.0
    x[9] *= np.float32(2.0 ** -99)
    x[10] = 100 + x[10] * 2.0 ** -20
    x[11] = -0.0
    for dtype in ("f32", "bf16"):
        pool = Pool(fkv, rng, 2, 1, 64, 16, "uint4")
        t = _cuda(x).to(DT[dtype])
        h = t.float().cpu().numpy()
        ctx.page_write(pool.pages, t, t, _cuda(np.arange(12) + 3))
        assert ctx.sync_status() == 0
        pool.write(h, h, np.arange(12) + 3)
        pool.same()
        t[0, 0, 5], t[9, 0, 63] = float("nan"), float("nan")
        h = t.float().cpu().numpy()
        # a NaN of a token that is not stored is no one's
        slots = np.where(np.arange(12) == 9, -1, np.arange(12) + 3)
        t[0, 0, 5] = 0.0
        ctx.page_write(pool.pages, t, t, _cuda(slots))
        assert ctx.sync_status() == 0
        t[0, 0, 5] = float("nan")
        ctx.page_write(pool.pages, t, t, _cuda(slots))
        assert ctx.sync_status() == -5
        pool.write(h, h, slots)
        pool.same()


@pytest.mark.parametrize("fmt", ["e4m3", "uint4"])
@pytest.mark.parametrize("T", [4, 900])
def test_positions_and_slots_outside(fkv, ctx, fmt, T):
    """Tokens of a position past the table, or a slot past the pool: left out (of a slot: not stored) and reported."""
    rng = np.random.default_rng(6)
    H, D, nb = 8, 64, 64
    pool = Pool(fkv, rng, nb, H, D, 16, fmt)
    x = torch.from_numpy(rng.standard_normal((T, 3 * H, D)).astype(np.float32)).cuda()
    cos, sin = _table(1000, 32)
    # (tokens at the ends of their pages, as those of 8-bit codes take one run of slots a call)
    slots, pos = np.arange(T) * (16 if T == 4 else 1), np.arange(T).astype(np.int32)
    i, j = (1, 3) if T == 4 else (15, 31)
    for what in ("pos", "slot"):
        s, p = slots.copy(), pos.copy()
        if what == "pos":
            p[i], p[j] = 1000, 2 ** 31 - 1
        else:
            s[i], s[j] = nb * 16, 1 << 40
        out = torch.full((T, H, D), 7.0, device="cuda")
        ctx.page_append(pool.pages, x[:, H:2 * H], x[:, 2 * H:], _cuda(s), _cuda(p), _cuda(cos), _cuda(sin), q=x[:, :H], q_out=out)
        assert ctx.sync_status() == -2
        h = x.cpu().numpy()
        t = paged.turn(h[:, :2 * H], p, cos, sin, 64)
        want = t[:, :H].copy()
        if what == "pos":
            want[[i, j]] = 7
        assert np.array_equal(out.cpu().numpy(), want)
        bad = np.isin(np.arange(T), [i, j])
        pool.write(t[:, H:], h[:, 2 * H:], np.where(bad, -1, s))
        pool.same()


def test_a_table_of_many_positions(fkv, ctx):
    """Positions up to 2^30 - 1: 64-bit offsets into the tables (one row for all of them, or rows 2 GB apart)."""
    pool = Pool(fkv, np.random.default_rng(7), 2, 1, 64, 16, "uint4")
    x = torch.randn((3, 3, 64), device="cuda")
    cos, sin = _table(5, 32)
    c, s = (_cuda(y[4:5]).expand(1 << 30, -1) for y in (cos, sin))
    pos = np.array([0, (1 << 30) - 1, 123456789], np.int32)
    out = ctx.page_append(pool.pages, x[:, 1:2], x[:, 2:], _cuda(np.arange(3)), _cuda(pos), c, s, q=x[:, :1])
    assert ctx.sync_status() == 0
    h = x.cpu().numpy()
    t = paged.turn(h[:, :2], [4] * 3, cos, sin, 64)
    assert np.array_equal(out.cpu().numpy(), t[:, :1])
    pool.write(t[:, 1:], h[:, 2:], np.arange(3))
    pool.same()
    big = torch.empty((2, 1 << 29), device="cuda")             # rows of 2 GB; the last one lies past 2^32 bytes
    big = torch.cat([big, big[:1]])
    big[2, :64] = torch.cat([_cuda(cos[4]), _cuda(sin[4])])
    out = ctx.page_append(pool.pages, x[:, 1:2], x[:, 2:], _cuda(np.arange(3)), _cuda(np.array([2, 2, 2], np.int32)),
                          big[:, :32], big[:, 32:64], q=x[:, :1])
    assert ctx.sync_status() == 0
    assert np.array_equal(out.cpu().numpy(), t[:, :1])
    pool.same()


def test_pages_far_apart(fkv, ctx):
    """4-bit pages more than 2^32 bytes apart, and numbers as well."""
    H, D, B = 1, 128, 16
    raw = torch.zeros(3 << 31, dtype=torch.uint8, device="cuda")
    k, v = (raw[o:].as_strided((2, H, B, D // 2), (5 << 30, 1024, 64, 1)) for o in (0, 1 << 20))
    num = raw.view(torch.bfloat16)[1 << 21:]
    ks, vs = (num[o:].as_strided((2, H, B, 2), (5 << 29, 32, 2, 1)) for o in (0, 1 << 12))
    pages = fkv.Pages(k, v, ks, vs)
    x = torch.randn((20, 2, D), device="cuda")
    slots = np.arange(10, 30)
    ctx.page_write(pages, x[:, :1], x[:, 1:], _cuda(slots))
    assert ctx.sync_status() == 0
    codes = [np.zeros((2, H, B, D // 2), np.uint8) for _ in range(2)]
    numbers = [np.zeros((2, H, B, 2), np.float32) for _ in range(2)]
    h = x.cpu().numpy()
    for i, (c, n, t, f) in enumerate(zip(codes, numbers, (k, v), (ks, vs))):
        paged.write4(c, n, h[:, i:i + 1], slots)
        assert np.array_equal(t.cpu().numpy(), c) and np.array_equal(f.float().cpu().numpy(), n)
    out = torch.zeros((1, 1, H, 32, D), device="cuda")
    ctx.page_read(pages, _cuda(np.array([30], np.int32)), _cuda(np.array([[0, 1]], np.int32)), 10, 30, 0, out, None)
    assert ctx.sync_status() == 0
    want = paged.values4(codes[0], numbers[0]).reshape(1, 32, D)[:, 10:30].astype(np.float32)
    assert np.array_equal(out[0, 0, :, 10:30].cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D,block", [(64, 16), (128, 48), (128, 128)])
def test_read_of_4_bits(fkv, ctx, D, block, dtype):
    rng = np.random.default_rng(8)
    H, lens = 3, [200, 0, 17, 129, 64]
    need = [-(-x // block) for x in lens]
    nb = sum(need) + 3
    pool = Pool(fkv, rng, nb, H, D, block, "uint4", by_token=block == 48)
    ids, table, at = rng.permutation(nb), np.full((5, max(need)), -1, np.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    for t0, t1 in ((0, 200), (5, 130), (16, 17), (150, 220), (3, 3)):
        shape = (2, 6, H, 230, D)
        k, v = (torch.full(shape, 7.0, dtype=DT[dtype], device="cuda") for _ in range(2))
        ctx.page_read(pool.pages, _cuda(np.array(lens, np.int32)), _cuda(table), t0, t1, 1, k, v)
        assert ctx.sync_status() == 0
        for c, s, got in zip(pool.codes, pool.scale, (k, v)):
            want = torch.full(shape, 7.0, dtype=DT[dtype])
            for r, x in enumerate(lens):
                to = min(x, t1)
                if to > t0:
                    y = paged.gather4(c, s, table[r], x)[:, t0:to].astype(np.float32)      # one rounding to float32
                    want[1, r, :, t0:to] = torch.from_numpy(y).to(DT[dtype])
            assert torch.equal(got.cpu(), want)


def test_captured_and_replayed_on_another_stream(fkv, ctx):
    rng = np.random.default_rng(9)
    H, D, T = 2, 128, 40
    cos, sin = _table(300, 64)
    dc, ds = _cuda(cos), _cuda(sin)
    x = torch.zeros((T, 4 * H, D), dtype=torch.bfloat16, device="cuda")
    slots, pos = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    for fmt in ("int8", "uint4"):
        pool = Pool(fkv, rng, 8, H, D, 16, fmt)
        out = torch.zeros((T, 2 * H, D), dtype=torch.bfloat16, device="cuda")
        pos.fill_(-1)
        go = lambda: ctx.page_append(pool.pages, x[:, 2 * H:3 * H], x[:, 3 * H:], slots, pos, dc, ds, q=x[:, :2 * H], q_out=out)
        go()                                                 # nothing but positions below zero: a call that does no harm
        assert ctx.sync_status() == 0
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        out.zero_()
        for first in (0, 37, 80):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)))
            n = T - first % 5
            s = np.where(np.arange(T) < n, first + np.arange(T), -1)
            p = np.where(np.arange(T) < n, 100 + first + np.arange(T), -1).astype(np.int32)
            slots.copy_(_cuda(s)), pos.copy_(_cuda(p))
            before = out.clone()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graph.replay()
            side.synchronize()
            assert ctx.sync_status() == 0
            h = x.float().cpu().numpy()
            t = paged.turn(h[:, :3 * H], p, cos, sin, D)
            want = torch.from_numpy(t[:, :2 * H]).bfloat16()
            want[n:] = before.cpu()[n:]
            assert torch.equal(out.cpu(), want)
            pool.write(t[:, 2 * H:], h[:, 3 * H:], s)
            pool.same()


@pytest.mark.parametrize("fmt", ["int8", "uint4"])
def test_one_head_one_token_and_gaps(fkv, ctx, fmt):
    """Dimensions of one (whose strides mean nothing), queries and outputs with gaps, tables with a gap, pages of 1024."""
    rng = np.random.default_rng(10)
    cos, sin = _table(2000, 32)
    wide = torch.zeros((2000, 80), device="cuda")
    wide[:, 4:36], wide[:, 40:72] = _cuda(cos), _cuda(sin)
    for T, Hq in ((1, 1), (1, 7), (33, 1)):
        pool = Pool(fkv, rng, 3, 1, 64, 1024, fmt)
        x = torch.from_numpy(rng.standard_normal((T, 2 * Hq + 3, 64)).astype(np.float32)).half().cuda()
        q, k, v = x[:, :2 * Hq:2], x[:, -2:-1], x[:, -1:]
        big = torch.full((T, 2, Hq, 128), 7.0, dtype=torch.float16, device="cuda")
        slots, pos = 1024 + 990 + np.arange(T), (1990 - T + np.arange(T)).astype(np.int32)
        ctx.page_append(pool.pages, k, v, _cuda(slots), _cuda(pos), wide[:, 4:36], wide[:, 40:72], q=q, q_out=big[:, 1, :, 64:])
        assert ctx.sync_status() == 0
        h = x.float().cpu().numpy()
        want = torch.from_numpy(paged.turn(h[:, :2 * Hq:2], pos, cos, sin, 64)).half()
        assert torch.equal(big[:, 1, :, 64:].cpu(), want) and (big[:, 0] == 7).all() and (big[:, 1, :, :64] == 7).all()
        pool.write(paged.turn(h[:, -2:-1], pos, cos, sin, 64), h[:, -1:], slots)
        pool.same()


def test_values_that_are_no_numbers_are_reported_where_they_are_stored(fkv, ctx):
    rng = np.random.default_rng(11)
    cos, sin = _table(100, 64)
    for fmt in ("e4m3", "uint4"):
        pool = Pool(fkv, rng, 8, 2, 128, 16, fmt)
        x = torch.from_numpy(rng.standard_normal((5, 8, 128)).astype(np.float32)).bfloat16().cuda()
        x[0, 1, 3], x[2, 4, 5], x[4, 7, 127] = float("nan"), float("nan"), float("inf")       # a query, a key, a value
        slots = np.arange(5) * 16
        slots[2] = -1
        go = lambda s: ctx.page_append(pool.pages, x[:, 4:6], x[:, 6:], _cuda(s), _cuda(np.arange(5, dtype=np.int32)), _cuda(cos),
                                       _cuda(sin), q=x[:, :4])
        out = go(slots)
        assert ctx.sync_status() == 0 and out[0, 1, 3].isnan() and out[0, 1, 67].isnan() and not out[1:].isnan().any()
        h = x.float().cpu().numpy()
        pool.write(paged.turn(h[:, 4:6], np.arange(5), cos, sin, 128), h[:, 6:], slots)
        pool.same()
        slots[2] = 32
        go(slots)
        assert ctx.sync_status() == -5
        pool.write(paged.turn(h[:, 4:6], np.arange(5), cos, sin, 128), h[:, 6:], slots)
        pool.same()


def test_append_refusals(fkv, ctx):
    pages = fkv.Pages.empty(4, 2, 16, 64, torch.uint8)
    x = torch.zeros((3, 2, 64), device="cuda")
    s, p = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    c = torch.zeros((10, 32), device="cuda")

    def refused(call, exc=None):
        with pytest.raises(exc or fkv.FkvError) as e:
            call()
        if exc is None:
            assert e.value.code == -1
    go = lambda **o: ctx.page_append(o.get("pages", pages), o.get("k", x), o.get("v", x), o.get("s", s), o.get("p", p),
                                     o.get("c", c), o.get("n", o.get("c", c)), q=o.get("q"), q_out=o.get("q_out"))
    refused(lambda: go(k=x.half()), ValueError)
    refused(lambda: go(k=x[:, :1], v=x[:, :1]), ValueError)
    refused(lambda: go(s=s[:2]), ValueError)
    refused(lambda: go(p=p.long()), ValueError)
    refused(lambda: go(c=c.double()), ValueError)
    refused(lambda: go(c=c.cpu()), ValueError)
    refused(lambda: go(n=c[:5]), ValueError)
    refused(lambda: go(q=x.half()), ValueError)
    refused(lambda: go(q=x[:2]), ValueError)
    refused(lambda: go(q_out=x), ValueError)
    refused(lambda: go(q=x, q_out=x[:, :1]), ValueError)
    refused(lambda: go(c=c[:, :4].contiguous()))             # 8 dimensions
    refused(lambda: go(c=torch.zeros((10, 40), device="cuda")))
    refused(lambda: go(c=c[:0]))
    refused(lambda: go(c=torch.zeros((10, 33), device="cuda")[:, 1:]))
    refused(lambda: go(k=x.flatten()[1:1 + 2 * 128].view(2, 2, 64), v=x[:2], s=s[:2]))     # 4-byte aligned
    refused(lambda: go(pages=fkv.Pages.empty(4, 2, 24, 64, torch.uint8)))
    refused(lambda: fkv.Pages(pages.k, pages.v, pages.k_scale.float(), pages.v_scale.float()), ValueError)
    refused(lambda: fkv.Pages(pages.k, pages.v, *[torch.zeros((4, 2), device="cuda")] * 2), ValueError)
    wide = torch.zeros((4, 2, 16, 4), dtype=torch.bfloat16, device="cuda")
    refused(lambda: fkv.Pages(pages.k, pages.v, wide[..., :2], wide[..., :2]), ValueError)
    odd = torch.zeros((4, 2 * 32 + 2), dtype=torch.bfloat16, device="cuda")[:, :64].unflatten(1, (2, 16, 2))
    refused(lambda: go(pages=fkv.Pages(pages.k, pages.v, odd, odd)))                       # numbers on 4-byte boundaries
    one = torch.zeros((1, 1, 1024, 32), dtype=torch.uint8, device="cuda")
    num = torch.zeros((1, 1, 1024, 2), dtype=torch.bfloat16, device="cuda")
    n = (1 << 22) + 1
    big = fkv.Pages(*[one.expand(n, -1, -1, -1)] * 2, *[num.expand(n, -1, -1, -1)] * 2)
    refused(lambda: go(pages=big, k=x[:, :1], v=x[:, :1]))
    refused(lambda: ctx.page_write(big, x[:, :1], x[:, :1], s))
    assert ctx.page_append(pages, x[:0], x[:0], s[:0], p[:0], c, c) is None
    assert ctx.sync_status() == 0
