"""Attention over 4-bit pages on the GPU against the float64 oracle (oracle/paged.py).

An output may be off by
  half a step of its type, of the value (eps / 2 |o|);
  roundings to fp16, half a step, 2^-11, each: of the weights, which multiply codes less
  their middle (few rows) or whole values (many), and there of the values: 2^-10 of the
  weighted sum of |c - 7.5| step + |middle| (2^-24 of the smallest normal weights is below
  2^-30 of the largest, times the number of keys);
  the scores' error as a relative one of the weights: fp32 products and sums of D terms,
  and the base-2 exponential's argument, each a few 2^-24 of the magnitudes that enter,
  2^-20 (sum |q| (15 step + |middle|) scale + cap + bias + |lse| + 16) times the same sum.
lse: the scores' error alone."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def fkv():
    import paper_2607_07144_gb300 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def ctx(fkv):
    return fkv.Context(256)


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Batch:
    """Requests of (positions before, new tokens) with pages scattered over a pool of random bytes."""

    def __init__(self, fkv, seed, lens, H, G, D, block, dtype, by_token=False, spare=3, gap=0, spread=0.3):
        rng = np.random.default_rng(seed)
        self.H, self.G, self.D, self.block = H, G, D, block
        self.before = [b for b, _ in lens]
        self.new = [n for _, n in lens]
        self.len = [max(0, b + n) for b, n in lens]          # before < 0: tokens at negative positions
        need = [-(-x // block) for x in self.len]
        nb = sum(need) + spare
        ids = rng.permutation(nb)
        width = max(1, max(need))
        self.table = np.full((len(lens), width), -1, np.int64)
        at = 0
        for r, x in enumerate(need):
            self.table[r, :x] = ids[at:at + x]
            at += x
        self.codes, self.numbers, dev = [], [], []
        for _ in range(2):
            c = rng.integers(0, 256, (nb, H, block, D // 2), dtype=np.uint8)
            step = paged.to_bf16((np.exp(rng.standard_normal((nb, H, block)) * spread) / 4).astype(np.float32))
            mid = paged.to_bf16((rng.standard_normal((nb, H, block)) * step * 4).astype(np.float32))
            n = np.stack([step, mid], -1)
            # slots past a request's end and unused pages: any numbers
            n[ids[at:]] = np.nan
            for r, x in enumerate(self.len):
                if x % block:
                    n[self.table[r, need[r] - 1], :, x % block:, 0] = np.inf
                    n[self.table[r, need[r] - 1], :, x % block:, 1] = np.nan
            self.codes.append(c)
            self.numbers.append(n)
            t = torch.from_numpy(c).cuda()
            dev.append(t.transpose(1, 2).contiguous().transpose(1, 2) if by_token else t)
        T = sum(self.new) + gap
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.q = torch.from_numpy(rng.standard_normal((T, H * G, D)).astype(np.float32)).to(DT[dtype]).cuda()
        self.pages = fkv.Pages(dev[0], dev[1], *(torch.from_numpy(s).bfloat16().cuda() for s in self.numbers))

    def run(self, ctx, **opt):
        lse = torch.full((self.q.shape[0], self.H * self.G), 7.0, device="cuda")
        out = torch.full_like(self.q, 7.0)
        ctx.page_attend(self.pages, self.q, _i32(self.cu), _i32(self.len), _i32(self.table),
                        opt.pop("max_new", max(self.new)), opt.pop("max_len", max(self.len)), out=out, lse=lse, **opt)
        return out, lse

    def check(self, ctx, rows=None, prefix=None, slopes=None, softcap=0.0, scale=None, skip=(), **mask):
        """rows: per request, the token indexes to compare (all if None); skip: requests that are left out."""
        sc = self.D ** -0.5 if scale is None else scale
        opt = dict(mask, softcap=softcap, scale=scale)
        if prefix is not None:
            opt["prefix"] = _i32(prefix)
        if slopes is not None:
            opt["slopes"] = torch.tensor(slopes, dtype=torch.float32, device="cuda")
        out, lse = self.run(ctx, **opt)
        assert ctx.sync_status() == (-2 if skip else 0)
        again, lse2 = self.run(ctx, **opt)
        ctx.sync_status()
        assert torch.equal(out, again) and torch.equal(lse, lse2)          # the same bits every time
        self.compare(out, lse, rows, prefix, slopes, softcap, sc, skip, mask)

    def compare(self, out, lse, rows, prefix, slopes, softcap, sc, skip, mask):
        eps = torch.finfo(self.q.dtype).eps / 2
        o, l, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), self.q.double().cpu().numpy()
        assert (o[self.cu[-1]:] == 7).all() and (l[self.cu[-1]:] == 7).all()
        for r, (n, length) in enumerate(zip(self.new, self.len)):
            if n == 0:
                continue
            if r in skip:
                assert (o[self.cu[r]:self.cu[r + 1]] == 7).all() and (l[self.cu[r]:self.cu[r + 1]] == 7).all()
                continue
            k, v = (paged.gather4(c, s, self.table[r], length) for c, s in zip(self.codes, self.numbers))
            ids = [int(i) for i in self.table[r, :-(-length // self.block)]]
            num = [np.abs(np.concatenate([s[i] for i in ids], 1)[:, :length]) if ids else np.zeros((self.H, 0, 2)) for s in self.numbers]
            big_v = np.abs(v - num[1][..., 1:] * np.sign(v)) + 2 * num[1][..., 1:]       # at least |c - 7.5| step + |middle|
            p0 = self.before[r]
            seen = paged.visible(n, length, mask.get("causal", True), mask.get("window", 0), mask.get("sinks", 0),
                                 None if prefix is None else prefix[r])
            pick = np.arange(n) if rows is None else np.unique(np.clip(np.asarray(rows), 0, n - 1))
            at = self.cu[r] + pick
            want = np.zeros((len(pick), self.H * self.G, self.D))
            wl, mass, size = want[:, :, 0].copy(), want.copy(), want[:, :, 0].copy()
            for e, i in enumerate(pick):
                row = q[self.cu[r] + i][None]
                want[e], wl[e], _, _ = (x[0] for x in paged.attend(row, k, v, sc, seen[i:i + 1], softcap, slopes, p0 + i))
                mass[e] = paged.attend(row, k, big_v, sc, seen[i:i + 1], softcap, slopes, p0 + i)[0][0]
                if seen[i].any():
                    most = (15 * num[0][:, seen[i], 0] + num[0][:, seen[i], 1]).max(1)
                    size[e] = abs(sc) * np.abs(row[0]).sum(-1) * np.repeat(most, self.G)
            bias = 0.0 if slopes is None else max(np.abs(slopes)) * length
            fin = np.isfinite(wl)
            ds = 2.0 ** -20 * (size + softcap + bias + np.where(fin, np.abs(wl), 0) + 16)
            bound = eps * np.abs(want) + (2.0 ** -10 + ds + length * 2.0 ** -30)[..., None] * mass * (1 + eps) + 1e-30
            assert (np.abs(o[at] - want) <= bound).all(), (r, np.max(np.abs(o[at] - want) / bound))
            assert np.array_equal(np.isneginf(l[at]), ~fin)
            assert (np.abs(np.where(fin, l[at], 0) - np.where(fin, wl, 0)) <= ds).all()


RAGGED = [(0, 1), (15, 1), (16, 1), (127, 1), (128, 1), (129, 1), (500, 1), (0, 0), (31, 1), (33, 1)]


@pytest.mark.parametrize("G", [1, 4, 7])
@pytest.mark.parametrize("block", [16, 48, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_steps(fkv, ctx, D, dtype, block, G):
    Batch(fkv, 1, RAGGED, 2, G, D, block, dtype, by_token=G == 4, gap=2).check(ctx)


DRAFTS = [(3, 5), (0, 3), (200, 7), (128, 1), (90, 4), (0, 0), (-3, 6), (700, 2)]


@pytest.mark.parametrize("opt", [dict(), dict(window=40, sinks=4), dict(window=1), dict(softcap=20.0), dict(softcap=1000.0),
                                 dict(causal=False), dict(slopes=True), dict(prefix=True), dict(scale=-0.2),
                                 dict(window=64, sinks=20, prefix=True, slopes=True, softcap=5.0), dict(scale=0.0)])
@pytest.mark.parametrize("D,dtype,block", [(64, "bf16", 16), (128, "f16", 32), (128, "bf16", 64)])
def test_drafts(fkv, ctx, D, dtype, block, opt):
    opt = dict(opt)
    b = Batch(fkv, 2, DRAFTS, 2, 3, D, block, dtype, by_token=block == 32)
    if "slopes" in opt:
        opt["slopes"] = [0.5, 0.1, -0.05, 0.3, 0.0, 0.02]
    if "prefix" in opt:
        opt["prefix"] = [2, 0, 150, 129, 5, 0, 2, 30]
    b.check(ctx, **opt)


@pytest.mark.parametrize("opt", [dict(), dict(window=100, sinks=7), dict(softcap=20.0), dict(softcap=1000.0), dict(causal=False),
                                 dict(slopes=True), dict(prefix=True), dict(window=64, sinks=300, prefix=True, slopes=True, softcap=5.0)])
@pytest.mark.parametrize("D,dtype,block,G", [(64, "f16", 16, 1), (128, "bf16", 64, 4), (128, "f16", 48, 1), (64, "bf16", 128, 2)])
def test_prompts(fkv, ctx, D, dtype, block, G, opt):
    opt = dict(opt)
    b = Batch(fkv, 3, [(0, 300), (37, 70), (0, 1), (500, 129), (0, 0), (-5, 64), (130, 257)], 2, G, D, block, dtype, by_token=block == 64)
    if "slopes" in opt:
        opt["slopes"] = list(0.3 * 0.5 ** np.arange(2 * G))
    if "prefix" in opt:
        opt["prefix"] = [100, 0, 1, 400, 0, 3, 20]
    b.check(ctx, rows=[0, 1, 15, 16, 63, 64, 127, 128, 200, 256, 299], **opt)


@pytest.mark.parametrize("opt", [dict(), dict(softcap=30.0), dict(slopes=[0.01, 0.001, -0.0005, 0.1])])
@pytest.mark.parametrize("new", [1, 6, 90])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_shares_of_a_long_sequence(fkv, ctx, D, dtype, new, opt):
    b = Batch(fkv, 4, [(30000, new)], 1, 4, D, 64, dtype)
    b.check(ctx, rows=[0, new // 2, new - 1], **opt)


@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_window_far_from_sinks_and_prefix(fkv, ctx, D, dtype, new):
    b = Batch(fkv, 5, [(x, new) for x in (300, 2100, 5000)], 1, 4, D, 16, dtype)
    rows = [0, new // 2, new - 1]
    for opt in (dict(sinks=1500), dict(prefix=[5, 600, 4100]), dict(sinks=700, prefix=[0, 1000, 300])):
        b.check(ctx, rows=rows, window=100, **opt)
    # the pages behind a window, and their table entries, may be gone
    for r, x in enumerate(b.len):
        b.table[r, 1:max(1, (b.before[r] - 100) // 16 - 1)] = -1
    out, lse = b.run(ctx, window=100, sinks=4)
    assert ctx.sync_status() == 0
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("new", [1, 7, 80])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_steps_of_any_size(fkv, ctx, D, dtype, new):
    """Rows' steps apart by factors up to 2^60, as of one sequence's silent and loud positions."""
    b = Batch(fkv, 6, [(200, new), (20, new)], 1, 2, D, 16, dtype, spread=0.1)
    rng = np.random.default_rng(60)
    for kv in (0, 1):
        far = np.exp2(rng.integers(-50 if kv else -3, 10 if kv else 1, b.numbers[kv].shape[:3]))[..., None].astype(np.float32)
        with np.errstate(invalid="ignore"):
            b.numbers[kv] = b.numbers[kv] * far
    p = b.pages
    b.pages = fkv.Pages(p.k, p.v, *(torch.from_numpy(s).bfloat16().cuda() for s in b.numbers))
    b.check(ctx, rows=[0, new - 1])


@pytest.mark.parametrize("new", [1, 70])
def test_rows_of_zero_and_of_one_value(fkv, ctx, new):
    """Values that have no range: steps of 2^-100, or 2^-16 of the middle."""
    b = Batch(fkv, 7, [(40, new)], 1, 1, 64, 16, "f16")
    for j in range(40 + new):
        n = b.numbers[1][b.table[0, j // 16], 0, j % 16]
        n[:] = [2.0 ** -100, 0.0] if j % 2 else [3.0 * 2.0 ** -16, 3.0]
        b.codes[1][b.table[0, j // 16], 0, j % 16] = 0x77
    v = torch.from_numpy(b.codes[1]).cuda()
    b.pages = fkv.Pages(b.pages.k, v, *(torch.from_numpy(s).bfloat16().cuda() for s in b.numbers))
    b.check(ctx)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 70])
def test_queries_of_any_size(fkv, ctx, dtype, new):
    b = Batch(fkv, 8, [(100, new), (3, new)], 1, 2, 128, 16, dtype)
    far = torch.exp2(torch.randint(-14, 3, b.q.shape, device="cuda").float())
    b.q = (b.q.float() * far).to(b.q.dtype)
    if dtype == "bf16":
        b.q[0] *= 2.0 ** 60
        b.q[0] *= 2.0 ** -58
        b.q[-1] *= 2.0 ** -70
    b.q[new] = 0
    b.check(ctx)


@pytest.mark.parametrize("G", [8, 9, 16, 17, 32, 33, 71])
@pytest.mark.parametrize("D,block,dtype", [(64, 80, "bf16"), (128, 96, "f16"), (128, 1024, "bf16")])
def test_many_query_heads_a_kv_head(fkv, ctx, D, block, dtype, G):
    """Rows around what one and two tiles, and the other kernel, take; pages of which 16, 32 and 64 rows are loaded together."""
    b = Batch(fkv, 20, [(300, 1), (0, 1), (64, 1), (1100, 1)], 1, G, D, block, dtype, gap=3)
    b.check(ctx)
    b.check(ctx, window=70, sinks=3)


@pytest.mark.parametrize("scale", [0.0, 1e-38, -0.1])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_vanishing_and_negative_scores_of_prompts(fkv, ctx, D, dtype, scale):
    b = Batch(fkv, 21, [(130, 300), (5, 40), (0, 3), (400, 1)], 1, 2, D, 16, dtype)
    b.check(ctx, scale=scale, rows=[0, 1, 39, 150, 299])
    b.check(ctx, scale=scale, rows=[0, 39, 299], window=37, sinks=3, prefix=[20, 0, 3, 7])


@pytest.mark.parametrize("new", [1, 5, 60])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16"), (128, "f16")])
def test_middles_far_above_steps(fkv, ctx, D, dtype, new):
    """Rows that are nearly constant, up to middles of 2^16 steps, beside others that are not."""
    b = Batch(fkv, 22, [(150, new), (17, new)], 1, 2, D, 16, dtype)
    rng = np.random.default_rng(70)
    for kv in (0, 1):
        n = b.numbers[kv]
        far = np.exp2(-rng.integers(0, 17, n.shape[:3]) * rng.integers(0, 2, n.shape[:3])).astype(np.float32)
        big = paged.to_bf16((rng.standard_normal(n.shape[:3]) * (0.2 if kv == 0 else 3)).astype(np.float32))
        with np.errstate(invalid="ignore"):
            step = np.maximum(np.abs(big) * far, np.float32(2.0 ** -100))
            n[..., 0] = np.where(far < 1, np.where(np.isfinite(n[..., 0]), step, n[..., 0]), n[..., 0])
            n[..., 1] = np.where(far < 1, np.where(np.isfinite(n[..., 1]), big, n[..., 1]), n[..., 1])
    p = b.pages
    b.pages = fkv.Pages(p.k, p.v, *(torch.from_numpy(s).bfloat16().cuda() for s in b.numbers))
    b.check(ctx, rows=[0, new // 2, new - 1])


@pytest.mark.parametrize("new", [1, 9, 70])
def test_large_float16_queries(fkv, ctx, new):
    b = Batch(fkv, 23, [(100, new)], 1, 4, 128, 32, "f16")
    b.q = (b.q.float() * 2.0 ** 13).clamp(-65504, 65504).half()
    b.check(ctx, scale=2.0 ** -17)


def test_bounds_far_above_the_lengths(fkv, ctx):
    """max_len of 2^30 sizes the launch, not the work."""
    for new in (1, 3, 50):
        b = Batch(fkv, 24, [(70, new), (0, new), (500, new)], 2, 2, 64, 16, "bf16")
        want, lse = b.run(ctx)
        width = 1 << 20                                        # a table row that could hold 2^24 positions
        tab = torch.zeros((3, width), dtype=torch.int32, device="cuda")
        tab[:, :b.table.shape[1]] = _i32(b.table)
        out = torch.full_like(b.q, 7.0)
        ctx.page_attend(b.pages, b.q, _i32(b.cu), _i32(b.len), tab, 64, 1 << 30, out=out)
        assert ctx.sync_status() == 0
        eps = torch.finfo(b.q.dtype).eps
        # other shares of the keys, other sums: each of the two is as near to the exact result as check() asks
        v = np.nanmax(np.abs(paged.values4(b.codes[1], np.nan_to_num(b.numbers[1], posinf=0.0))))
        assert (out.double() - want.double()).abs().max().item() <= eps * want.double().abs().max().item() + 2 * 2.0 ** -10 * 2 * v


def test_prompts_captured_and_replayed_with_other_lengths(fkv, ctx):
    for dtype, D in (("f16", 64), ("bf16", 128)):
        b = Batch(fkv, 25, [(700, 90), (20, 64)], 2, 2, D, 16, dtype)
        d = dict(ln=_i32(b.len), out=torch.zeros_like(b.q))
        run = lambda: ctx.page_attend(b.pages, b.q, _c, d["ln"], _t, 90, max(b.len), out=d["out"])
        _c, _t = _i32(b.cu), _i32(b.table)
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        for cut in (0, 5, 80):
            d["ln"].copy_(_i32([max(0, x - cut) for x in b.len]))
            run()
            want = d["out"].clone()
            d["out"].zero_()
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
            s.synchronize()
            assert torch.equal(d["out"], want)
        assert ctx.sync_status() == 0


@pytest.mark.parametrize("new", [1, 6, 90])
def test_requests_that_do_not_hold_together(fkv, ctx, new):
    b = Batch(fkv, 9, [(60, new), (40, new), (90, new)], 2, 2, 64, 16, "bf16")
    b.len[1] = 10 ** 6
    b.check(ctx, skip=(1,), max_len=200)


def test_pages_outside_the_pool(fkv, ctx):
    for new in (1, 70):
        b = Batch(fkv, 10, [(60, new), (90, new)], 2, 2, 128, 16, "bf16")
        keep = b.table.copy()
        b.table[0, 1], b.table[0, 2] = 10 ** 6, -7
        out, lse = b.run(ctx)
        assert ctx.sync_status() == -2
        b.table = keep
        good, lse2 = b.run(ctx)
        assert torch.equal(out[new:], good[new:]) and torch.equal(lse[new:], lse2[new:])


def test_views_and_a_split_output(fkv, ctx):
    """Queries as a slice of a fused projection, an output of other strides, out over q."""
    for new in (1, 100):
        b = Batch(fkv, 11, [(70, new), (5, new)], 2, 2, 64, 32, "bf16")
        want, lse = b.run(ctx)
        wide = torch.zeros((2 * new, 12, 64), dtype=torch.bfloat16, device="cuda")
        wide[:, 3:7] = b.q
        big = torch.full((2 * new, 2, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        args = (_i32(b.cu), _i32(b.len), _i32(b.table), new, max(b.len))
        ctx.page_attend(b.pages, wide[:, 3:7], *args, out=big[:, 1])
        assert torch.equal(big[:, 1], want) and (big[:, 0] == 7).all()
        ctx.page_attend(b.pages, wide[:, 3:7], *args, out=wide[:, 3:7])
        assert torch.equal(wide[:, 3:7], want)
        assert ctx.sync_status() == 0


def test_pages_far_apart(fkv, ctx):
    """Pages, and their numbers, more than 2^32 bytes apart."""
    for new in (1, 40):
        b = Batch(fkv, 12, [(20, new)], 1, 2, 128, 64, "bf16")
        nb = len(b.codes[0])
        gap = 5 << 30
        raw = torch.zeros(gap * (nb - 1) + (1 << 22), dtype=torch.uint8, device="cuda")
        half = raw.view(torch.bfloat16)
        dev = [raw[o:].as_strided((nb, 1, 64, 64), (gap, 4096, 64, 1)) for o in (0, 1 << 16)]
        num = [half[o:].as_strided((nb, 1, 64, 2), (gap // 2, 128, 2, 1)) for o in (1 << 16, 1 << 17)]
        for t, c, f, s in zip(dev, b.codes, num, b.numbers):
            t.copy_(torch.from_numpy(c))
            f.copy_(torch.from_numpy(s).bfloat16())
        b.pages = fkv.Pages(*dev, *num)
        b.check(ctx)
        del raw, half, dev, num


def test_overlapping_calls_and_replays(fkv, ctx):
    """Two captured calls, each with its own workspace, replayed at once on two streams with other lengths."""
    both = []
    for seed, new in ((13, 1), (14, 3)):
        b = Batch(fkv, seed, [(9000, new)], 1, 4, 128, 64, "bf16")
        d = dict(cu=_i32(b.cu), ln=_i32(b.len), tab=_i32(b.table), out=torch.zeros_like(b.q))
        run = lambda b=b, d=d, new=new: ctx.page_attend(b.pages, b.q, d["cu"], d["ln"], d["tab"], new, max(b.len), out=d["out"])
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        both.append((b, d, g, run))
    for cut in (0, 17, 4000):
        want = []
        for b, d, g, run in both:
            d["ln"].copy_(_i32([x - cut for x in b.len]))
            run()
            want.append(d["out"].clone())
            d["out"].zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for b, d, g, run in both:
                s = torch.cuda.Stream()
                with torch.cuda.stream(s):
                    g.replay()
            torch.cuda.synchronize()
            for (b, d, g, run), w in zip(both, want):
                assert torch.equal(d["out"], w)
    assert ctx.sync_status() == 0


def test_serving_loop_and_archive(fkv, oracle_mod):
    """Prompts, steps and a request that ends: plan, append with rotation and attend, captured once and replayed;
    then the positions that leave the 4-bit pages go through the residual VQ, as a cache's do."""
    rng = np.random.default_rng(18)
    H, G, D, block, n = 2, 2, 64, 16, 4
    cb = rng.standard_normal((1, H, 1, 256, D)).astype(np.float32)
    ctx = fkv.Context(256, codebooks=(cb, cb))
    nb, width, rows = 24, 8, 12
    pages = fkv.Pages.empty(nb, H, block, D, torch.uint8)
    codes = [t.cpu().numpy() for t in (pages.k, pages.v)]
    numbers = [t.float().cpu().numpy() for t in (pages.k_scale, pages.v_scale)]
    table, free, taken = np.full((n, width), -1), np.arange(nb), 0
    ln = np.zeros(n, np.int64)
    angle = np.arange(width * block)[:, None] * 10000.0 ** (-np.arange(D // 2) / (D // 2))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    dc, ds = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    d = dict(new=_i32(np.zeros(n)), ln=_i32(ln), table=_i32(table), free=_i32(free), taken=_i32([0]), cu=_i32(np.zeros(n + 1)),
             slots=torch.zeros(rows, dtype=torch.int64, device="cuda"), pos=_i32(np.zeros(rows)))
    x = torch.zeros((rows, 2 * H + H * G, D), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((rows, H * G, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((rows, H * G), device="cuda")

    def step():
        ctx.page_plan(d["new"], d["ln"], d["table"], d["free"], d["taken"], block, d["cu"], d["slots"], d["pos"])
        q = ctx.page_append(pages, x[:, :H], x[:, H:2 * H], d["slots"], d["pos"], dc, ds, q=x[:, 2 * H:], q_out=x[:, 2 * H:])
        ctx.page_attend(pages, q, d["cu"], d["ln"], d["table"], 9, width * block, out=out, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                            # nothing new: a call that does no harm
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    assert ctx.sync_status() == 0
    for new in ([7, 2, 0, 3], [1, 1, 9, 1], [1, 1, 1, -1], [1, 1, 1, 5], [1, -1, 1, 1], [1, 9, 1, 1]):
        d["new"].copy_(_i32(new))
        x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)))
        h = x.float().cpu().numpy()
        out.fill_(7)
        graph.replay()
        assert ctx.sync_status() == 0
        before = np.where(np.asarray(new) < 0, 0, ln)
        cu, slots, pos, ln, taken, table, free, ok = paged.plan(new, ln, table, free, taken, block, rows)
        assert ok and np.array_equal(d["slots"].cpu().numpy(), slots) and np.array_equal(d["pos"].cpu().numpy(), pos)
        k = paged.turn(h[:, :H], pos, cos, sin, D)
        for c, s, y in zip(codes, numbers, (k, h[:, H:2 * H])):
            paged.write4(c, s, y, slots)
        q = torch.from_numpy(paged.turn(h[:, 2 * H:], pos, cos, sin, D)).bfloat16().double().numpy()
        o = out.double().cpu().numpy()
        for r in range(n):
            m = max(new[r], 0)
            if not m:
                continue
            k, v = (paged.gather4(c, s, table[r], int(ln[r])) for c, s in zip(codes, numbers))
            want, wl, _, size = paged.attend(q[cu[r]:cu[r] + m], k, v, D ** -0.5, paged.visible(m, int(ln[r])), p0=int(before[r]))
            # whole values here: |c - 7.5| step + |middle| is at most 2 max |v| of a row, products 4 max |k| sum |q|
            most = np.repeat(np.abs(v).max((1, 2)), G)[None, :, None]
            size = D ** -0.5 * np.abs(q[cu[r]:cu[r] + m]).sum(-1) * 4 * np.repeat(np.abs(k).max((1, 2)), G)
            bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.0 ** -20 * (size + np.abs(wl) + 16) + 1e-6)[..., None] * 2 * most
            assert (np.abs(o[cu[r]:cu[r] + m] - want) <= bound * (1 + 2.0 ** -8)).all()
        assert (o[cu[n]:] == 7).all()
    assert np.array_equal(pages.k.cpu().numpy()[table[0, 0]], codes[0][table[0, 0]])
    # the oldest positions of every request leave for the archive
    t1 = int(ln.min())
    K, V = (torch.zeros((1, n, H, 16, D), dtype=torch.float32, device="cuda") for _ in range(2))
    ctx.page_read(pages, d["ln"], d["table"], 0, t1, 0, K, V)
    R = ctx.record_len()
    sym = torch.zeros((n, t1 * R), dtype=torch.uint8, device="cuda")
    ctx.rvq_encode(0, K, 0, t1, sym)
    ctx.rvq_encode(1, V, 0, t1, sym)
    assert ctx.sync_status() == 0
    from oracle import parity
    s = sym.cpu().numpy()
    for r in range(n):
        idx = oracle_mod.indices_from_records(s[r], H, 1, 1)
        for kv in (0, 1):
            val = paged.gather4(codes[kv], numbers[kv], table[r], t1).astype(np.float32).astype(np.float64)
            for hh in range(H):
                oi, gap = oracle_mod.rvq_encode(val[hh], cb[0, hh])
                assert parity.compare_rvq(idx[kv][hh], oi, gap)[0] == 0


def test_refusals(fkv, ctx):
    b = Batch(fkv, 19, [(40, 1), (60, 2)], 2, 2, 64, 16, "bf16")
    cu, ln, tab = _i32(b.cu), _i32(b.len), _i32(b.table)
    out = torch.full_like(b.q, 7.0)

    def refused(call, exc=None):
        with pytest.raises(exc or fkv.FkvError) as e:
            call()
        if exc is None:
            assert e.value.code == -1
    go = lambda q=b.q, **o: ctx.page_attend(o.pop("pages", b.pages), q, cu, ln, tab, 2, 62, out=out, **o)
    refused(lambda: go(softcap=-1.0))
    refused(lambda: go(scale=float("inf")))
    refused(lambda: go(window=-1))
    refused(lambda: go(q=b.q.float()), ValueError)
    refused(lambda: ctx.page_attend(b.pages, b.q[:, :3], cu, ln, tab, 2, 62))
    refused(lambda: go(pages=fkv.Pages.empty(20, 2, 24, 64, torch.uint8)))
    refused(lambda: go(pages=fkv.Pages.empty(20, 2, 16, 128, torch.uint8)), ValueError)
    # 4-byte aligned numbers, pages a fraction of 16 numbers apart
    wide = torch.zeros((20, 2 * 32 + 2), dtype=torch.bfloat16, device="cuda")
    odd = wide[:, :64].unflatten(1, (2, 16, 2))
    refused(lambda: go(pages=fkv.Pages(*[torch.zeros((20, 2, 16, 32), dtype=torch.uint8, device="cuda")] * 2, odd, odd)))
    assert (out == 7).all() and ctx.sync_status() == 0


def _fill(how, shape, rng):
    """Numbers (step, middle) as memory that was never written may hold them."""
    if how == "random":
        return (rng.integers(0, 1 << 16, shape + (2,)).astype(np.uint32) << 16).view(np.float32)
    one = {"nan": (np.nan, np.nan), "middle": (0.25, np.inf), "step": (np.inf, 0.5), "minus": (-np.inf, -np.inf),
           "large": (2.0 ** 100, -2.0 ** 116), "small": (0.0, 2.0 ** 100)}[how]
    return np.broadcast_to(np.asarray(one, np.float32), shape + (2,))


def _leave_unwritten(fkv, b, how, where):
    """Pages as b's, but for the numbers of the positions where[r] of request r; what the oracle reads stays."""
    rng = np.random.default_rng(90)
    dev = []
    for s in b.numbers:
        s = s.copy()
        for r, j in enumerate(where):
            s[b.table[r, j // b.block], :, j % b.block] = _fill(how, (len(j), b.H), rng)
        dev.append(torch.from_numpy(s).bfloat16().cuda())
    b.pages = fkv.Pages(b.pages.k, b.pages.v, *dev)


@pytest.mark.parametrize("opt", [dict(), dict(softcap=20.0), dict(slopes=[0.1, 0.02, -0.01, 0.0])])
@pytest.mark.parametrize("how", ["nan", "middle", "step", "minus", "large", "small", "random"])
@pytest.mark.parametrize("new", [1, 7, 80])
@pytest.mark.parametrize("D,dtype,block", [(64, "f16", 48), (128, "bf16", 16)])
def test_positions_that_no_row_sees_hold_anything(fkv, ctx, D, dtype, block, new, how, opt):
    """Before a window and behind the sinks, in units of 16 positions of which rows see others."""
    b = Batch(fkv, 26, [(300, new), (45, new), (1000, new)], 2, 2, D, block, dtype)
    seen = [paged.visible(new, x, window=40, sinks=5).any(0) for x in b.len]
    assert all((~s).any() for s in seen[::2])
    _leave_unwritten(fkv, b, how, [np.flatnonzero(~s) for s in seen])
    b.check(ctx, rows=[0, new // 2, new - 1], window=40, sinks=5, **opt)


@pytest.mark.parametrize("opt", [dict(), dict(slopes=[0.1, 0.02, -0.01, 0.0])])
@pytest.mark.parametrize("how", ["nan", "middle", "step", "minus"])
@pytest.mark.parametrize("new", [4, 15, 80])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16"), (128, "f16")])
def test_padded_tokens_do_not_reach_the_others(fkv, ctx, D, dtype, new, how, opt):
    """The last tokens of each request were never stored: theirs are no one's rows, and the others' are as ever."""
    b = Batch(fkv, 27, [(300, new), (45, new), (7, new)], 2, 2, D, 16, dtype)
    _leave_unwritten(fkv, b, how, [np.arange(x - 3, x) for x in b.len])
    given = {k: torch.tensor(v, dtype=torch.float32, device="cuda") for k, v in opt.items()}
    out, lse = b.run(ctx, **given)
    assert ctx.sync_status() == 0
    b.compare(out, lse, np.arange(new - 3), None, opt.get("slopes"), 0.0, D ** -0.5, (), {})


@pytest.mark.parametrize("slopes", [None, [0.01, -0.02]])
@pytest.mark.parametrize("new", [1, 5, 60])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_near_the_largest_numbers(fkv, ctx, D, new, slopes):
    """Query rows of 2^121, whose elements cancel, against keys whose dimensions are alike: every score is zero before the
    bias, and every product and sum on the way an integer of few bits times a power of two.  What is left of the bounds
    above are the weights' and the values' roundings, the bias's error and the exponential's."""
    b = Batch(fkv, 28, [(150, new), (17, new)], 1, 2, D, 16, "bf16")
    c = b.codes[0]
    c[:] = (c[..., :1] & 15) * 17
    b.numbers[0] = b.numbers[0] * np.float32(2.0 ** -28)
    b.pages = fkv.Pages(torch.from_numpy(c).cuda(), b.pages.v, *(torch.from_numpy(s).bfloat16().cuda() for s in b.numbers))
    rng = np.random.default_rng(91)
    sign = rng.permuted(np.broadcast_to(np.arange(D) % 2 * 2 - 1, tuple(b.q.shape)), axis=-1)
    b.q = torch.from_numpy(np.ascontiguousarray(sign * 2.0 ** 121, np.float32)).bfloat16().cuda()
    opt = {} if slopes is None else dict(slopes=torch.tensor(slopes, device="cuda"))
    out, lse = b.run(ctx, scale=0.5, **opt)
    assert ctx.sync_status() == 0
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, length in enumerate(b.len):
        v = paged.gather4(b.codes[1], b.numbers[1], b.table[r], length)[0]
        for i in range(new):
            p = b.before[r] + i
            for u in range(2):
                x = (0.0 if slopes is None else slopes[u]) * (np.arange(p + 1) - p)
                w = np.exp(x)
                want, mass = w @ v[:p + 1] / w.sum(), np.abs(v[:p + 1]).max()
                ds = 2.0 ** -20 * (np.abs(x).max() + abs(np.log(w.sum())) + 16)
                # (a value is at most twice the mass in |c - 7.5| step + |middle|)
                bound = 2.0 ** -9 * np.abs(want) + (2.0 ** -10 + ds + length * 2.0 ** -30) * 2 * mass
                assert (np.abs(o[b.cu[r] + i, u] - want) <= bound).all()
                assert abs(l[b.cu[r] + i, u] - np.log(w.sum())) <= ds


@pytest.mark.parametrize("new", [1, 6, 70])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_far_above_one(fkv, ctx, D, new):
    """Rows of 2^50 to 2^66 against keys as much below."""
    b = Batch(fkv, 29, [(200, new), (33, new)], 1, 2, D, 32, "bf16")
    far = torch.exp2(torch.randint(50, 67, b.q.shape[:2] + (1,), device="cuda").float())
    b.q = (b.q.float() * far).bfloat16()
    b.numbers[0] = b.numbers[0] * np.float32(2.0 ** -60)
    b.pages = fkv.Pages(b.pages.k, b.pages.v, *(torch.from_numpy(s).bfloat16().cuda() for s in b.numbers))
    b.check(ctx, rows=[0, 1, new // 2, new - 1])


@pytest.mark.parametrize("new", [1, 7, 80])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_keys_of_any_size(fkv, ctx, D, dtype, new):
    """Keys' steps and middles apart by factors up to 2^60, and values' as well."""
    b = Batch(fkv, 30, [(200, new), (20, new)], 1, 2, D, 16, dtype, spread=0.1)
    rng = np.random.default_rng(61)
    for kv in (0, 1):
        far = np.exp2(rng.integers(-60, 1, b.numbers[kv].shape[:3]))[..., None].astype(np.float32)
        with np.errstate(invalid="ignore"):
            b.numbers[kv] = b.numbers[kv] * far
    b.pages = fkv.Pages(b.pages.k, b.pages.v, *(torch.from_numpy(s).bfloat16().cuda() for s in b.numbers))
    b.check(ctx, rows=[0, new // 2, new - 1])
