"""Paged 8-bit K/V cache on the GPU against its float64 oracle (oracle/paged.py).

Plans, codes and scales have to be equal.  An attention output may be off by
  half a step of its type, of the value (eps / 2 |o|);
  the weights' rounding to fp16 (half a step, 2^-11, of each weight; 2^-24 of
  the smallest normal ones is below 2^-30 of the largest weight, times the
  number of keys), and the scores' error as a relative one of the weights:
  fp32 products and sums of D terms, and the base-2 exponential's argument, each
  a few 2^-24 of the magnitudes that enter: 2^-20 (sum |q||k| scale + cap + bias
  + |lse| + 16);
the last two times the weighted sum of |v|.  lse: the scores' error alone."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
FMT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


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

    def __init__(self, fkv, seed, lens, H, G, D, block, fmt, dtype, by_token=False, spare=3, gap=0):
        rng = np.random.default_rng(seed)
        self.H, self.G, self.D, self.block, self.fmt = H, G, D, block, fmt
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
        self.codes = []
        self.scale = []
        for _ in range(2):
            # slots past a request's end and unused pages: any bytes, NaN codes among them
            c = rng.integers(0, 256, (nb, H, block, D), dtype=np.uint8)
            for r, x in enumerate(self.len):
                for j in range(need[r]):
                    m = min(block, x - j * block)
                    y = rng.standard_normal((H, m, D)) * (100 if fmt == "e4m3" else 32)
                    c[self.table[r, j], :, :m] = paged.to_codes(y, fmt)
            s = np.exp2(rng.integers(-9, -5, (nb, H))) if fmt == "e4m3" else np.exp(rng.standard_normal((nb, H)) * 0.3) / 32
            s = s.astype(np.float32)
            s[ids[at:]] = np.nan                             # no request's pages
            self.codes.append(c)
            self.scale.append(s)
        T = sum(self.new) + gap
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.q = torch.from_numpy(rng.standard_normal((T, H * G, D)).astype(np.float32)).to(DT[dtype]).cuda()
        dev = []
        for c in self.codes:
            t = torch.from_numpy(c).cuda().view(FMT[fmt]) if fmt == "e4m3" else torch.from_numpy(c.view(np.int8)).cuda()
            dev.append(t.transpose(1, 2).contiguous().transpose(1, 2) if by_token else t)
        self.pages = fkv.Pages(dev[0], dev[1], *(torch.from_numpy(s).cuda() for s in self.scale))

    def run(self, ctx, **opt):
        lse = torch.full((self.q.shape[0], self.H * self.G), 7.0, device="cuda")
        out = torch.full_like(self.q, 7.0)
        ctx.page_attend(self.pages, self.q, _i32(self.cu), _i32(self.len), _i32(self.table),
                        opt.pop("max_new", max(self.new)), opt.pop("max_len", max(self.len)), out=out, lse=lse, **opt)
        return out, lse

    def check(self, ctx, rows=None, prefix=None, slopes=None, softcap=0.0, scale=None, **mask):
        """rows: per request, the token indexes to compare (all if None)."""
        sc = self.D ** -0.5 if scale is None else scale
        opt = dict(mask, softcap=softcap, scale=scale)
        if prefix is not None:
            opt["prefix"] = _i32(prefix)
        if slopes is not None:
            opt["slopes"] = torch.tensor(slopes, dtype=torch.float32, device="cuda")
        out, lse = self.run(ctx, **opt)
        assert ctx.sync_status() == 0
        again, lse2 = self.run(ctx, **opt)
        assert torch.equal(out, again) and torch.equal(lse, lse2)          # the same bits every time
        eps = torch.finfo(self.q.dtype).eps / 2
        o, l, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), self.q.double().cpu().numpy()
        assert (o[self.cu[-1]:] == 7).all() and (l[self.cu[-1]:] == 7).all()
        for r, (n, length) in enumerate(zip(self.new, self.len)):
            if n == 0:
                continue
            k, v = (paged.gather(c, s, self.table[r], length, self.fmt) for c, s in zip(self.codes, self.scale))
            p0 = self.before[r]
            seen = paged.visible(n, length, mask.get("causal", True), mask.get("window", 0), mask.get("sinks", 0),
                                 None if prefix is None else prefix[r])
            pick = np.arange(n) if rows is None else np.unique(np.clip(np.asarray(rows), 0, n - 1))
            at = self.cu[r] + pick
            want = np.zeros((len(pick), self.H * self.G, self.D))
            wl, mass, size = want[:, :, 0].copy(), want.copy(), want[:, :, 0].copy()
            for e, i in enumerate(pick):
                a, b, c, d = paged.attend(q[self.cu[r] + i][None], k, v, sc, seen[i:i + 1], softcap, slopes, p0 + i)
                want[e], wl[e], mass[e], size[e] = a[0], b[0], c[0], d[0]
            bias = 0.0 if slopes is None else max(slopes) * length
            fin = np.isfinite(wl)
            ds = 2.0 ** -20 * (size + softcap + bias + np.where(fin, np.abs(wl), 0) + 16)
            bound = eps * np.abs(want) + (2.0 ** -11 + ds + length * 2.0 ** -30)[..., None] * mass * (1 + eps) + 1e-30
            assert (np.abs(o[at] - want) <= bound).all(), (r, np.max(np.abs(o[at] - want) / bound))
            assert np.array_equal(np.isneginf(l[at]), ~fin)
            assert (np.abs(np.where(fin, l[at], 0) - np.where(fin, wl, 0)) <= ds).all()


RAGGED = [(0, 1), (15, 1), (16, 1), (127, 1), (128, 1), (129, 1), (500, 1), (0, 0), (31, 1), (33, 1)]


@pytest.mark.parametrize("G", [1, 4, 7])
@pytest.mark.parametrize("block", [16, 48, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [64, 128])
def test_steps(fkv, ctx, D, fmt, dtype, block, G):
    Batch(fkv, 1, RAGGED, 2, G, D, block, fmt, dtype, by_token=G == 4, gap=2).check(ctx)


@pytest.mark.parametrize("first,second", [(3, -100), (20, -100), (-100, 20), (60, -60), (100, -20), (-100, -100)])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D,new", [(64, 1), (128, 7), (128, 40), (64, 300)])
def test_value_scales_far_apart(fkv, ctx, D, new, fmt, first, second):
    """Pages whose V scales differ by up to 2^120 (one of zeros has 2^-100) count alike in the sum of weights.
    A weight is held as 2^(y - m + bits) in float32, y = log2 of weight x scale: what lies 2^126 under 2^-130
    of the row's largest y (bits > 4, m at most the largest y rounded up) may be flushed to zero, in the sum
    and in the product; `lost` is that part of the weights."""
    b = Batch(fkv, 33, [(200, new), (64, new)], 2, 4, D, 32, fmt, "bf16")
    for r in range(2):
        for j in range(-(-b.len[r] // 32)):
            b.scale[1][b.table[r, j]] = 2.0 ** (second if j % 2 else first)
    b.pages.v_scale.copy_(torch.from_numpy(b.scale[1]))
    out, lse = b.run(ctx)
    assert ctx.sync_status() == 0
    o, l, q = (t.double().cpu().numpy() for t in (out, lse, b.q))
    for r, n in enumerate(b.new):
        k, v = (paged.gather(c, s, b.table[r], b.len[r], fmt) for c, s in zip(b.codes, b.scale))
        vs = b.scale[1][b.table[r, np.arange(b.len[r]) // 32]].astype(np.float64)       # [position, head]
        rows = slice(b.cu[r], b.cu[r + 1])
        want, wl, mass, size = paged.attend(q[rows], k, v, D ** -0.5, paged.visible(n, b.len[r], True, 0, 0, None))
        for i in range(n):
            end = b.before[r] + i + 1
            for u in range(b.H * b.G):
                x = D ** -0.5 * (k[u // b.G, :end] @ q[b.cu[r] + i, u])
                y = x / np.log(2) + np.log2(vs[:end, u // b.G])
                w = np.exp(x - wl[i, u])
                low = y < y.max() - 130
                lost, gone = w[low].sum(), w[low] @ np.abs(v[u // b.G, :end][low])
                assert lost < 0.5
                ds = 2.0 ** -20 * (size[i, u] + abs(wl[i, u]) + 16)
                assert abs(l[b.cu[r] + i, u] - wl[i, u]) <= ds - np.log1p(-lost)
                bound = (2.0 ** -8 * np.abs(want[i, u]) + (2.0 ** -11 + ds + end * 2.0 ** -30) * mass[i, u] * 1.01 +
                         (lost * mass[i, u] + gone) / (1 - lost) * 1.01 + 1e-30)
                assert (np.abs(o[b.cu[r] + i, u] - want[i, u]) <= bound).all()


MASKS = [dict(causal=False), dict(window=1), dict(window=37, sinks=4), dict(window=300, sinks=130), dict(softcap=5.0),
         dict(slopes=True), dict(prefix=[3, 90, 200, 1000, 0, 17]), dict(window=20, sinks=2, prefix=[0, 140, 300, 7, 1, 1]),
         dict(causal=False, window=30, sinks=3, softcap=20.0, slopes=True), dict(scale=-0.3)]


@pytest.mark.parametrize("opt", MASKS)
@pytest.mark.parametrize("D,fmt,dtype,G,block", [(64, "int8", "bf16", 3, 16), (128, "e4m3", "f16", 4, 32),
                                                 (128, "int8", "bf16", 1, 64)])
def test_masks(fkv, ctx, D, fmt, dtype, G, block, opt):
    lens = [(0, 5), (130, 3), (260, 40), (97, 150), (0, 1), (-3, 7)]
    b = Batch(fkv, 2, lens, 2, G, D, block, fmt, dtype)
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = [2.0 ** (-i / 2 - 1) for i in range(2 * G)]
    b.check(ctx, **opt)


@pytest.mark.parametrize("D,fmt", [(64, "e4m3"), (128, "int8")])
@pytest.mark.parametrize("new", [2, 4, 5, 16, 17, 64, 127, 128, 129, 256, 257, 700])
def test_prompts(fkv, ctx, D, fmt, new):
    rows = [0, 1, 2, 15, 16, 17, 31, 32, 63, 64, 65, 127, 128, 129, 255, 256, 400, 698, 699]
    Batch(fkv, 3, [(0, new), (70, new), (0, max(0, new - 3)), (200, 1)], 2, 4, D, 32, fmt, "bf16").check(ctx, rows=rows)


@pytest.mark.parametrize("lens", [[(9000, 1)], [(20000, 1), (0, 1), (40, 1)], [(8200, 4)], [(6000, 40), (10, 3)]])
@pytest.mark.parametrize("D,fmt", [(64, "int8"), (128, "e4m3")])
def test_long(fkv, ctx, D, fmt, lens):
    b = Batch(fkv, 4, lens, 1, 4, D, 64, fmt, "bf16")
    b.check(ctx, rows=[0, 3, 39])
    b.check(ctx, rows=[0, 3, 39], window=5000, sinks=4)


@pytest.mark.parametrize("where", ["first", "last", "spread"])
def test_scales_of_any_size_mix(fkv, ctx, where):
    """Pages whose value scales differ by 2^60, and a key scale that makes one page's scores dominate."""
    b = Batch(fkv, 5, [(700, 1), (333, 20)], 2, 2, 128, 16, "e4m3", "bf16")
    rng = np.random.default_rng(6)
    for s in b.scale:
        s[np.isnan(s)] = 1.0
    v = b.scale[1]
    used = b.table[0]
    if where == "spread":
        v *= np.exp2(rng.integers(-30, 30, v.shape)).astype(np.float32)
    else:
        v[used[0 if where == "first" else used.size - 1]] *= np.float32(2.0 ** 60)
        b.scale[0][used[3]] *= 8
    b.pages.k_scale.copy_(torch.from_numpy(b.scale[0]))
    b.pages.v_scale.copy_(torch.from_numpy(v))
    b.check(ctx)


@pytest.mark.parametrize("lens", [[(5000, 1)], [(900, 40)], [(3000, 300)]])
def test_pages_of_zeros(fkv, ctx, lens):
    """Values that are all zero, in pages of the smallest scale, at the first and at every page."""
    for every in (False, True):
        b = Batch(fkv, 21, lens, 1, 2, 128, 16, "e4m3", "bf16")
        for r in range(len(lens)):
            ids = b.table[r] if every else b.table[r, :2]
            b.codes[1][ids], b.scale[1][ids] = 0, np.float32(paged.FLOOR)
            b.pages.v.view(torch.uint8)[torch.from_numpy(ids).cuda()] = 0
        b.pages.v_scale.copy_(torch.from_numpy(b.scale[1]))
        b.check(ctx, rows=[0, 5, 39, 299])
        if every:
            assert not b.run(ctx)[0][:sum(b.new)].any()


def test_queries_of_any_size(fkv, ctx):
    b = Batch(fkv, 7, [(300, 2), (150, 30)], 2, 2, 64, 16, "int8", "bf16")
    b.q[0] *= 2.0 ** 60
    b.q[1] = 0
    b.q[3] *= 2.0 ** -130
    b.q[4, :, ::2] *= 2.0 ** -30
    b.q[0] *= 2.0 ** -62
    b.check(ctx)


def test_masked_nan_and_infinite_values_do_not_spread(fkv, ctx):
    """NaN codes and infinite or NaN scales where no row looks: past the end, before a window, on unused pages."""
    b = Batch(fkv, 8, [(200, 1), (45, 30), (0, 140)], 2, 4, 128, 16, "e4m3", "f16")
    out, lse = b.run(ctx)
    for r, x in enumerate(b.len):
        last = b.table[r, -(-x // 16) - 1]
        if x % 16:
            for c, t in zip(b.codes, (b.pages.k, b.pages.v)):
                c[last, :, x % 16:] = 0x7F
                t[last, :, x % 16:].view(torch.int8).fill_(0x7F)
    out2, lse2 = b.run(ctx)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    b.check(ctx)


def _nan_codes(b, where):
    """NaN codes at the positions where[r] of request r; what the oracle reads stays."""
    for t in (b.pages.k, b.pages.v):
        t = t.view(torch.uint8)
        for r, js in enumerate(where):
            for j in js:
                t[b.table[r, j // b.block], :, j % b.block] = 0x7f if j % 2 else 0xff


@pytest.mark.parametrize("opt", [dict(), dict(softcap=20.0), dict(slopes=[0.1, 0.02, 0.01, 0.0])])
@pytest.mark.parametrize("new", [1, 7, 80])
@pytest.mark.parametrize("D,dtype,block", [(64, "f16", 48), (128, "bf16", 16)])
def test_positions_that_no_row_sees_hold_anything(fkv, ctx, D, dtype, block, new, opt):
    """Before a window and behind the sinks, in units of 16 positions of which rows see others."""
    b = Batch(fkv, 26, [(300, new), (45, new), (1000, new)], 2, 2, D, block, "e4m3", dtype)
    seen = [paged.visible(new, x, window=40, sinks=5).any(0) for x in b.len]
    assert all((~s).any() for s in seen[::2])
    _nan_codes(b, [np.flatnonzero(~s) for s in seen])
    b.check(ctx, rows=[0, new // 2, new - 1], window=40, sinks=5, **opt)


@pytest.mark.parametrize("new", [4, 15, 80, 200])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_padded_tokens_do_not_reach_the_others(fkv, ctx, D, dtype, new):
    """The last tokens of each request were never stored, of one nothing of their page: theirs are no one's rows, and
    the others' are as ever: twice what either may be off by, 2^-10 covering weights and scores, and 14 the largest value."""
    b = Batch(fkv, 27, [(288 + (19 - new) % 16, new), (45, new), (7, new)], 2, 2, D, 16, "e4m3", dtype)
    want, lse = b.run(ctx)
    _nan_codes(b, [np.arange(x - 3, x) for x in b.len])
    for s in (b.pages.k_scale, b.pages.v_scale):
        s[b.table[0, b.len[0] // 16]] = float("nan")
    out, lse2 = b.run(ctx)
    assert ctx.sync_status() == 0
    eps = torch.finfo(b.q.dtype).eps / 2
    for x in b.cu[:-1]:
        o, w = (y[x:x + new - 3].double() for y in (out, want))
        assert ((o - w).abs() <= 2 * (eps * w.abs() + 2.0 ** -10 * 14)).all()
        assert ((lse2 - lse)[x:x + new - 3].abs() <= 2.0 ** -10).all()


def test_padded_rows_and_skipped_requests_stay(fkv, ctx):
    b = Batch(fkv, 9, [(40, 1), (60, 5), (20, 1)], 2, 2, 64, 16, "e4m3", "bf16", gap=5)
    good, _ = b.run(ctx)
    out, lse = b.run(ctx, max_new=4)                       # the second request has more new tokens than declared
    assert ctx.sync_status() == -2
    assert (out[1:6] == 7).all() and (lse[1:6] == 7).all()
    assert torch.equal(out[:1], good[:1]) and torch.equal(out[6:7], good[6:7])
    out, _ = b.run(ctx, max_len=50)                        # ... or is longer
    assert ctx.sync_status() == -2
    assert (out[1:6] == 7).all() and torch.equal(out[:1], good[:1])


def test_requests_after_one_that_does_not_hold_together_are_served(fkv, ctx):
    """Row numbers of two requests that are out of order: the third, whose shares are joined by their own launch,
    gets its row all the same."""
    b = Batch(fkv, 45, [(10, 1), (10, 1), (20000, 1)], 1, 4, 64, 16, "int8", "f16", gap=2)
    good, lse = b.run(ctx)
    assert ctx.sync_status() == 0
    b.cu = np.array([0, 9, 2, 3])
    out, lse2 = b.run(ctx)
    assert ctx.sync_status() == -2
    assert torch.equal(out[2], good[2]) and torch.equal(lse2[2], lse[2])
    keep = [0, 1, 3, 4]
    assert (out[keep] == 7).all() and (lse2[keep] == 7).all()


def test_a_page_outside_the_pool_is_reported(fkv, ctx):
    b = Batch(fkv, 10, [(40, 1), (60, 5)], 1, 2, 64, 16, "e4m3", "bf16")
    good, _ = b.run(ctx)
    for bad in (-5, 1 << 30):
        keep = b.table[1, 1]
        b.table[1, 1] = bad
        out, _ = b.run(ctx)
        assert ctx.sync_status() == -2
        assert torch.equal(out[:1], good[:1])
        b.table[1, 1] = keep


def test_requests_without_positions(fkv, ctx):
    """Lengths of zero: nothing to see, with new tokens and without."""
    for lens in ([(0, 0), (0, 1)], [(-1, 1), (0, 2), (-9, 9)], [(-40, 40), (5, 3)]):
        Batch(fkv, 22, lens, 2, 4, 64, 16, "int8", "f16").check(ctx)
    b = Batch(fkv, 23, [(-2, 2)], 1, 1, 128, 16, "e4m3", "bf16")
    out, lse = b.run(ctx, max_len=0)
    assert ctx.sync_status() == 0 and not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("new", [1, 60])
def test_views_with_strides(fkv, ctx, new):
    """K and V pages side by side in one tensor, queries and outputs as slices of wider rows."""
    b = Batch(fkv, 24, [(300, new), (17, 1)], 3, 2, 128, 32, "e4m3", "bf16")
    want, lse = b.run(ctx)
    both = torch.stack([b.pages.k.view(torch.uint8), b.pages.v.view(torch.uint8)], 1)      # [pages, 2, heads, block, dim]
    scales = torch.stack([b.pages.k_scale, b.pages.v_scale], 2)                             # [pages, heads, 2]
    pages = fkv.Pages(both[:, 0].view(torch.float8_e4m3fn), both[:, 1].view(torch.float8_e4m3fn), scales[:, :, 0], scales[:, :, 1])
    T = b.q.shape[0]
    wide = torch.full((T, 14, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 4:10] = b.q
    res = torch.full((T, 9, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.page_attend(pages, wide[:, 4:10], _i32(b.cu), _i32(b.len), _i32(np.hstack([b.table, b.table]))[:, :b.table.shape[1]],
                    max(b.new), max(b.len), out=res[:, 2:8])
    assert ctx.sync_status() == 0
    assert torch.equal(res[:, 2:8], want) and (res[:, :2] == 7).all() and (res[:, 8:] == 7).all()


@pytest.mark.parametrize("lens", [[(40, 1)], [(300, 1), (5, 2)], [(900, 5)], [(20000, 1)], [(100, 60)], [(3000, 40)], [(90, 700)]])
def test_output_over_the_queries(fkv, ctx, lens):
    """out may be q itself: one share, shares joined in their cluster or by a launch, few rows and many."""
    b = Batch(fkv, 46, lens, 2, 4, 128, 16, "e4m3", "bf16", gap=1)
    want, _ = b.run(ctx)
    q = b.q.clone()
    ctx.page_attend(b.pages, q, _i32(b.cu), _i32(b.len), _i32(b.table), max(b.new), max(b.len), out=q)
    assert ctx.sync_status() == 0
    assert torch.equal(q[:-1], want[:-1]) and torch.equal(q[-1], b.q[-1])


def test_calls_of_nothing(fkv, ctx):
    """No tokens, no requests, or a bound of no new tokens: nothing is done."""
    b = Batch(fkv, 47, [(40, 1), (60, 5)], 2, 2, 64, 16, "int8", "f16")
    out, lse = b.run(ctx, max_new=0)
    assert (out == 7).all() and (lse == 7).all()
    cu, none = _i32([0]), _i32([])
    out = torch.full_like(b.q, 7.0)
    ctx.page_attend(b.pages, b.q, cu, none, _i32(b.table), 5, 65, out=out)
    ctx.page_attend(b.pages, b.q[:0], _i32([0, 0, 0]), _i32(b.len), _i32(b.table), 5, 65, out=out[:0])
    assert (out == 7).all() and ctx.sync_status() == 0


@pytest.mark.parametrize("by_token", [False, True])
def test_pages_past_four_gigabytes(fkv, ctx, by_token):
    """Byte offsets that do not fit 32 bits: a pool of 5 GiB whose last pages are written, read and attended to."""
    H, D, block = 2, 128, 64
    nb = (5 << 30) // (H * D * block)
    shape = (nb, block, H, D) if by_token else (nb, H, block, D)
    pools = [torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
    views = [p.transpose(1, 2) if by_token else p for p in pools]
    scale = [torch.zeros((nb, H), device="cuda") for _ in range(2)]
    pages = fkv.Pages(views[0], views[1], scale[0], scale[1])
    rng = np.random.default_rng(25)
    n = 150
    ids = np.array([nb - 1, nb - 3, nb // 2 + 7])
    slots = ids[np.arange(n) // block] * block + np.arange(n) % block
    kv = torch.from_numpy(rng.standard_normal((n, 2, H, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    ctx.page_write(pages, kv[:, 0], kv[:, 1], torch.from_numpy(slots).cuda())
    small = [np.zeros((3, H, block, D), np.uint8) for _ in range(2)]
    sc = [np.zeros((3, H), np.float32) for _ in range(2)]
    for i in range(2):
        paged.write(small[i], sc[i], kv[:, i].double().cpu().numpy(), np.arange(n), "int8")
        at = torch.from_numpy(ids).cuda()
        got = views[i][at].contiguous().view(torch.uint8).cpu().numpy()
        for j in range(3):
            m = min(block, n - j * block)
            assert np.array_equal(got[j, :, :m], small[i][j, :, :m])
        assert np.array_equal(scale[i][at].cpu().numpy(), sc[i])
    table = _i32([ids])
    out = torch.zeros((1, 1, H, n, D), dtype=torch.float32, device="cuda")
    ctx.page_read(pages, _i32([n]), table, 0, n, 0, out, None)
    want = paged.gather(small[0], sc[0], np.arange(3), n, "int8")
    assert np.array_equal(out[0, 0].cpu().numpy(), want.astype(np.float32))
    for new in (1, 40):
        q = torch.from_numpy(rng.standard_normal((new, 2 * H, D)).astype(np.float32)).to(torch.bfloat16).cuda()
        o = ctx.page_attend(pages, q, _i32([0, new]), _i32([n]), table, new, n)
        k, v = (paged.gather(small[i], sc[i], np.arange(3), n, "int8") for i in range(2))
        w, _, mass, size = paged.attend(q.double().cpu().numpy(), k, v, D ** -0.5, paged.visible(new, n), p0=n - new)
        bound = 2.0 ** -8 * np.abs(w) + (2.0 ** -11 + 2.0 ** -20 * (size + 24))[..., None] * mass
        assert (np.abs(o.double().cpu().numpy() - w) <= bound * (1 + 2.0 ** -8)).all()
    assert ctx.sync_status() == 0


def test_first_calls_inside_a_capture():
    """A fresh process captures every paged call before any has run, replays it twice, and gets what eager calls give."""
    import os
    import subprocess
    import sys
    code = """
import torch, paper_2607_07144_gb300 as fkv
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
def state():
    g = torch.Generator(device="cuda").manual_seed(1)
    p = fkv.Pages.empty(40, 2, 16, 64, torch.int8)
    for t in (p.k, p.v): t.zero_()
    return dict(p=p, new=i32([300, 1, 40]), ln=i32([0, 0, 0]), tab=torch.full((3, 24), -1, dtype=torch.int32, device="cuda"),
                free=torch.arange(40, dtype=torch.int32, device="cuda"), taken=i32([0]), cu=i32([0] * 4),
                slots=torch.zeros(5000, dtype=torch.int64, device="cuda"), pos=torch.zeros(5000, dtype=torch.int32, device="cuda"),
                x=torch.randn((5000, 8, 64), generator=g, device="cuda", dtype=torch.float16),
                o=torch.zeros((5000, 4, 64), dtype=torch.float16, device="cuda"),
                s=torch.zeros((3, 4, 64), dtype=torch.float16, device="cuda"), one=i32([0, 1, 2, 3]),
                k=torch.zeros((1, 3, 2, 320, 64), device="cuda"), v=torch.zeros((1, 3, 2, 320, 64), device="cuda"))
def step(ctx, d):
    ctx.page_plan(d["new"], d["ln"], d["tab"], d["free"], d["taken"], 16, d["cu"], d["slots"], d["pos"])
    ctx.page_write(d["p"], d["x"][:, :2], d["x"][:, 2:4], d["slots"])
    ctx.page_attend(d["p"], d["x"][:, 4:], d["cu"], d["ln"], d["tab"], 300, 320, out=d["o"])
    ctx.page_attend(d["p"], d["x"][:3, 4:], d["one"], d["ln"], d["tab"], 1, 320, out=d["s"])
    ctx.page_read(d["p"], d["ln"], d["tab"], 0, 320, 0, d["k"], d["v"])
ctx = fkv.Context(256)
a, b = state(), state()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step(ctx, a)
for new in ([300, 1, 40], [5, 3, 1]):
    for d in (a, b): d["new"].copy_(i32(new))
    g.replay()
    step(ctx, b)
    assert ctx.sync_status() == 0
    for n in ("ln", "tab", "taken", "cu", "slots", "pos", "o", "s", "k", "v"):
        assert torch.equal(a[n], b[n]), n
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=280)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("slopes", [None, [0.0, 0.0]])
@pytest.mark.parametrize("D,fmt,dtype", [(64, "int8", "f16"), (128, "e4m3", "bf16")])
def test_weights_stored_before_a_larger_score_keep_their_share(fkv, ctx, D, fmt, dtype, slopes):
    """A tile of many rows whose second half holds a score 2^18 times its first half's largest weight, and more
    above what came before; its value is zero (a sink's), so that the output is the first half's alone: 2^-18 of
    the largest weight times 100, far above the 2^-30 below which weights may be zero."""
    b = Batch(fkv, 40, [(512, 64)], 1, 2, D, 16, fmt, dtype)
    for c in b.codes:
        c[:] = 0
    k, v = (c[b.table[0]].transpose(1, 0, 2, 3).reshape(1, -1, D) for c in b.codes)
    one = lambda x: paged.to_codes(np.array([x]), fmt)[0]
    k[0, 138, 0], k[0, 228, 0], v[0, 138] = one(8.0), one(26.0), one(100.0)        # 138, 228: halves of 128 .. 255
    for c, x, t in zip(b.codes, (k, v), (b.pages.k, b.pages.v)):
        c[b.table[0]] = x.reshape(1, -1, 16, D).transpose(1, 0, 2, 3)
        t.view(torch.uint8).copy_(torch.from_numpy(c))
    for s, t in zip(b.scale, (b.pages.k_scale, b.pages.v_scale)):
        s[:] = 1
        t.fill_(1.0)
    b.q.zero_()
    b.q[:, :, 0] = 1.0
    b.check(ctx, scale=float(np.log(2.0)), slopes=slopes)
    assert (b.run(ctx, scale=float(np.log(2.0)))[0][:, :, 0] > 3e-4).all()


def _compare(b, ctx, rel=2.0 ** -20, const=16.0, rows=None, **opt):
    """Batch.check with an allowance of its own for the scores' error: rel (size + |lse|) + 2^-20 const;
    and outputs below the type's smallest normal number, which step by eps times that (fp16: off by 2^-25)."""
    out, lse = b.run(ctx, **opt)
    assert ctx.sync_status() == 0
    eps, tiny = torch.finfo(b.q.dtype).eps / 2, torch.finfo(b.q.dtype).tiny
    o, l, q = (t.double().cpu().numpy() for t in (out, lse, b.q))
    for r, (n, length) in enumerate(zip(b.new, b.len)):
        k, v = (paged.gather(c, s, b.table[r], length, b.fmt) for c, s in zip(b.codes, b.scale))
        seen = paged.visible(n, length, opt.get("causal", True), opt.get("window", 0), opt.get("sinks", 0), None)
        for i in range(n) if rows is None else sorted({x % n for x in rows}):
            at = b.cu[r] + i
            want, wl, mass, size = paged.attend(q[at][None], k, v, opt.get("scale") or b.D ** -0.5, seen[i:i + 1],
                                                opt.get("softcap", 0.0), None, b.before[r] + i)
            ds = rel * (size[0] + np.abs(wl[0])) + 2.0 ** -20 * const
            bound = eps * np.abs(want[0]) + (2.0 ** -11 + ds + length * 2.0 ** -30)[:, None] * mass[0] * (1 + eps) + eps * tiny
            assert (np.abs(o[at] - want[0]) <= bound).all(), (r, i, np.max(np.abs(o[at] - want[0]) / bound))
            assert (np.abs(l[at] - wl[0]) <= ds).all(), (r, i, np.max(np.abs(l[at] - wl[0]) / ds))


@pytest.mark.parametrize("cap", [0.7, 30.0, 64.0, 65.0, 300.0, 1e3, 1e5, 1e8, 1e30, 3e38])
@pytest.mark.parametrize("scale", [None, 5.0])
@pytest.mark.parametrize("D,fmt,dtype,G", [(64, "int8", "f16", 1), (128, "e4m3", "bf16", 4)])
def test_caps_of_any_size(fkv, ctx, D, fmt, dtype, G, scale, cap):
    """cap tanh(s / cap) is s for a large cap: the allowance does not grow with the cap.  Up to 64 it is taken as
    cap - 2 cap / (1 + e^2y): exponential and quotient of 2 ulp each and the sums' roundings err by
    cap 1.4 2^-22 <= 23 2^-20.  Above, relative to s: e^2y >= e gives 2^-20.8, the series below it less, beside
    the products' own error."""
    b = Batch(fkv, 41, [(130, 3), (60, 40), (300, 1), (0, 2)], 2, G, D, 16, fmt, dtype)
    _compare(b, ctx, 2.0 ** -19, 40.0, [0, -1], softcap=cap, scale=scale)


@pytest.mark.parametrize("opt", [dict(), dict(softcap=20.0), dict(softcap=1e4), dict(slopes=True), dict(causal=False)])
@pytest.mark.parametrize("window,sinks", [(20, 0), (20, 2), (300, 130)])
@pytest.mark.parametrize("D,fmt,dtype,new", [(64, "e4m3", "f16", 1), (128, "e4m3", "bf16", 5), (64, "e4m3", "bf16", 60),
                                             (128, "int8", "f16", 200), (128, "int8", "bf16", 1)])
def test_pages_that_no_row_sees_are_not_looked_up(fkv, ctx, D, fmt, dtype, new, window, sinks, opt):
    """Pages behind a window may be gone: their table entries lie outside the pool, or name a page of NaN codes
    whose scales are NaN and infinite; page 0 is such a page too."""
    b = Batch(fkv, 42, [(700, new), (333, new), (5, 1)], 2, 4, D, 16, fmt, dtype)
    spare = sorted(set(range(b.codes[0].shape[0])) - set(b.table.ravel().tolist()))
    if 0 not in spare:                                     # a spare page changes places with page 0
        z = spare.pop()
        b.table = np.where(b.table == 0, z, b.table)
        for x in b.codes + b.scale:
            x[[0, z]] = x[[z, 0]]
    poison = [0] + [x for x in spare if x]
    for c, s in zip(b.codes, b.scale):
        c[poison] = 0x7F
        s[poison] = np.nan
        s[poison[1:], 0] = np.inf
    for t, x in zip((b.pages.k.view(torch.uint8), b.pages.v.view(torch.uint8), b.pages.k_scale, b.pages.v_scale),
                    b.codes + b.scale):
        t.copy_(torch.from_numpy(x))
    gone = 0
    for r, (n, length) in enumerate(zip(b.new, b.len)):
        seen = paged.visible(n, length, opt.get("causal", True), window, sinks, None).any(0)
        for j in range(-(-length // 16)):
            if not seen[16 * j:16 * j + 16].any():
                b.table[r, j] = (-1, -2, poison[0], poison[-1])[j % 4]
                gone += 1
    assert gone > 3
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = [0.5, 0.25, 0.03, -0.02] * 2
    b.check(ctx, rows=[0, 1, new // 2, new - 1], window=window, sinks=sinks, **opt)


# ------------------------------------------------------------------ plans --
def _plan(ctx, new, ln, table, free, taken, block, rows, in_place=False):
    t = dict(new=_i32(new), ln=_i32(ln), table=_i32(table), free=_i32(free), taken=_i32([taken]),
             cu=_i32(np.full(len(new) + 1, 5)), slots=torch.full((rows,), 9, dtype=torch.int64, device="cuda"),
             pos=_i32(np.full(rows, 9)))
    lo, to = (None, None) if in_place else (_i32(np.zeros(len(new))), _i32([0]))
    ctx.page_plan(t["new"], t["ln"], t["table"], t["free"], t["taken"], block, t["cu"], t["slots"], t["pos"], lo, to)
    got = [t["cu"], t["slots"], t["pos"], t["ln"] if in_place else lo, t["taken"] if in_place else to, t["table"], t["free"]]
    return [x.cpu().numpy() for x in got]


def _plan_case(seed, n, block, hi, new_hi, ends, spare=4):
    rng = np.random.default_rng(seed)
    ln = rng.integers(0, hi + 1, n)
    new = rng.integers(0, new_hi + 1, n)
    new[rng.random(n) < ends] = -1
    need = -(-ln // block)
    width = int(max(((ln + np.maximum(new, 0) + block - 1) // block).max(), 1)) + 1
    total = int(need.sum() + ((np.maximum(new, 0) + block - 1) // block + 1).sum()) + spare
    ids = rng.permutation(total)
    table = np.full((n, width), -1, np.int64)
    at = 0
    for r in range(n):
        table[r, :need[r]] = ids[at:at + need[r]]
        at += need[r]
    free = np.concatenate([np.full(at, -1), ids[at:]])
    return new, ln, table, free, at, int(np.maximum(new, 0).sum())


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,block,hi,new_hi,ends", [(1, 16, 0, 1, 0), (1, 16, 100, 5000, 0), (3, 48, 40, 0, 0),
                                                    (7, 32, 100, 3, 0.4), (64, 16, 2000, 1, 0.1), (65, 64, 3, 200, 0.5),
                                                    (513, 16, 50, 40, 0.2), (5000, 32, 90, 2, 0.3), (16384, 16, 20, 1, 0.1)])
def test_plan(ctx, n, block, hi, new_hi, ends, in_place):
    new, ln, table, free, taken, tokens = _plan_case(n, n, block, hi, new_hi, ends)
    want = paged.plan(new, ln, table, free, taken, block, tokens + 11)
    assert want[7]
    got = _plan(ctx, new, ln, table, free, taken, block, tokens + 11, in_place)
    assert ctx.sync_status() == 0
    for g, w in zip(got, want[:7]):
        assert np.array_equal(g.reshape(-1), np.asarray(w).reshape(-1))


@pytest.mark.parametrize("why", ["free", "rows", "width", "taken", "negative", "huge", "huge length"])
def test_plan_that_does_not_fit_changes_nothing(ctx, why):
    new, ln, table, free, taken, tokens = _plan_case(77, 40, 16, 100, 30, 0.2)
    rows = tokens
    if why == "free":
        new[:], rows = 30, 30 * 40
        free = free[:taken + 1]
    if why == "rows":
        rows = tokens - 1
    if why == "width":
        table = np.ascontiguousarray(table[:, :3])
    if why == "taken":
        taken = 0
    if why == "negative":
        ln[7] = -1
    if why == "huge":
        new[3:9] = 1 << 30
    if why == "huge length":
        ln[5] = (1 << 30) + 1
    want = paged.plan(new, ln, table, free, taken, 16, rows)
    assert not want[7]
    got = _plan(ctx, new, ln, table, free, taken, 16, rows)
    assert ctx.sync_status() == -2
    for g, w in zip(got, want[:7]):
        assert np.array_equal(g.reshape(-1), np.asarray(w).reshape(-1))


def test_plan_without_requests(ctx):
    got = _plan(ctx, np.zeros(0, np.int64), np.zeros(0, np.int64), np.zeros((1, 2)), [4, 5], 1, 16, 3)
    assert ctx.sync_status() == 0
    assert got[0].tolist() == [0] and got[1].tolist() == [-1] * 3 and got[4].tolist() == [1]


# ----------------------------------------------------------------- writes --
def _pool(fkv, rng, nb, H, D, block, fmt, by_token=False):
    codes = [rng.integers(0, 256, (nb, H, block, D), dtype=np.uint8) for _ in range(2)]
    for c in codes:
        c[(c & 127) == 127] = 5                               # valid codes everywhere
        c[c == 128] = 5
    scale = [np.exp2(rng.integers(-9, -4, (nb, H))).astype(np.float32) for _ in range(2)]
    dev = []
    for c in codes:
        t = torch.from_numpy(c).cuda().view(FMT[fmt]) if fmt == "e4m3" else torch.from_numpy(c.view(np.int8)).cuda()
        dev.append(t.transpose(1, 2).contiguous().transpose(1, 2) if by_token else t)
    return codes, scale, fkv.Pages(dev[0], dev[1], *(torch.from_numpy(s).cuda() for s in scale))


def _same(pages, codes, scale):
    for t, c in zip((pages.k, pages.v), codes):
        assert np.array_equal(t.view(torch.uint8).cpu().numpy(), c)
    for t, s in zip((pages.k_scale, pages.v_scale), scale):
        assert np.array_equal(t.cpu().numpy().view(np.uint32), s.view(np.uint32))


@pytest.mark.parametrize("block", [16, 48, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D,H", [(64, 3), (128, 2)])
def test_write(fkv, ctx, D, H, fmt, dtype, block):
    rng = np.random.default_rng(11)
    runs = [(0, 1), (3, 1), (block - 1, 1), (0, block), (5, 7), (block - 3, block + 10), (1, 0), (0, 3 * block + 1)]
    nb = sum(-(-(o + n) // block) for o, n in runs) + 2
    codes, scale, pages = _pool(fkv, rng, nb, H, D, block, fmt, by_token=H == 3)
    ids, at, slots = rng.permutation(nb), 0, []
    for off, n in runs:
        pos = off + np.arange(n)
        slots += list(ids[at + pos // block] * block + pos % block) + [-1] * (n % 2)
        at += -(-(off + n) // block)
    slots = np.array(slots)
    T = len(slots)
    kv = torch.from_numpy((rng.standard_normal((T, 2, H, D)) * np.exp(rng.standard_normal((T, 1, 1, 1)) * 2))
                          .astype(np.float32)).to(DT[dtype]).cuda()
    kv[4, 0] = 0
    k, v = kv[:, 0], kv[:, 1]
    ctx.page_write(pages, k, v, torch.from_numpy(slots).cuda())
    assert ctx.sync_status() == 0
    for c, s, x in zip(codes, scale, (k, v)):
        paged.write(c, s, x.double().cpu().numpy(), slots, fmt)
    _same(pages, codes, scale)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_token_by_token(fkv, ctx, fmt):
    """A page filled one token a call, scales growing and not: the codes of every step."""
    rng = np.random.default_rng(12)
    codes, scale, pages = _pool(fkv, rng, 3, 2, 64, 16, fmt)
    for i in range(20):
        slots = np.array([16 + i if i < 16 else 32 + i - 16])
        x = [torch.from_numpy(rng.standard_normal((1, 2, 64)).astype(np.float32)).cuda() * 2.0 ** int(rng.integers(-6, 6))
             for _ in range(2)]
        ctx.page_write(pages, x[0], x[1], torch.from_numpy(slots).cuda())
        for c, s, y in zip(codes, scale, x):
            paged.write(c, s, y.double().cpu().numpy(), slots, fmt)
    assert ctx.sync_status() == 0
    _same(pages, codes, scale)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_write_of_unusual_values(fkv, ctx, fmt):
    rng = np.random.default_rng(13)
    codes, scale, pages = _pool(fkv, rng, 4, 1, 64, 16, fmt)
    x = rng.standard_normal((6, 1, 64)).astype(np.float32)
    x[0, 0, :4] = [np.inf, -np.inf, 0.0, -0.0]
    x[1] = 0
    x[2] *= np.float32(2.0 ** -120)
    x[3] *= np.float32(2.0 ** 100)
    x[4, 0, 0] = 448.0 * 4
    x[5] = 1e-42
    slots = np.array([0, 16, 17, 33, 34, 48])
    t = torch.from_numpy(x).cuda()
    ctx.page_write(pages, t, t, torch.from_numpy(slots).cuda())
    assert ctx.sync_status() == 0
    for c, s in zip(codes, scale):
        paged.write(c, s, x.astype(np.float64), slots, fmt)
    _same(pages, codes, scale)
    # NaN: stored as zero, and reported
    x[0, 0, 5] = np.nan
    t = torch.from_numpy(x).cuda()
    ctx.page_write(pages, t, t, torch.from_numpy(slots).cuda())
    assert ctx.sync_status() == -5
    for c, s in zip(codes, scale):
        paged.write(c, s, x.astype(np.float64), slots, fmt)
    _same(pages, codes, scale)


def test_slots_outside_the_pool_are_skipped_and_reported(fkv, ctx):
    rng = np.random.default_rng(14)
    codes, scale, pages = _pool(fkv, rng, 3, 2, 64, 16, "e4m3")
    x = torch.from_numpy(rng.standard_normal((4, 2, 64)).astype(np.float32)).cuda()
    slots = np.array([4, 48, 1 << 40, 20])
    ctx.page_write(pages, x, x, torch.from_numpy(slots).cuda())
    assert ctx.sync_status() == -2
    for c, s in zip(codes, scale):
        paged.write(c, s, x.double().cpu().numpy(), slots, "e4m3")
    _same(pages, codes, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("T", [3, 200, 700])
def test_write_keeps_scales_within_the_pools_range(fkv, ctx, T, fmt, dtype):
    """A page's scale is at most 2^100, as attention wants it: values beyond its largest code are stored as that."""
    H, D = 8, 64
    rng = np.random.default_rng(43)
    nb = max(T // 16, 3) + 1
    codes, scale, pages = _pool(fkv, rng, nb, H, D, 16, fmt)
    x = torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).cuda() * 2.0 ** 118
    x[0] *= 2.0 ** -60
    x[1, 0, 3] = float("inf")
    x = x.to(DT[dtype])
    slots = np.arange(T) * (1 if T > 16 else 16)           # runs of a page, or a token a page
    ctx.page_write(pages, x, x, torch.from_numpy(slots).cuda())
    for c, s in zip(codes, scale):
        paged.write(c, s, x.double().cpu().numpy(), slots, fmt)
    _same(pages, codes, scale)
    assert max(s.max() for s in scale) == 2.0 ** 100
    # keys of the smallest scale, queries of zero: the mean of the values
    pages.k_scale.fill_(2.0 ** -100)
    q = torch.zeros((1, H, D), dtype=torch.bfloat16, device="cuda")
    n = 16 if T > 16 else 1
    table = _i32([[1]]) if T > 16 else _i32([[2]])
    lse = torch.zeros((1, H), device="cuda")
    out = ctx.page_attend(pages, q, _i32([0, 1]), _i32([n]), table, 1, n, lse=lse)
    assert ctx.sync_status() == 0
    v = paged.gather(codes[1], scale[1], [1 if T > 16 else 2], n, fmt)
    want = v.mean(1)
    bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(v).mean(1)
    assert (np.abs(out[0].double().cpu().numpy() - want) <= bound).all()
    assert np.abs(lse[0].cpu().numpy() - np.log(n)).max() < 1e-4


# ------------------------------------------------------------------ reads --
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D,fmt,block", [(64, "int8", 16), (128, "e4m3", 48), (128, "int8", 128)])
def test_read(fkv, ctx, D, fmt, block, dtype):
    lens = [(200, 0), (0, 0), (17, 0), (129, 0), (64, 0)]
    b = Batch(fkv, 15, lens, 3, 1, D, block, fmt, "bf16", by_token=block == 48)
    for t0, t1 in ((0, 200), (5, 130), (16, 17), (150, 220), (3, 3)):
        shape = (2, 6, 3, 230, D)
        k, v = (torch.full(shape, 7.0, dtype=DT[dtype], device="cuda") for _ in range(2))
        ctx.page_read(b.pages, _i32(b.len), _i32(b.table), t0, t1, 1, k, v)
        assert ctx.sync_status() == 0
        for c, s, got in zip(b.codes, b.scale, (k, v)):
            want = torch.full(shape, 7.0, dtype=DT[dtype])
            for r, x in enumerate(b.len):
                to = min(x, t1)
                if to > t0:
                    y = paged.gather(c, s, b.table[r], x, fmt)[:, t0:to].astype(np.float32)   # exact or one rounding
                    want[1, r, :, t0:to] = torch.from_numpy(y).to(DT[dtype])
            assert torch.equal(got.cpu(), want)
        one = torch.full(shape, 7.0, dtype=DT[dtype], device="cuda")
        ctx.page_read(b.pages, _i32(b.len), _i32(b.table), t0, t1, 1, None, one)
        assert torch.equal(one, v)


def test_read_of_pages_outside_the_pool(fkv, ctx):
    b = Batch(fkv, 16, [(60, 0), (40, 0)], 2, 1, 64, 16, "int8", "bf16")
    k = torch.full((1, 2, 2, 60, 64), 7.0, dtype=torch.float16, device="cuda")
    b.table[0, 1] = 10 ** 6
    ctx.page_read(b.pages, _i32([60, 500]), _i32(b.table), 0, 60, 0, k, None)
    assert ctx.sync_status() == -2
    assert (k[0, 0, :, 16:32] == 7).all() and (k[0, 0, :, :16] != 7).any()


# --------------------------------------------------------------- refusals --
def test_refusals(fkv, ctx):
    b = Batch(fkv, 17, [(40, 1), (60, 2)], 2, 2, 64, 16, "e4m3", "bf16")
    cu, ln, tab = _i32(b.cu), _i32(b.len), _i32(b.table)
    out = torch.full_like(b.q, 7.0)

    def refused(call, exc=None):
        with pytest.raises(exc or fkv.FkvError) as e:
            call()
        if exc is None:
            assert e.value.code == -1
    go = lambda **o: ctx.page_attend(b.pages, o.pop("q", b.q), cu, ln, o.pop("tab", tab), 2, o.pop("max_len", 62), out=out, **o)
    refused(lambda: go(softcap=-1.0))
    refused(lambda: go(softcap=float("nan")))
    refused(lambda: go(scale=float("inf")))
    refused(lambda: go(window=-1))
    refused(lambda: go(sinks=-1))
    refused(lambda: go(max_len=(1 << 30) + 1))
    refused(lambda: go(q=b.q[:, :3].contiguous()), ValueError)                 # out of another shape
    refused(lambda: ctx.page_attend(b.pages, b.q[:, :3], cu, ln, tab, 2, 62))   # 3 query heads for 2 KV heads
    refused(lambda: ctx.page_attend(b.pages, b.q.float(), cu, ln, tab, 2, 62))
    refused(lambda: go(q=b.q.cpu()), ValueError)
    refused(lambda: go(tab=tab.long()), ValueError)
    refused(lambda: go(slopes=torch.ones(3, device="cuda")), ValueError)
    assert (out == 7).all()
    x = torch.zeros((3, 2, 64), device="cuda")
    s = torch.zeros(3, dtype=torch.int64, device="cuda")
    refused(lambda: ctx.page_write(b.pages, x, x.half(), s))
    refused(lambda: ctx.page_write(b.pages, x[:, :1], x[:, :1], s), ValueError)
    refused(lambda: ctx.page_write(b.pages, x, x, s[:2]), ValueError)
    refused(lambda: ctx.page_write(b.pages, x.flatten()[1:1 + 2 * 128].view(2, 2, 64), x[:2], s))    # 4-byte aligned
    k = torch.zeros((1, 2, 2, 60, 64), dtype=torch.float16, device="cuda")
    refused(lambda: ctx.page_read(b.pages, ln, tab, 0, 61, 0, k, None))
    refused(lambda: ctx.page_read(b.pages, ln, tab, 5, 4, 0, k, None))
    refused(lambda: ctx.page_read(b.pages, ln, tab, 0, 60, 0, k, k.float()))
    refused(lambda: ctx.page_read(b.pages, ln, tab, 0, 60, 1, k, None), ValueError)
    refused(lambda: _plan(ctx, [1], [0], [[0, 0]], [1], 0, 24, 4))              # pages of 24
    refused(lambda: ctx.page_attend(fkv.Pages.empty(4, 2, 24, 64), b.q, cu, ln, tab, 2, 62))
    refused(lambda: ctx.page_attend(fkv.Pages.empty(4, 2, 16, 96), b.q, cu, ln, tab, 2, 62), ValueError)
    assert ctx.sync_status() == 0


def test_write_slots_are_32_bits(fkv, ctx):
    """A pool of more than 2^32 slots is refused; in one of 2^32, slots from there on (their low 32 bits name
    a slot of the pool) are skipped and reported."""
    one = torch.zeros((1, 1, 1024, 64), dtype=torch.int8, device="cuda")
    scale = torch.ones((1, 1), device="cuda")
    x = torch.ones((2, 1, 64), dtype=torch.bfloat16, device="cuda")
    pool = lambda n: fkv.Pages(*[one.expand(n, -1, -1, -1)] * 2, *[scale.expand(n, -1)] * 2)
    with pytest.raises(fkv.FkvError) as e:
        ctx.page_write(pool((1 << 22) + 1), x, x, torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert e.value.code == -1 and ctx.sync_status() == 0
    ctx.page_write(pool(1 << 22), x, x, torch.tensor([1 << 32, (1 << 40) + 5], device="cuda"))
    assert ctx.sync_status() == -2
    assert not one.any() and (scale == 1).all()


def test_a_refused_pool_leaves_the_next_call_its_workspace(fkv):
    """A pool of pages of 24 is refused; a call of the same sizes on a good pool gets the workspace that it needs."""
    ctx = fkv.Context(256)
    b = Batch(fkv, 44, [(20000, 1)], 1, 4, 64, 16, "int8", "f16")
    with pytest.raises(fkv.FkvError) as e:
        ctx.page_attend(fkv.Pages.empty(900, 1, 24, 64, torch.int8), b.q, _i32(b.cu), _i32(b.len), _i32(b.table), 1, 20001)
    assert e.value.code == -1
    b.check(ctx)


def test_workspace_is_on_the_device(fkv, ctx):
    """A workspace on the host, or one with gaps, is refused before its pointer goes anywhere."""
    b = Batch(fkv, 30, [(600, 1)], 1, 4, 64, 16, "int8", "f16")
    cu, ln, tab = _i32(b.cu), _i32(b.len), _i32(b.table)
    size = 1 << 24
    for ws in (torch.empty(size, dtype=torch.uint8), torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            ctx.page_attend(b.pages, b.q, cu, ln, tab, 1, 601, workspace=ws)
    assert ctx.sync_status() == 0


def test_memory_of_another_stream(fkv, ctx):
    """What a call on another stream allocates is that stream's: memory freed in the current one's order may
    still be read there when the call writes it."""
    b = Batch(fkv, 31, [(600, 1)], 1, 4, 64, 16, "int8", "f16")
    cu, ln, tab = _i32(b.cu), _i32(b.len), _i32(b.table)
    want = ctx.page_attend(b.pages, b.q, cu, ln, tab, 1, 601)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = ctx.page_attend(b.pages, b.q, cu, ln, tab, 1, 601, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    p = out.data_ptr()
    seg = [s for s in torch.cuda.memory_snapshot() if s["address"] <= p < s["address"] + s["total_size"]]
    assert len(seg) == 1 and seg[0]["stream"] == side.cuda_stream


def test_scale_within_float32(fkv, ctx):
    """A scale whose multiplier is no float32 number would turn scores of zero into NaN: refused."""
    b = Batch(fkv, 32, [(40, 1)], 1, 2, 64, 16, "e4m3", "bf16")
    for opt in (dict(scale=3e38), dict(scale=-3e38), dict(softcap=1e-39), dict(scale=1e3, softcap=1e-36)):
        with pytest.raises(fkv.FkvError) as e:
            b.run(ctx, **opt)
        assert e.value.code == -1
    b.q.zero_()
    out, lse = b.run(ctx, softcap=1e-30)[:2]
    assert torch.isfinite(out).all() and torch.isfinite(torch.as_tensor(lse)).all()


@pytest.mark.parametrize("scale", [0.0, 1e-38])
def test_masks_of_vanishing_scores(fkv, ctx, scale):
    """Scores that are zero, or too small for float32, still have their masks."""
    for D, dtype in ((64, "f16"), (128, "bf16")):
        b = Batch(fkv, 34, [(130, 300), (5, 40), (0, 3), (400, 1)], 1, 2, D, 16, "int8", dtype)
        b.check(ctx, scale=scale)
        b.check(ctx, scale=scale, window=37, sinks=3, prefix=[20, 0, 3, 7])


@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("D,fmt,dtype", [(64, "int8", "f16"), (128, "e4m3", "bf16")])
def test_bias_at_every_end(fkv, ctx, D, fmt, dtype, new):
    """Biased scores, walked from the last tile back: ends in each of a tile's quarters, shares of long ones."""
    b = Batch(fkv, 35, [(x, new) for x in (0, 31, 32, 63, 64, 95, 96, 127, 128, 160, 300, 2100)], 1, 4, D, 16, fmt, dtype)
    rows = [0, new // 2, new - 1]
    slopes = [0.5, 0.25, 0.03, -0.02]
    b.check(ctx, rows=rows, slopes=slopes)
    b.check(ctx, rows=rows, slopes=slopes, window=100, sinks=40, prefix=[0, 10, 40, 0, 70, 1, 0, 128, 0, 5, 200, 600])
    long = Batch(fkv, 36, [(20000, new)], 1, 4, D, 32, fmt, dtype)
    long.check(ctx, rows=rows, slopes=slopes)


@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("D,fmt,dtype", [(64, "int8", "f16"), (128, "e4m3", "bf16")])
def test_window_far_from_sinks_and_prefix(fkv, ctx, D, fmt, dtype, new):
    """A window's keys and the first ones are both looked at, however many the latter are."""
    b = Batch(fkv, 37, [(x, new) for x in (300, 2100, 5000)], 1, 4, D, 16, fmt, dtype)
    rows = [0, new // 2, new - 1]
    for opt in (dict(sinks=1500), dict(sinks=1 << 40), dict(prefix=[5, 600, 4100]), dict(sinks=700, prefix=[0, 1000, 300])):
        b.check(ctx, rows=rows, window=100, **opt)
    b.check(ctx, rows=rows, window=1, sinks=129)


# --------------------------------------------------------------- together --
def test_serving_loop_and_archive(fkv, oracle_mod):
    """Prompts, steps and a request that ends, all captured once and replayed; then the positions that leave
    the pages go through the residual VQ, as a cache's do."""
    rng = np.random.default_rng(18)
    H, G, D, block, n = 2, 2, 64, 16, 4
    cb = rng.standard_normal((1, H, 1, 256, D)).astype(np.float32)
    ctx = fkv.Context(256, codebooks=(cb, cb))
    nb, width, rows = 24, 8, 12
    pages = fkv.Pages.empty(nb, H, block, D, torch.float8_e4m3fn)
    codes = [t.view(torch.uint8).cpu().numpy() for t in (pages.k, pages.v)]
    scale = [t.cpu().numpy() for t in (pages.k_scale, pages.v_scale)]
    table, free, taken = np.full((n, width), -1), np.arange(nb), 0
    ln = np.zeros(n, np.int64)
    d = dict(new=_i32(np.zeros(n)), ln=_i32(ln), table=_i32(table), free=_i32(free), taken=_i32([0]), cu=_i32(np.zeros(n + 1)),
             slots=torch.zeros(rows, dtype=torch.int64, device="cuda"), pos=_i32(np.zeros(rows)))
    x = torch.zeros((rows, 2 * H + H * G, D), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((rows, H * G, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((rows, H * G), device="cuda")

    def step():
        ctx.page_plan(d["new"], d["ln"], d["table"], d["free"], d["taken"], block, d["cu"], d["slots"], d["pos"])
        ctx.page_write(pages, x[:, :H], x[:, H:2 * H], d["slots"])
        ctx.page_attend(pages, x[:, 2 * H:], d["cu"], d["ln"], d["table"], 9, width * block, out=out, lse=lse)

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
        out.fill_(7)
        graph.replay()
        assert ctx.sync_status() == 0
        before = np.where(np.asarray(new) < 0, 0, ln)
        cu, slots, _, ln, taken, table, free, ok = paged.plan(new, ln, table, free, taken, block, rows)
        assert ok and np.array_equal(d["slots"].cpu().numpy(), slots) and d["taken"].item() == taken
        h = x.double().cpu().numpy()
        for c, s, y in zip(codes, scale, (h[:, :H], h[:, H:2 * H])):
            paged.write(c, s, y, slots, "e4m3")
        o = out.double().cpu().numpy()
        for r in range(n):
            m = max(new[r], 0)
            if not m:
                continue
            k, v = (paged.gather(c, s, table[r], int(ln[r]), "e4m3") for c, s in zip(codes, scale))
            want, wl, mass, size = paged.attend(h[cu[r]:cu[r] + m, 2 * H:], k, v, D ** -0.5, paged.visible(m, int(ln[r])),
                                                p0=int(before[r]))
            bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -20 * (size + np.abs(wl) + 16) + 1e-6)[..., None] * mass
            assert (np.abs(o[cu[r]:cu[r] + m] - want) <= bound * (1 + 2.0 ** -8)).all()
        assert (o[cu[n]:] == 7).all()
    # the oldest positions of every request leave for the archive
    t1 = int(ln.min())
    K, V = (torch.zeros((1, n, H, 16, D), dtype=torch.float32, device="cuda") for _ in range(2))
    ctx.page_read(pages, d["ln"], d["table"], 0, t1, 0, K, V)
    R = ctx.record_len()
    sym = torch.zeros((n, t1 * R), dtype=torch.uint8, device="cuda")
    ctx.rvq_encode(0, K, 0, t1, sym)
    ctx.rvq_encode(1, V, 0, t1, sym)
    assert ctx.sync_status() == 0
    s = sym.cpu().numpy()
    for r in range(n):
        idx = oracle_mod.indices_from_records(s[r], H, 1, 1)
        for kv in (0, 1):
            val = paged.gather(codes[kv], scale[kv], table[r], t1, "e4m3")
            for hh in range(H):
                oi, gap = oracle_mod.rvq_encode(val[hh], cb[0, hh])
                from oracle import parity
                assert parity.compare_rvq(idx[kv][hh], oi, gap)[0] == 0


def test_overlapping_calls_on_two_streams(fkv, ctx):
    """Two calls at once, each with its own workspace, give what each gives alone."""
    b1 = Batch(fkv, 19, [(9000, 1)], 1, 4, 128, 64, "e4m3", "bf16")
    b2 = Batch(fkv, 20, [(7000, 3)], 1, 4, 128, 64, "e4m3", "bf16")
    w1, w2 = b1.run(ctx)[0], b2.run(ctx)[0]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s1):
            o1 = b1.run(ctx)[0]
        with torch.cuda.stream(s2):
            o2 = b2.run(ctx)[0]
        torch.cuda.synchronize()
        assert torch.equal(o1, w1) and torch.equal(o2, w2)
