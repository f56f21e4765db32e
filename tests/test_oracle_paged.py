"""Pins of the paged cache's oracle, and what the binding refuses before any
call: codes, scales, plans and masks that can be checked by hand (CPU)."""
import numpy as np
import pytest
import torch

from oracle import paged


def test_e4m3_table_is_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(paged.E4M3_VALUES))
    f = ~np.isnan(t)
    assert np.array_equal(t[f], paged.E4M3_VALUES[f])


def test_e4m3_rounding_is_torchs():
    g = torch.Generator().manual_seed(3)
    x = torch.cat([torch.randn(4000, generator=g) * 100, torch.randn(4000, generator=g) * 0.01,
                   torch.tensor([0.0, 448.0, 464.0, 1e9, -1e9, 2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875])])
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(paged.to_codes(x.double().numpy(), paged.E4M3), want)


@pytest.mark.parametrize("amax,want", [(448.0, 1.0), (449.0, 2.0), (447.0, 1.0), (896.0, 2.0), (897.0, 4.0),
                                       (1.75 * 2 ** -60, 2.0 ** -68), (0.0, 2.0 ** -100), (2.0 ** -140, 2.0 ** -100)])
def test_e4m3_scales(amax, want):
    assert paged.scale_of(amax, paged.E4M3) == want


def test_int8_scales():
    assert paged.scale_of(254.0, paged.INT8) == 2.0
    assert paged.scale_of(1.0, paged.INT8) == np.float32(1) / np.float32(127)


def test_scales_stay_within_the_pools_range():
    for fmt in (paged.E4M3, paged.INT8):
        assert paged.scale_of(2.0 ** 120, fmt) == 2.0 ** 100 and paged.scale_of(2.0 ** -120, fmt) == 2.0 ** -100


def test_a_grown_scale_rounds_earlier_rows_again():
    codes, scale = np.zeros((1, 1, 16, 1), np.uint8), np.zeros((1, 1), np.float32)
    paged.write(codes, scale, np.array([[[100.0]]]), np.array([3]), paged.INT8)   # rows 0..2 count as earlier ones
    assert scale[0, 0] == np.float32(100.0) / np.float32(127) and codes[0, 0, 3, 0] == 127
    paged.write(codes, scale, np.array([[[200.0]]]), np.array([4]), paged.INT8)
    assert scale[0, 0] == np.float32(200.0) / np.float32(127)
    assert codes[0, 0, 3, 0] in (63, 64) and codes[0, 0, 4, 0] == 127
    paged.write(codes, scale, np.array([[[1.0]]]), np.array([5]), paged.INT8)     # smaller: the scale stays
    assert scale[0, 0] == np.float32(200.0) / np.float32(127) and codes[0, 0, 5, 0] == 1


def test_plan_by_hand():
    table = np.array([[7, 8, -1, -1], [3, -1, -1, -1], [4, 5, 6, -1]])
    free = np.array([0, 0, 0, 0, 0, 0, 20, 21, 22, 23])
    cu, slots, pos, ln, taken, tab, fr, ok = paged.plan([2, -1, 17], [31, 16, 40], table, free, 6, 16, 22)
    # request 1 gives page 3 back; request 0 takes it, request 2 takes page 20
    assert ok and cu.tolist() == [0, 2, 2, 19] and taken == 7
    assert tab[0].tolist() == [7, 8, 3, -1] and tab[2].tolist() == [4, 5, 6, 20]
    assert slots[:2].tolist() == [8 * 16 + 15, 3 * 16] and pos[:2].tolist() == [31, 32]
    assert slots[2:10].tolist() == [6 * 16 + 8 + i for i in range(8)] and slots[10] == 20 * 16
    assert slots[19:].tolist() == [-1] * 3 and ln.tolist() == [33, 0, 57]


@pytest.mark.parametrize("why", ["free", "rows", "width", "taken", "negative"])
def test_plan_is_all_or_nothing(why):
    new, ln, free, taken, rows = [5, 30], [3, 14], np.arange(6), 2, 40
    table = np.array([[0, -1, -1], [1, -1, -1]])
    if why == "free":
        free = free[:3]
    if why == "rows":
        rows = 34
    if why == "width":
        table = table[:, :2]
    if why == "taken":
        new, taken = [-1, 1], 0
    if why == "negative":
        ln = [-3, 14]
    cu, slots, pos, after, tk, tab, fr, ok = paged.plan(new, ln, table, free, taken, 16, rows)
    assert not ok and not cu.any() and (slots == -1).all() and after.tolist() == ln and tk == taken
    assert np.array_equal(tab, table)


def test_masks_by_hand():
    m = paged.visible(3, 5)
    assert m.astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 1, 1]]
    m = paged.visible(2, 6, window=2, sinks=1)
    assert m.astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    m = paged.visible(2, 6, window=1, prefix=2)
    assert m.astype(int).tolist() == [[1, 1, 0, 0, 1, 0], [1, 1, 0, 0, 0, 1]]
    m = paged.visible(2, 4, causal=False, window=2)
    assert m.astype(int).tolist() == [[0, 1, 1, 1], [0, 0, 1, 1]]
    assert not paged.visible(4, 2)[:2].any() and paged.visible(4, 2)[3].all()      # two tokens lie before position 0


def test_attention_by_hand():
    k = np.array([[[1.0], [0.0]]])
    v = np.array([[[4.0], [8.0]]])
    q = np.array([[[np.log(3.0)]]])
    out, lse, mass, size = paged.attend(q, k, v, 1.0, np.ones((1, 2), bool))
    assert np.isclose(out[0, 0, 0], 0.75 * 4 + 0.25 * 8) and np.isclose(lse[0, 0], np.log(4.0))
    out, lse, _, _ = paged.attend(q, k, v, 1.0, np.zeros((1, 2), bool))
    assert out[0, 0, 0] == 0 and lse[0, 0] == -np.inf


def test_pages_refuse_host_tensors_and_other_shapes():
    import paper_2607_07144_gb300 as fkv
    k, s = torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.ones((2, 1))
    with pytest.raises(ValueError):
        fkv.Pages(k, k, s, s)
    with pytest.raises(ValueError):
        fkv.Pages(k.float(), k.float(), s, s)
    with pytest.raises(ValueError):
        fkv.Pages(k, k[:, :, :8], s, s)
