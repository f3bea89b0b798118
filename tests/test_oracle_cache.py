"""The cache oracle against what it does not share code with: torch's e4m3 type, closed forms, hand-worked rows."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O


def test_the_grid_is_the_type():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    every = every[every.isfinite()]
    assert sorted(set(every.abs().tolist())) == O.GRID.tolist()


def test_rounding_is_the_types_own_and_ties_go_to_even():
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(4000, generator=g) * s for s in (1e-3, 0.1, 3, 100)]).clamp(-448, 448)
    mid = torch.tensor((O.GRID[1:] + O.GRID[:-1]) / 2).float()      # exact in fp32
    x = torch.cat([x, mid, -mid, torch.tensor([0.0, 448.0, -448.0])])
    want = x.to(torch.float8_e4m3fn).double()
    assert [O.to_code(v) for v in x.double().tolist()] == want.tolist()


@pytest.mark.parametrize("row,codes,scale", [
    ([448.0, 1.0], [448.0, 1.0], 127),
    ([450.0, 1.0], [224.0, 0.5], 128),               # bf16 450 is over 448: the next power of two, 225 rounds to 224
    ([1.75, -0.5], [448.0, -128.0], 119),
    ([1.76, -0.5], [224.0, -64.0], 120),             # (1.76 stands for any value just over 1.75: 225.28 -> 224)
    ([0.0, 0.0], [0.0, 0.0], 7),
    ([2.0 ** -130, 0.0], [2.0 ** -9 * 0.5, 0.0], 7), # 2^-130 / 2^-120 = 2^-10: half of the smallest code, a tie with 0
    ([float("inf"), 1.0], [0.0, 0.0], 255),
    ([float("nan"), 1.0], [0.0, 0.0], 255),
])
def test_rows_by_hand(row, codes, scale):
    got, s = O.quantise_row(row)
    if row[0] == 2.0 ** -130:
        codes = [0.0, 0.0]                           # ties go to the even place: 0
    assert s == scale and got.tolist() == codes


def test_the_scale_loses_nothing_but_the_codes_rounding():
    rng = np.random.default_rng(0)
    for size in (1e-20, 1e-3, 1.0, 300.0, 1e30):
        x = torch.tensor(rng.standard_normal(128) * size).bfloat16().double().numpy()
        codes, s = O.quantise_row(x)
        y = O.row_values(codes, s)
        assert (np.abs(y - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * 2.0 ** (s - 127))).all()
        assert (torch.tensor(y).bfloat16().double().numpy() == y).all()        # what is held is a bf16 number
        again, t = O.quantise_row(y)
        assert (O.row_values(again, t) == y).all()                             # and is written again as it is


def test_visible_positions():
    assert O.visible(3, 0, 0) == [0, 1, 2, 3]
    assert O.visible(9, 3, 0) == [7, 8, 9]
    assert O.visible(9, 3, 2) == [0, 1, 7, 8, 9]
    assert O.visible(2, 5, 4) == [0, 1, 2]
    assert O.visible(0, 1, 0) == [0]


def test_attention_closed_forms():
    rng = np.random.default_rng(3)
    v = rng.standard_normal((7, 4))
    out, lse = O.attend_row(np.zeros(4), rng.standard_normal((7, 4)), v, 0.5)   # equal scores: the mean
    assert np.allclose(out, v.mean(0), atol=1e-15) and math.isclose(lse, math.log(7))
    k = np.eye(4) * 200
    out, lse = O.attend_row(np.array([1.0, 0, 0, 0]), k, v[:4], 1.0)            # one score far above the others: its value
    assert np.allclose(out, v[0], atol=1e-15) and math.isclose(lse, 200.0)
    q, k = rng.standard_normal(4), rng.standard_normal((7, 4))
    p = torch.softmax(torch.tensor(0.3 * k @ q), 0).numpy()
    out, lse = O.attend_row(q, k, v, 0.3)
    assert np.allclose(out, p @ v, atol=1e-14) and math.isclose(lse, float(torch.logsumexp(torch.tensor(0.3 * k @ q), 0)))
    a, la = O.attend_row(q, k[:3], v[:3], 0.3)                                  # parts meet by their lse
    b, lb = O.attend_row(q, k[3:], v[3:], 0.3)
    assert np.allclose(a * math.exp(la - lse) + b * math.exp(lb - lse), out, atol=1e-14)
    assert O.attend_row(q, k[:0], v[:0], 0.3)[1] == -math.inf


def test_places_and_lengths_out_of_range():
    row = [3, -1, 9, 0]
    assert O.place(row, 5, 8, 4) == (3, 5) and O.place(row, 31, 8, 4) == (0, 7)
    assert O.place(row, 8, 8, 4) is None and O.place(row, 16, 8, 4) is None and O.place(row, 32, 8, 4) is None and O.place(row, -1, 8, 4) is None
    assert [O.held_length(L, row, 8) for L in (-1, 0, 32, 33)] == [-1, 0, 32, -1]
    assert [O.held_count([0, 5, 6, -1], b, 5) for b in range(4)] == [0, 5, 0, 0]
