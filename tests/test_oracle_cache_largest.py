"""The oracle at the end of bf16's range: what is held is finite, and the nearest finite value that the format has."""
import numpy as np
import torch

from oracle import cache_oracle as O


def test_every_bf16_number_is_held_as_the_nearest_finite_value():
    tops = torch.arange(0x7e00, 0x7f80, dtype=torch.int16).view(torch.bfloat16).double().numpy()
    for x in tops:
        codes, s = O.quantise_row([x, -x, 0.0])
        y = O.row_values(codes, s)
        assert torch.tensor(y).bfloat16().isfinite().all() and (torch.tensor(y).bfloat16().double().numpy() == y).all()
        can = O.GRID * 2.0 ** (s - 127)
        can = can[can < 2.0 ** 128]
        assert abs(y[0] - x) == np.abs(can - x).min() and y[1] == -y[0] and y[2] == 0
    assert O.quantise_row([248 * 2.0 ** 120, 2.0 ** 120])[0].tolist() == [240.0, 1.0]
    assert O.quantise_row([447 * 2.0 ** 119, 256 * 2.0 ** 119])[0].tolist() == [448.0, 256.0]     # the scale below holds 256
