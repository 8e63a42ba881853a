"""Sine and cosine of rotary positions in fp32, by themselves, at positions near whole half turns, against 64-bit functions of the angle as
the header defines it, positions * inv_freq in 64 bits (needs an MI355X).

Bar: 2 units in the last place of the result, as include/rotary.h states it.  The angle that is left of a turn, at most pi/4, is rounded to
fp32 once: half a unit of the sine, 0.56 of the cosine at most.  The series' last sum rounds once more, half a unit; what goes into it, a
third of the result at most, holds three roundings, another half; what is left out is below a tenth."""
import math

import numpy as np
import pytest
import torch

from paper_2601_12698_amd import serving as S

pytestmark = pytest.mark.gpu

# numerators of the fractions next to pi and to half of it, where a sine or a cosine nearly vanishes; their neighbours; borders of 24, 32 and 53 bits
POSITIONS = [0, 1, -1, 2, 3, 11, 22, 333, 355, 710, 103993, 104348, 208341, 312689, 833719, 1146408, 4272943, 5419351, 10838702, 80143857, 165707065,
             -355, -833719, -5419351, 103994, 833720, 1 << 24, (1 << 24) + 1, (1 << 31) + 7, -(1 << 31), 245850922, 411557987, (1 << 40) + 3, (1 << 52) + 1]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("freq", [1.0, 0.5, 10000.0 ** -0.25, 10000.0 ** -0.875, 1.0 / 3.0])
def test_sine_and_cosine(freq, inverse):
    T = len(POSITIONS)
    x = torch.zeros(T, 1, 2, device="cuda")
    x[:, :, 0] = 1.0                                          # (1, 0) turns to (cos, sin)
    out = torch.empty_like(x)
    pos = torch.tensor([POSITIONS], device="cuda")
    S.rotary_run(x, None, out, None, pos, torch.tensor([freq], dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.uint8, device="cuda"), "fp32",
                 inverse=inverse)
    got = out.cpu().numpy()[:, 0].astype(np.float64)
    for t, p in enumerate(POSITIONS):
        a = float(p) * freq
        for what, want, have in (("cos", math.cos(a), got[t, 0]), ("sin", -math.sin(a) if inverse else math.sin(a), got[t, 1])):
            step = max(float(np.spacing(np.float32(abs(want)))), 2.0 ** -149)
            assert abs(have - want) <= 2.0 * step, (what, p, want, have, abs(have - want) / step)
