"""Codes of binary32 rows whose products h * weight have up to 48 bits, at and beside halves: equal to the exact quotient's, halves
to even."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import lm
from test_gpu_rms_norm import run_fwd

pytestmark = pytest.mark.gpu

# h and weight of an element, and of the row's largest product: 127 h w / (h0 w0) is a half, or some 2^-49 beside one
PAIRS = [(14722983, 10609670, 15244078, 15774162), (11762013, 6084835, 11184001, 14643470), (9758205, 9043769, 9043769, 12090654),
         (8730811, 8415875, 12752870, 16443325), (11791153, 16455546, 14329918, 16455546), (15882965, 9343586, 10936732, 15882965),
         (15665903, 6124057, 12248114, 15665903), (16189123, 6192360, 15414911, 16355011), (8814549, 8409227, 11380923, 7915277),
         (11982432, 5299729, 12832133, 15518455), (11355491, 8778288, 15106771, 16271987), (11423468, 11820811, 12737154, 13669113)]


def exact_code(h, w, h0, w0):
    return round(Fraction(127 * h * w, h0 * w0))          # (a Fraction rounds halves to even)


@pytest.mark.parametrize("dim", [64, 1000, 9001, 20000])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -60, 2.0 ** 60])
def test_pairs_at_and_beside_halves(dim, scale):
    """Each pair, with both signs, in a row of its own beside small elements; scale: of all of h."""
    for i, (h, w, h0, w0) in enumerate(PAIRS):
        x, weight = np.ones((4, dim)), np.ones(dim)
        weight[[3, dim - 2]] = w, w0
        x[:, 3], x[:, dim - 2] = [h, -h, h, -h], [h0, h0, -h0, -h0]
        x, weight = torch.from_numpy(x * scale).float().cuda(), torch.from_numpy(weight).float().cuda()
        codes = run_fwd(x, None, weight, ("codes", "scales"))["codes"].cpu().numpy()
        want = exact_code(h, w, h0, w0)
        assert codes[:, 3].tolist() == [want, -want, want, -want], i
        assert codes[:, dim - 2].tolist() == [127, 127, -127, -127]


@pytest.mark.parametrize("dim", [127, 4096, 8192, 16400])
def test_rows_of_halves(dim):
    """Rows of h = (2n + 1) a under one weight of 24 bits, the largest 254 a: every quotient n + 1/2 exactly."""
    rs = np.random.RandomState(dim)
    a, n = rs.randint(1 << 15, 66000, (9, 1)), rs.randint(0, 127, (9, dim))
    n[:, 5] = 126
    h = (2 * n + 1) * a * rs.choice([-1, 1], (9, dim))
    h[:, 7] = 254 * a[:, 0]
    weight = np.full(dim, 15767325.0)
    for w in (15767325, 8875831, 12582911):
        weight[:] = w
        out = run_fwd(torch.from_numpy(h).float().cuda(), None, torch.from_numpy(weight).float().cuda(), ("codes", "scales"))
        want = np.where(n % 2 == 0, n, n + 1) * np.sign(h)
        want[:, 7] = 127
        assert np.array_equal(out["codes"].cpu().numpy()[:, :dim], want)
        r = lm.rms_norm(h, weight, 1e-5)[1]
        assert np.array_equal(lm.code_rows(h, weight, r)[0], want)

