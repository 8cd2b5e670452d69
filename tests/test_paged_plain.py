"""The plain forms that the GPU tests of the paged cache compare with, held to what they must give by their definitions."""
import numpy as np
import torch

import paged_plain as pp


def test_quantised_rows():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * np.exp(3 * rng.standard_normal((50, 1)))
    y, e = pp.quantise(x)
    top = np.abs(x).max(-1)
    assert (top <= 448.0 * 2.0 ** e).all() and (top > 448.0 * 2.0 ** (e - 1)).all()
    assert (np.abs(y - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** (e[:, None] - 10.0))).all()      # half a step
    again, e2 = pp.quantise(y)
    assert np.array_equal(again, y) and (e2 <= e).all()
    y, e = pp.quantise(np.array([[0.0] * 8, [448.0] * 8, [448.1] * 8, [np.inf] + [1.0] * 7, [np.nan] + [3.0] * 7]))
    assert list(e[:3]) == [-100, 0, 1] and (y[0] == 0).all() and (y[1] == 448).all()
    assert y[3, 0] == 448.0 * 2.0 ** e[3] and np.isnan(y[4]).all()
    # the e4m3 numbers themselves, against torch's conversion
    z = torch.linspace(-448, 448, 20001, dtype=torch.float64)
    z[0] = -448
    one = torch.cat([z, torch.tensor([448.0])])
    assert np.array_equal(pp.quantise(one.numpy()[None])[0][0], one.float().to(torch.float8_e4m3fn).double().numpy())


def test_verify_by_hand():
    p = np.array([[0.5, 0.5, 0.0], [0.2, 0.3, 0.5], [0.0, 0.0, 1.0]])
    q = np.array([[0.5, 0.25, 0.25], [0.2, 0.8, 0.0]])
    assert pp.verify(p, q, [0, 1], [0.9, 0.9, 0.5], 2) == (1, [0, 2, -1])        # 0.9 * 0.8 >= 0.3: what is left is entry 2
    assert pp.verify(p, q, [0, 1], [0.9, 0.3, 0.5], 2) == (2, [0, 1, 2])
    assert pp.verify(p, q, [2, 1], [0.0, 0.0, 0.0], 2) == (0, [1, -1, -1])       # 0 < 0 fails: entry 1 is left
    assert pp.verify(p, None, [0, 1], [0.4, 0.9, 0.2], 2) == (1, [0, 0, -1])        # 0.2 * 0.7 lies in entry 0's 0.2
    assert pp.verify(p, None, [0, 1], [0.4, 0.9, 0.3], 0) == (0, [0, -1, -1])
