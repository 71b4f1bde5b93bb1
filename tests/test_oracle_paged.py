"""CPU tests of the paged cache's oracle: against worked values, PyTorch's own 8-bit type and the dense attention oracle."""
import numpy as np
import torch

from oracle import attention as oat
from oracle import numeric as onum
from oracle import paged as op
import synthetic_inputs as si


def test_up12():
    assert op.up12(1.0) == 1.0 and op.up12(1.0 + 2.0 ** -11) == 1.0 + 2.0 ** -11 and op.up12(1.0 + 2.0 ** -20) == 1.0 + 2.0 ** -11
    assert op.up12(4095.5) == 4096.0


def test_e4m3_values_are_pytorchs():
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(op.E4M3, want)


def test_worked_rows():
    # the largest value 448 makes the scale 1: the codes are the values' own roundings, ties to even
    x = np.array([[448.0, -17.0, 18.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -0.0625]])
    code, s = op.quantise(x, "e4m3")
    assert s[0] == 1.0 and code[0].tolist() == [448.0, -16.0, 18.0, 20.0, 0.0, 2 * 2.0 ** -9, 0.0, -0.0625]
    code, s = op.quantise(np.array([[127.0, 0.5, 1.5, -2.5, 126.4]]), "i8")
    assert s[0] == 1.0 and code[0].tolist() == [127.0, 0.0, 2.0, -2.0, 126.0]
    code, s = op.quantise(np.array([[0.0, 0.0], [np.inf, 1.0], [np.nan, 2.0]]), "i8")
    assert s[0] == 2.0 ** -100 and np.isnan(s[1:]).all() and (code == 0).all()


def test_rounding_is_pytorchs():
    x = np.random.default_rng(1).standard_normal((200, 64))
    code, s = op.quantise(x, "e4m3")
    y = torch.from_numpy(x / s[:, None]).float().to(torch.float8_e4m3fn).double().numpy()
    assert (code != y).mean() < 1e-4                                             # (PyTorch rounds twice)
    assert np.abs(code).max() == 448.0 and np.abs(code * s[:, None] - x).max() <= 16.0 * s.max()


def test_attend_is_attention():
    dt, n = "f16", 37
    q, k, v = (si.normal_bits((1, 2, n, 16), dt, i, 1.0) for i in range(3))
    want = oat.sdpa(q, k, v, dt)[0].transpose(1, 0, 2)
    dq, dk, dv = (onum.decode(x, dt)[0].transpose(1, 0, 2) for x in (q, k, v))
    table = np.array([[3, 0, 2, 1, 4]])
    pool = np.zeros((2, 5, 8, 2, 16))
    for i, x in enumerate((dk, dv)):
        for j in range(n):
            pool[i, table[0, j // 8], j % 8] = x[j]
    got = op.attend(dq, pool[0], pool[1], table, [0, n], [n], causal=False)[0]
    assert np.abs(got - want).max() < 1e-12
    # causal: the last token alone sees the same keys; the first sees itself
    got = op.attend(dq, pool[0], pool[1], table, [0, n], [n])[0]
    assert np.abs(got[-1] - want[-1]).max() < 1e-12 and np.abs(got[0] - dv[0]).max() < 1e-12
    # a window of one position: every token its own value
    assert np.abs(op.attend(dq, pool[0], pool[1], table, [0, n], [n], window=1)[0] - dv).max() < 1e-12
