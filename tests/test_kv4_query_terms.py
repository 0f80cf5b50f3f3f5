"""What the attention's queries keep as sums of 8-bit numbers (CPU): a replay of the
split in E4M3, every mantissa at every exponent below a block's largest magnitude,
against the limits that gvr_kv4.h states."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def kept(x, terms):
    """x as the sum of `terms` E4M3 numbers 2^-4 apart (the block's largest magnitude scaled into [2^7, 2^8))."""
    total, rest, unit = torch.zeros_like(x), x.clone(), 1.0
    for _ in range(terms):
        t = rest.float().to(torch.float8_e4m3fn).double()
        total += t * unit
        rest, unit = 16.0 * (rest - t), unit / 16.0
    return total


@pytest.mark.parametrize("bits,terms,exact,off", [(8, 2, 13, 21), (11, 3, 14, 25)])
def test_limits(bits, terms, exact, off):
    mantissas = 1.0 + torch.arange(2 ** (bits - 1), dtype=torch.float64) / 2 ** (bits - 1)
    for below in range(40):                      # a block whose largest magnitude is 2^7; 256 at most is the same at 2^8
        x = mantissas * 2.0 ** (7 - below)
        err = (kept(x, terms) - x).abs().max().item()
        assert err <= 2.0 ** (7 - off)
        if below <= exact:
            assert err == 0.0
        elif below == exact + 1:
            assert err > 0.0                     # the limit is no larger than it has to be
    stated = open(os.path.join(ROOT, "include", "gvr_kv4.h")).read()
    assert "exact down to 2^-13 (2^-14)" in stated and "off by at most 2^-21 (2^-25)" in stated
