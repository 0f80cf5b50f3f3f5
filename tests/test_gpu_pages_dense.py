"""Page steps over page tables that hold more tokens than a request has rows in a dense cache."""
import numpy as np
import pytest
import torch

from oracle.pages import Pool
from tests.gpu_cases import note
from tests.kv4_cases import DEV
from tests.test_gpu_pages import G, check, ints  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [64, 4000])   # one workgroup, three kernels
@pytest.mark.parametrize("ld", [0, 1, 13, 40, 47, 48])
def test_steps(G, T, ld):  # noqa: F811
    rng = np.random.default_rng(ld + T)
    pool, ref = G.new_page_pool(60, 8, 9, 6), Pool(60, 8, 9, 6)
    for i in range(6):
        new = rng.integers(0, 12, 9)
        keep = rng.integers(0, 49, 9) if i % 2 else None
        note("pages dense T %d ld %d step %d" % (T, ld, i))
        got = G.gvr_page_step(pool, ints(new), T, keep=None if keep is None else ints(keep), ld=ld)
        check(pool, ref, got, ref.step(new, T, keep, ld), i)


def test_keys_of_other_requests_stay(G):  # noqa: F811
    """A request's keys past its rows of the indexer's cache go nowhere: not into the next request's first rows."""
    note("pages dense keys")
    ld, R, D = 10, 3, 128
    pool = G.new_page_pool(12, 16, R, 1)
    codes = torch.full((R * ld, D), 0x55, dtype=torch.uint8, device=DEV)
    scale = torch.full((R * ld, 1), 9.0, device=DEV)
    for new in ([2, 3, 4], [12, 0, 11]):
        step = G.gvr_page_step(pool, ints(new), 32, ld=ld)
        keys = torch.randn((32, D), device=DEV)
        G.gvr_fp8_quantize(keys, slots=step.dense, codes=codes, scale=scale)
        made = G.gvr_fp8_quantize(keys)
        at = step.dense.cpu().numpy()
        assert (at < R * ld).all() and len(set(at[at >= 0])) == (at >= 0).sum()
        for t in np.flatnonzero(at >= 0):
            assert torch.equal(codes[at[t]], made.codes[t]) and torch.equal(scale[at[t]], made.scale[t])
        if new[0] == 2:
            second = codes[ld:2 * ld].clone(), scale[ld:2 * ld].clone()
    assert torch.equal(codes[ld:2 * ld], second[0]) and torch.equal(scale[ld:2 * ld], second[1])
    assert (codes[ld + 3:2 * ld] == 0x55).all()
