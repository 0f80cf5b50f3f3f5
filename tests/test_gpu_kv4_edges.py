"""Attention over the 4-bit cache at the edges of its numbers: values that are
not finite, weights that underflow, counts of query tokens that name nothing."""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from tests.gpu_cases import note
from tests.kv4_cases import DEV, TORCH, UNIT, Sequences, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def held(k, v, page=16):
    """One sequence of k, v [n][heads][D] in consecutive pages: its cache, block table and lengths on the GPU, and what
    the records stand for."""
    n, heads, D = k.shape
    rec = O.record(k, v)
    pages = (n + page - 1) // page
    cache = np.zeros((pages * page, rec.shape[1]), np.uint8)
    cache[:n] = rec
    return (torch.from_numpy(cache.reshape(pages, page, -1)).to(DEV),
            torch.arange(pages, dtype=torch.int32, device=DEV).view(1, -1),
            torch.tensor([n], dtype=torch.int32, device=DEV), *O.values(rec, heads, D))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("nq", [1, 33])
def test_visible_nan_of_a_part_without_weight(G, dtype, D, nq):
    """A value that is NaN, in a token whose weight underflows (768 below the largest score), is visible all the same:
    its 32 dimensions are NaN, split or not, and the others are not touched."""
    rng = np.random.default_rng(61)
    n, group, block = 4000, 4, 1
    k = np.full((n, 1, D), -6.0)
    k[n - nq - 40:n - nq + 1] = 6.0            # every row's largest scores, 768 and more above the others
    v = rng.standard_normal((n, 1, D))
    v[5, 0, 32 * block] = np.nan
    cache, table, lens, kk, vv = held(k, v)
    q = torch.full((nq, group, D), 8.0, dtype=TORCH[dtype], device=DEV)
    scale = 8.0 / D                            # scores of +-384
    assert G.gvr_kv4_attention_workspace(q, cache, table, lens, 1) > 0
    nan = np.zeros(D, bool)
    nan[32 * block:32 * block + 32] = True
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("visible NaN without weight: %s D=%d nq=%d %s" % (dtype, D, nq, "split" if ws is None else "whole"))
        out = f64(G.gvr_kv4_attention(q, cache, table, lens, 1, scale=scale, workspace=ws))
        for i in range(nq):
            ref, _, mag = O.attention(f64(q)[i], kk[:n - nq + 1 + i], np.nan_to_num(vv[:n - nq + 1 + i]), scale)
            assert np.isnan(out[i][:, nan]).all(), "row %d lost the NaN" % i
            # the weights are 0 and 1: sums in float32 and one rounding
            tol = UNIT[dtype] * np.abs(ref) + 2 * (n + 64) * 2.0 ** -24 * mag + 2.0 ** -24
            assert (np.abs(out[i] - ref) <= tol)[:, ~nan].all()
