"""Rotary positions on the GPU at the edges of their sizes: tables of 2^30 positions,
threads that serve several heads, gradients through autograd."""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from oracle.rope_prior import yarn_theta
from tests.gpu_cases import note
from tests.kv4_cases import DEV, TORCH, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def test_table_of_more_than_2_30_positions(G):
    """8.6 GB of one pair: the first and last positions and some between."""
    n = 2 ** 30 + 3
    note("table of 2^30 + 3 positions")
    t = G.gvr_rope_table(n, dict(d_rope=2), device=DEV)
    pos = np.unique(np.concatenate([[0, 1, 63, 64, 255, 256, 2 ** 29, 2 ** 30, n - 2, n - 1],
                                    np.random.default_rng(0).integers(0, n, 1000)]))
    got = f64(t[torch.from_numpy(pos).to(DEV)])[:, 0]
    phase = pos * yarn_theta(d=2)[0]
    ref = np.stack([np.cos(phase), np.sin(phase)], axis=-1)
    # float64's own unit of the phase (2^30 * 2^-52), and one rounding to float32
    assert np.abs(got - ref).max() <= 2.0 ** -24 + 2.0 ** -21
