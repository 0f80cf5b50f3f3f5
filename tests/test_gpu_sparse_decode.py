"""The example's path end to end against the oracle: prompt into the 4-bit
cache, then decode steps whose queries attend to the tokens that the indexer
and the Top-K selected."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from oracle import kv4 as O
from tests.gpu_cases import note
from tests.kv4_cases import DEV, Sequences, check_attention, f64

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    oracle.build(force=False)


def held(layer, ctx):
    """The layer's sequences as the tests' comparison takes them."""
    s = Sequences.__new__(Sequences)
    s.table, s.cache = layer.blocks.cpu().numpy(), layer.cache.cpu().numpy()
    s.ctx, s.page, s.heads, s.D = list(ctx), layer.page, layer.kv_heads, layer.D
    return s


@pytest.mark.parametrize("drafts", [1, 2])
def test_prompt_then_steps(drafts):
    from sparse_decode import SparseLayer, fp8
    torch.manual_seed(drafts)
    R, n, K = 3, 90, 32
    layer = SparseLayer(R, 128, q_heads=8, kv_heads=2, head_dim=64, K=K, page=16, drafts=drafts)
    rope = O.rope_table(128, 64)

    def heads(m, h):
        return torch.randn((R * m, h, 64), device=DEV).bfloat16()

    q, k, v = heads(n, 8), heads(n, 2), heads(n, 2)
    out = layer.prompt(q, k, v, fp8((R * n, 128), DEV))
    pos = np.tile(np.arange(n), R)
    # the kernels' rotation, in float32 and rounded to the queries' type
    table = layer.table.cpu().numpy()
    assert np.abs(table - rope).max() <= 2.0 ** -24 + 1e-11
    turned = torch.from_numpy(O.rotate(q.float().cpu().numpy(), pos, table)).bfloat16()
    # the cache holds the rotated keys and the values as the oracle quantises them
    seqs = held(layer, [n] * R)
    for b in range(R):
        rec = O.record(O.rotate(k[b * n:(b + 1) * n].float().cpu().numpy(), np.arange(n), table),
                       v[b * n:(b + 1) * n].float().cpu().numpy())
        assert np.array_equal(seqs.cache.reshape(-1, rec.shape[1])[seqs.slots(b, np.arange(n))], rec)
    note("example: prompt, %d drafts" % drafts)
    check_attention(out, None, turned, seqs, [n * b for b in range(R + 1)], 64 ** -0.5, what="prompt")
    ctx = n
    for step in range(3):
        q, k, v = heads(drafts, 8), heads(drafts, 2), heads(drafts, 2)
        out = layer.decode(q, k, v, fp8((R * drafts, 64, 128), DEV), fp8((R * drafts, 128), DEV))
        pos = np.tile(np.arange(ctx, ctx + drafts), R)
        ctx += drafts
        turned = torch.from_numpy(O.rotate(q.float().cpu().numpy(), pos, table)).bfloat16()
        sel = layer.selected.cpu().numpy()
        for r in range(R * drafts):
            t = sel[r][sel[r] >= 0]
            assert len(t) == K and len(set(t)) == K and (np.diff(t) > 0).all() and t[-1] <= pos[r]
        note("example: step %d, %d drafts" % (step, drafts))
        check_attention(out, None, turned, held(layer, [ctx] * R), [drafts * b for b in range(R + 1)], 64 ** -0.5,
                        selection=sel, what="step %d" % step)
        assert np.isfinite(f64(out)).all()
