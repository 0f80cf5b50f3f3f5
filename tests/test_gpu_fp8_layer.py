"""The operators as a layer uses them, one after the other: hidden states through 8-bit projections, a page step, the
indexer's keys quantised into their cache, the attention over what the Top-K selected; each against the oracles."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from oracle import fp8 as F
from oracle import indexer as I
from oracle import kv4 as O
from oracle.pages import Pool
from tests.fp8_cases import close, cut_off, product_bound
from tests.gpu_cases import note
from tests.kv4_cases import DEV, Sequences, check_attention

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    oracle.build(force=False)
    return g


@pytest.mark.parametrize("drafts", [1, 2])
def test_hidden_states_to_attention(G, drafts):
    from sparse_decode import Projections, SparseLayer
    torch.manual_seed(drafts)
    R, n, K, longest, hidden, page = 3, 90, 32, 128, 200, 16
    layer = SparseLayer(R, longest, q_heads=8, kv_heads=2, head_dim=64, K=K, page=page, drafts=drafts)
    project = Projections(hidden, q_heads=8, kv_heads=2, head_dim=64)
    order = layer.pool.free_pages.cpu().tolist()
    pages = Pool(len(order), page, R, longest // page)
    pages.free = list(order)
    weight = project.weight.codes.cpu().numpy(), project.weight.scale.cpu().numpy()
    table = layer.table.cpu().numpy()
    keys = np.zeros((R, longest, 128))
    ctx = 0
    for step, m in enumerate([n, drafts, drafts, drafts]):
        note("layer: drafts %d step %d" % (drafts, step))
        x = torch.randn((R * m, hidden), device=DEV).bfloat16()
        parts = project(x)
        # the product of the hidden states' codes and the weight's
        qx = F.quantise(x.float().cpu().numpy())
        ref, mag = F.product(*qx, *weight, 128)
        y = torch.cat([t.flatten(1) for t in parts], dim=1)
        close(y, ref, product_bound(mag, ref, hidden, "bf16", cut_off(F.values(*qx), F.values(*weight, 128))))
        q, k, v, iq, ik = parts
        out = layer.prompt(q, k, v, ik) if step == 0 else layer.decode(q, k, v, iq, ik)
        want = pages.step([m] * R, R * m, ld=longest)
        assert np.array_equal(layer.blocks.cpu().numpy(), pages.table()) and layer.length.tolist() == pages.length
        # the indexer's keys in their cache
        codes, scale = F.quantise(ik[:, 0].float().cpu().numpy(), pow2=True)
        assert np.array_equal(layer.index_k.cpu().numpy().reshape(R * longest, 128)[want["dense"]], codes)
        assert np.array_equal(layer.index_scale.cpu().numpy().reshape(-1)[want["dense"]], scale[:, 0])
        keys.reshape(R * longest, 128)[want["dense"]] = F.values(codes, scale)
        turned = torch.from_numpy(O.rotate(q.float().cpu().numpy(), want["positions"], table)).bfloat16()
        ctx += m
        seqs = Sequences.__new__(Sequences)
        seqs.table, seqs.cache = layer.blocks.cpu().numpy(), layer.cache.cpu().numpy()
        seqs.ctx, seqs.page, seqs.heads, seqs.D = [ctx] * R, page, 2, 64
        sel = None
        if step:
            # a selected token's score is no lower than any other's, by more than both scores' rounding
            sel = layer.selected.cpu().numpy()
            qc, qs = F.quantise(iq.float().cpu().numpy(), pow2=True)
            w = layer.index_w.cpu().numpy() * qs[:, :, 0]
            args = (qc, w, layer.index_k.cpu().numpy(), layer.index_scale.cpu().numpy())
            scores = I.indexer_scores(*args, group=drafts, row_len=want["row_len"])
            slack = 2 * (128 + 64 + 4) * 2.0 ** -24 * I.magnitude(*args, group=drafts, row_len=want["row_len"])
            for r in range(R * m):
                see = want["row_len"][r]
                rest = np.setdiff1d(np.arange(see), sel[r])
                assert len(set(sel[r])) == K and sel[r].max() < see
                assert scores[r, sel[r]].min() >= (scores[r, rest] - slack[r, rest]).max() - slack[r, sel[r]].max()
        check_attention(out, None, turned, seqs, [m * b for b in range(R + 1)], 64 ** -0.5, selection=sel, what="step %d" % step)


def test_made_tensors_belong_to_the_stream(G):
    from tests.test_gpu_streams import owner
    s, side = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.randn((300, 640), device=DEV).bfloat16()
    pool = G.new_page_pool(50, 16, 4, 8)
    new = torch.tensor([3, 0, 20, 1], dtype=torch.int32, device=DEV)
    note("fp8 streams")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        q = G.gvr_fp8_quantize(x, stream=s)
        a, b = G.gvr_fp8_quantize_matrix(x, transposed=True, stream=s)
        y = G.gvr_fp8_matmul(*q, *a, stream=s)
        step = G.gvr_page_step(pool, new, 64, ld=128, stream=s)
        torch.cuda.synchronize()
        for t in (*q, *a, *b, y, *step):
            assert owner(t.data_ptr()) == s.cuda_stream
    assert torch.equal(y, G.gvr_fp8_matmul(*G.gvr_fp8_quantize(x), *G.gvr_fp8_quantize_matrix(x)))


def test_captured_training_step(G):
    """Forward and backward of the linear layer in a graph, replayed with new inputs."""
    note("fp8 captured step")
    x = torch.randn((200, 384), device=DEV).bfloat16().requires_grad_()
    w = torch.randn((256, 384), device=DEV).requires_grad_()
    dy = torch.randn((200, 256), device=DEV).bfloat16()

    def step():
        y = G.gvr_fp8_linear(x, w)
        return (y.detach(), *torch.autograd.grad(y, (x, w), dy))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        with torch.no_grad():
            x.copy_(torch.randn_like(x))
            w.copy_(torch.randn_like(w))
            dy.copy_(torch.randn_like(dy))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b), i


def test_two_graphs_share_a_workspace(G):
    """Split products of two graphs through one workspace, replayed in turn."""
    note("fp8 shared workspace")
    a = G.gvr_fp8_quantize(torch.randn((128, 4096), device=DEV).bfloat16())
    b = [G.gvr_fp8_quantize_matrix(torch.randn((n, 4096), device=DEV), square=True) for n in (1024, 768)]
    n = max(G.gvr_fp8_matmul_workspace(*a, *m) for m in b)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    eager = [G.gvr_fp8_matmul(*a, *m, workspace=ws) for m in b]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for m in b:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(G.gvr_fp8_matmul(*a, *m, workspace=ws))
        graphs.append(g)
    for i in range(6):
        ws.fill_(0xFF)   # (nothing is expected of its contents)
        outs[i % 2].zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], eager[i % 2])
    # less workspace: fewer splits, another order of the sums
    none = G.gvr_fp8_matmul(*a, *b[0], workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
    assert (none.float() - eager[0].float()).abs().max() <= 2.0 ** -7 * none.float().abs().max()


def test_offsets_past_32_bits(G):
    """A matrix of more than 2^32 bytes of codes, quantised and multiplied: its last rows are those of a small one."""
    note("fp8 far offsets")
    rows, K = 540000, 8192
    assert rows * K > 1 << 32
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device=DEV)
    tail = torch.randn((300, K), device=DEV).bfloat16()
    x[-300:] = tail
    w = G.gvr_fp8_quantize_matrix(torch.randn((48, K), device=DEV), square=True)
    q = G.gvr_fp8_quantize(x)
    small = G.gvr_fp8_quantize(tail)
    assert torch.equal(q.codes[-300:], small.codes) and torch.equal(q.scale[-300:], small.scale)
    assert int(q.codes[:-300].max()) == 0
    y = G.gvr_fp8_matmul(*q, *w)
    ref = G.gvr_fp8_matmul(*small, *w)
    assert (y[:-300] == 0).all()
    # (another split of the sum, perhaps)
    assert (y[-300:].float() - ref.float()).abs().max() <= 2.0 ** -7 * ref.float().abs().max()
    del q, y
    t = G.gvr_fp8_quantize_matrix(x, straight=False, transposed=True)
    want = G.gvr_fp8_quantize_matrix(x[-384:].contiguous(), straight=False, transposed=True)   # (whole blocks of rows)
    assert rows % 128 == 96   # the last block of 128 rows starts 96 rows before the end
    assert torch.equal(t.codes[:, -96:], G.gvr_fp8_quantize_matrix(x[-96:].contiguous(), straight=False, transposed=True).codes)
    assert want.codes.shape == (K, 384)
