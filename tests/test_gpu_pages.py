"""Page steps on the GPU against the oracle, whole numbers for whole numbers."""
import numpy as np
import pytest
import torch

from oracle.pages import Pool
from tests.gpu_cases import note
from tests.kv4_cases import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def check(pool, ref, got, want, what):
    for name, a in got._asdict().items():
        if a is not None:
            assert np.array_equal(a.cpu().numpy(), want[name]), (what, name)
    assert np.array_equal(pool.block_table.cpu().numpy(), ref.table()), (what, "table")
    assert pool.ctx_len.cpu().tolist() == ref.length, what
    n = int(pool.free_count.cpu()[0])
    assert n == len(ref.free) and pool.free_pages[:n].cpu().tolist() == ref.free, what


@pytest.mark.parametrize("requests,page,width,pages,longest,T", [
    (1, 64, 10, 10, 100, 128), (5, 1, 40, 60, 9, 40), (37, 16, 12, 200, 60, 700), (256, 16, 4, 300, 3, 256),
    (300, 8, 20, 2000, 40, 2048), (300, 8, 20, 2000, 40, 9000), (1100, 4, 6, 3000, 5, 1500), (2500, 16, 9, 9000, 30, 40000)])
def test_random_steps(G, requests, page, width, pages, longest, T):
    rng = np.random.default_rng(requests + page)
    pool, ref = G.new_page_pool(pages, page, requests, width), Pool(pages, page, requests, width)
    for i in range(8):
        new = np.where(rng.random(requests) < 0.7, rng.integers(-2, longest + 1, requests), 0)
        keep = None
        if i % 2:
            length = np.array(ref.length)
            keep = np.where(rng.random(requests) < 0.5, rng.integers(-3, length + 3), length)
            keep = np.where(rng.random(requests) < 0.2, 0, keep)
        note("pages %s step %d" % ((requests, page, width, pages, longest, T), i))
        got = G.gvr_page_step(pool, ints(new), T, keep=None if keep is None else ints(keep), ld=width * page)
        check(pool, ref, got, ref.step(new, T, keep, width * page), i)


@pytest.mark.parametrize("requests,T", [(40, 500), (40, 5000)])
def test_a_step_taken_back_restores_the_pool(G, requests, T):
    note("pages back %d" % T)
    rng = np.random.default_rng(T)
    pool = G.new_page_pool(900, 16, requests, 20)
    G.gvr_page_step(pool, ints(rng.integers(0, 100, requests)), 5000)
    for _ in range(3):   # a stack in no particular order
        G.gvr_page_step(pool, ints(rng.integers(0, 20, requests)), 5000, keep=ints(rng.integers(0, 60, requests)))
    n = int(pool.free_count[0])
    before = [pool.block_table.clone(), pool.ctx_len.clone(), pool.free_pages[:n].clone(), pool.free_count.clone()]
    step = G.prepare_gvr_page_step(pool, ints(rng.integers(0, 12, requests)), T)
    undo = G.prepare_gvr_page_step(pool, ints(np.zeros(requests)), 0, keep=before[1])
    first = [t.clone() for t in step() if t is not None]
    assert int(step.out.taken.sum()) > 0
    undo()
    after = [pool.block_table, pool.ctx_len, pool.free_pages[:n], pool.free_count]
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    assert all(torch.equal(a, b) for a, b in zip(first, [t for t in step() if t is not None]))


def test_edges(G):
    note("pages edges")
    for T in (0, 5, 3000):   # no requests: every row is padding
        s = G.gvr_page_step(G.new_page_pool(4, 16, 0, 3), ints([]), T)
        assert s.q_start.tolist() == [0] and (s.slots == -1).all() and (s.positions == 0).all() and (s.row_len == 0).all()
    for T in (0, 3000):      # no pages, no width, no rows
        pool, ref = G.new_page_pool(0, 16, 2, 0), Pool(0, 16, 2, 0)
        check(pool, ref, G.gvr_page_step(pool, ints([0, 3]), T), ref.step([0, 3], T), T)
    big = 2 ** 31 - 1        # sums beyond 32 bits
    for T in (10, 3000):
        pool, ref = G.new_page_pool(10, 4, 5, 2), Pool(10, 4, 5, 2)
        new = [3, big, big, big, 2]
        check(pool, ref, G.gvr_page_step(pool, ints(new), T), ref.step(new, T), T)
    # lengths and counts outside what they can be count as the nearest that they can
    pool = G.new_page_pool(6, 4, 2, 2)
    pool.ctx_len.copy_(ints([-7, 1000]))
    pool.free_count.fill_(99)
    s = G.gvr_page_step(pool, ints([2, 1]), 8)
    assert s.taken.tolist() == [2, 0] and pool.ctx_len.tolist() == [2, 8] and int(pool.free_count[0]) == 5
    # a table entry that is no page
    pool.block_table.fill_(-1)
    assert G.gvr_page_step(pool, ints([1, 0]), 8).slots.tolist() == [-1] * 8


def test_replayed_graph_and_given_workspace(G):
    """Two graphs of one pool share a workspace; replays in turn go on from where the pool stands."""
    for T in (64, 4000):
        note("pages graph %d" % T)
        pool, ref = G.new_page_pool(400, 8, 30, 30), Pool(400, 8, 30, 30)
        new, keep = ints(np.zeros(30)), ints(np.full(30, 2 ** 31 - 1))
        ws = torch.empty(G.gvr_page_step_workspace(30), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        graphs, calls = [], []
        for rows, ld in ((T, None), (T // 2, 1000)):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                calls.append(G.prepare_gvr_page_step(pool, new, rows, keep=keep, ld=ld, workspace=ws))
                calls[-1]()
            graphs.append(g)
        rng = np.random.default_rng(T)
        for i in range(8):
            n = rng.integers(0, 3 if T == 64 else 90, 30)
            k = rng.integers(0, 50, 30) if i == 4 else np.full(30, 2 ** 31 - 1)
            new.copy_(ints(n))
            keep.copy_(ints(k))
            graphs[i % 2].replay()
            torch.cuda.synchronize()
            check(pool, ref, calls[i % 2].out, ref.step(n, T if i % 2 == 0 else T // 2, k, 1000 * (i % 2)), i)
