"""Tensors that a call makes for a given stream belong to that stream: torch's allocator orders a block's uses by the stream that it was
allocated on, so a block of another stream could still be in use there."""
import pytest
import torch

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


def owner(ptr):
    """Handle of the stream whose pool the block at ptr belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= ptr < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no segment holds the block")


@pytest.mark.parametrize("kind", ["stream", "handle", "default handle", "current"])
def test_made_tensors_belong_to_the_stream(G, kind):
    s = torch.cuda.Stream()
    side = torch.cuda.Stream()
    given = {"stream": s, "handle": s.cuda_stream, "default handle": 0, "current": side}[kind]
    want = {"stream": s.cuda_stream, "handle": s.cuda_stream, "default handle": 0, "current": side.cuda_stream}[kind]
    note("streams: %s" % kind)
    cache = torch.randint(0, 100, (300, 16, G.gvr_kv4_record_bytes(2, 64)), dtype=torch.uint8, device=DEV)
    tab = torch.arange(300, dtype=torch.int32, device=DEV).view(1, -1)
    lens = torch.tensor([4800], dtype=torch.int32, device=DEV)
    q = torch.randn((1, 8, 64), device=DEV).bfloat16()
    pos = torch.zeros(1, dtype=torch.int32, device=DEV)
    slots = torch.arange(40, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cs = G.gvr_rope_table(8, dict(d_rope=64), device=DEV, stream=given)
        torch.cuda.synchronize()
        y = G.gvr_rope_rotate(q, pos, cs, stream=given)
        k, v = G.gvr_kv4_read(cache, slots, 2, 64, stream=given)
        out = G.gvr_kv4_attention(q, cache, tab, lens, 2, stream=given)
        call = G.prepare_gvr_kv4_attention(q, cache, tab, lens, 2, stream=given)
        call()
        torch.cuda.synchronize()
        assert G.gvr_kv4_attention_workspace(q, cache, tab, lens, 2) > 1
        workspace = call._args[2].value
        for name, ptr in (("table", cs.data_ptr()), ("rotated", y.data_ptr()), ("keys", k.data_ptr()),
                          ("values", v.data_ptr()), ("attention", out.data_ptr()), ("prepared", call.out.data_ptr()),
                          ("workspace", workspace)):
            assert owner(ptr) == want, name
        assert torch.equal(out, call.out) and torch.equal(out, G.gvr_kv4_attention(q, cache, tab, lens, 2))


def test_made_tensors_of_the_selection_belong_to_the_stream(G):
    s, side = torch.cuda.Stream(), torch.cuda.Stream()
    scores = torch.randn((3, 5000), device=DEV)
    q = torch.zeros((3, 64, 128), dtype=torch.uint8, device=DEV)
    w, k, ks = torch.ones((3, 64), device=DEV), torch.zeros((3, 300, 128), dtype=torch.uint8, device=DEV), torch.ones((3, 300), device=DEV)
    lens = torch.full((3,), 300, dtype=torch.int32, device=DEV)
    note("streams: selection")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        made = [G.gvr_topk(scores, None, None, 2048, stream=s), G.radix_topk(scores, None, None, 2048, stream=s),
                G.gvr_topk_ex(scores, None, None, 2048, stream=s), G.prepare_gvr_topk(scores, None, None, 2048, stream=s)(),
                G.gvr_rope_g(5000, device=DEV, stream=s), G.gvr_rope_prior(5000, 2048, device=DEV, stream=s),
                G.gvr_indexer_scores(q, w, k, ks, lens, stream=s), *G.gvr_indexer_topk(q, w, k, ks, lens, None, 100, stream=s)]
        torch.cuda.synchronize()
        for i, t in enumerate(made):
            assert owner(t.data_ptr()) == s.cuda_stream, i
        assert torch.equal(made[0], made[1]) and torch.equal(made[0], made[2]) and torch.equal(made[0], made[3])
