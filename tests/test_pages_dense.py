"""What pins the oracle's rows of a dense cache with fewer rows than a page table holds tokens (CPU)."""
import numpy as np
import pytest

from oracle.pages import Pool


def test_tokens_without_a_row():
    p = Pool(pages=6, page=4, requests=2, width=3)
    s = p.step([6, 3], T=10, ld=4)
    # both are served; the first has rows 0 .. 3, the second 4 .. 7
    assert s["taken"].tolist() == [6, 3] and s["row_len"].tolist() == [1, 2, 3, 4, 5, 6, 1, 2, 3, 0]
    assert s["dense"].tolist() == [0, 1, 2, 3, -1, -1, 4, 5, 6, -1]
    assert p.step([1, 2], T=3, ld=4)["dense"].tolist() == [-1, 7, -1]
    assert p.step([1, 1], T=2, ld=0)["dense"].tolist() == [-1, -1]


@pytest.mark.parametrize("ld", [1, 7, 30])
def test_no_row_belongs_to_two_requests(ld):
    rng = np.random.default_rng(ld)
    p = Pool(pages=60, page=8, requests=5, width=5)
    owner = {}
    for _ in range(20):
        s = p.step(rng.integers(0, 9, 5), T=60, keep=rng.integers(0, 33, 5), ld=ld)
        of = np.searchsorted(s["q_start"][1:], np.arange(60), side="right")
        for r, row in zip(of, s["dense"]):
            assert row < 5 * ld and (row < 0 or owner.setdefault(int(row), r) == r)
    assert len(owner) > 5 * ld // 2
