"""What pins the oracle of the page step (CPU)."""
import copy

import numpy as np

from oracle.pages import Pool


def test_hand_worked_step():
    p = Pool(pages=6, page=4, requests=3, width=3)
    s = p.step([5, 0, 3], T=10, ld=100)
    # pages 5, 4 to the first request, 3 to the third
    assert p.tables == [[5, 4], [], [3]] and p.length == [5, 0, 3] and p.free == [0, 1, 2]
    assert s["q_start"].tolist() == [0, 5, 5, 8] and s["taken"].tolist() == [5, 0, 3]
    assert s["slots"].tolist() == [20, 21, 22, 23, 16, 12, 13, 14, -1, -1]
    assert s["positions"].tolist() == [0, 1, 2, 3, 4, 0, 1, 2, 0, 0]
    assert s["dense"].tolist() == [0, 1, 2, 3, 4, 200, 201, 202, -1, -1]
    assert s["row_len"].tolist() == [1, 2, 3, 4, 5, 1, 2, 3, 0, 0]
    # the first is cut back to 2 (page 4 returns), the second asks for more pages than are left, the third for none
    s = p.step([0, 13, 1], T=20, keep=[2, 0, 3])
    assert p.length == [2, 0, 4] and p.tables == [[5], [], [3]] and p.free == [0, 1, 2, 4]
    assert s["taken"].tolist() == [0, 0, 1] and s["q_start"].tolist() == [0, 0, 13, 14]
    assert s["slots"].tolist() == [-1] * 13 + [15] + [-1] * 6
    # wider than the table; more rows than the buffers hold
    assert p.step([0, 13, 0], T=20)["taken"].tolist() == [0, 0, 0]
    assert p.step([3, 3, 1], T=6)["taken"].tolist() == [3, 3, 0]
    assert p.step([3, -4, 1], T=6)["q_start"].tolist() == [0, 3, 3, 4]


def test_pages_are_never_lost_or_shared_and_steps_can_be_taken_back():
    rng = np.random.default_rng(1)
    p = Pool(pages=60, page=8, requests=7, width=12)
    for i in range(300):
        before = copy.deepcopy(p)
        keep = [int(rng.integers(0, n + 1)) if rng.random() < 0.4 else n for n in p.length]
        if rng.random() < 0.3:
            keep[int(rng.integers(0, 7))] = 0
        new = [int(rng.integers(0, 40)) if rng.random() < 0.5 else 0 for _ in range(7)]
        s = p.step(new, T=150, keep=keep)
        held = [q for t in p.tables for q in t]
        assert sorted(held + p.free) == list(range(60))
        assert [len(t) for t in p.tables] == [-(-n // 8) for n in p.length]
        live = s["slots"][s["slots"] >= 0]
        assert len(set(live.tolist())) == len(live) == s["taken"].sum()
        if keep == before.length:   # nothing was cut back
            undone = copy.deepcopy(p)
            undone.step([0] * 7, T=0, keep=keep)
            assert undone.tables == before.tables and undone.free == before.free and undone.length == before.length


def test_planted_mistakes():
    """Handing pages out from the bottom, pushing them in the other order, and letting a later request overtake
    one that was refused change the hand-worked step."""
    class Bottom(Pool):
        def step(self, *a, **k):
            self.free.reverse()
            r = Pool.step(self, *a, **k)
            self.free.reverse()
            return r
    p = Bottom(6, 4, 3, 3)
    assert p.step([5, 0, 3], T=10)["slots"].tolist()[:5] != [20, 21, 22, 23, 16]
    q = Pool(6, 4, 3, 3)
    q.step([12, 0, 0], T=12)
    q.step([0, 0, 0], T=1, keep=[0, 0, 0])
    assert q.free == [0, 1, 2, 3, 4, 5]
    q = Pool(2, 4, 3, 3)
    assert q.step([4, 12, 4], T=30)["taken"].tolist() == [4, 0, 0]   # (no overtaking among those that need pages)
