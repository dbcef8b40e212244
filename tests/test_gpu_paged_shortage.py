"""Pages that were missing in paged_extend and given back by paged_release all the same: a step
that goes on without the host looking."""
from __future__ import annotations

import random

import pytest
import torch

from tests import paged_refs as refs
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32 = torch.int32


@pytest.fixture(scope="module")
def pa():
    import paper_2609_29219_amd as pa
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return pa


def ints(values):
    return torch.tensor(values, dtype=I32, device=DEV)


def release(table, seq, keep, free, n_free, page):
    """n_left and the list: page numbers below zero are no pages."""
    free, n_free = list(free), min(max(n_free, 0), len(free))
    for row, s, k in zip(table, seq, keep):
        for p in row[-(-k // page):min(-(-s // page), len(row))]:
            if p >= 0 and n_free < len(free):
                free[n_free] = p
                n_free += 1
    return n_free, free


def test_a_shortage_that_nobody_saw(pa):
    announce("paged_release after a shortage")
    page, P = 8, 6
    table = torch.full((3, 5), -1, dtype=I32, device=DEV)
    free, n_free, seq = ints([3, 0, 5, 1, 4, 2]), ints([P]), ints([0, 0, 0])
    # 9 pages asked for, 6 there: the last request lacks three
    slots, _, _, kv, left = pa.paged_extend(table, seq, ints([16, 24, 30]), free, n_free, page, 70)
    assert left.tolist() == [-3] and table.tolist()[2] == [3, -1, -1, -1, -1]
    # all of it is counted as if it were there; the last request ends
    left = pa.paged_release(table, kv, ints([16, 24, 0]), free, left, page)
    assert left.tolist() == [1] and free.tolist()[0] == 3
    # a new one in its place gets that page, and lacks one
    seq = ints([16, 24, 0])
    slots, _, _, kv, left = pa.paged_extend(table, seq, ints([0, 0, 9]), free, left, page, 9)
    assert left.tolist() == [-1] and slots.tolist() == [24 + i for i in range(8)] + [-1]
    # everything ends: each page is there once
    left = pa.paged_release(table, kv, ints([0, 0, 0]), free, left, page)
    assert left.tolist() == [P] and sorted(free.tolist()) == list(range(P))


@pytest.mark.parametrize("R,page", [(1, 8), (5, 16), (64, 16), (65, 8), (600, 16), (3000, 32)])
@pytest.mark.parametrize("holes", [0.0, 0.003, 0.3, 1.0])
def test_holes_anywhere(pa, R, page, holes):
    announce(f"paged_release R={R} page={page} holes={holes}")
    rng = random.Random(R)
    for wide in (0, 3000):  # (a wide table may be walked another way)
        seq = [rng.choice([0, page, rng.randint(0, 60 * page)]) for _ in range(R)]
        keep = [rng.choice([0, s, rng.randint(0, s), s + 100]) for s in seq]
        held = [-(-s // page) for s in seq]
        most = max(max(held), wide if R < 100 else 0) + 1
        table = [[(-1 - rng.randrange(3) if rng.random() < holes else rng.randrange(1 << 20))
                  if i < h else -9 for i in range(most)] for h in held]
        valid = release(table, seq, keep, [0] * (sum(held) + 9), 4, page)[0]
        for room in (sum(held) + 9, valid, max(4, valid - 5), 4):
            free = [rng.randrange(1 << 20) for _ in range(room)]
            n_left, want = release(table, seq, keep, free, 4, page)
            got = ints(free)
            left = pa.paged_release(ints(table), ints(seq), ints(keep), got, ints([4]), page)
            # behind the pages that are there the list is nobody's
            assert left.tolist() == [n_left] and got.tolist()[:n_left] == want[:n_left]
            if holes == 0.0:
                assert refs.release(table, seq, keep, free, 4, page) == (n_left, got.tolist())


def test_many_steps_short_of_pages(pa):
    # requests that come, grow, lose drafted tokens and end, with too few pages every other step
    announce("paged steps short of pages")
    rng, page, P, R, most = random.Random(4), 8, 60, 9, 20
    table, seq = torch.full((R, most), -1, dtype=I32, device=DEV), ints([0] * R)
    free, n_free = torch.randperm(P, device=DEV).int(), ints([P])
    short = 0
    for _ in range(60):
        new = [rng.choice([0, 1, 5, 40]) if s < 110 else 0 for s in seq.tolist()]
        *_, kv, left = pa.paged_extend(table, seq, ints(new), free, n_free, page, sum(new) + 1)
        short += left.item() < 0
        keep = [rng.choice([s, s, max(0, s - 3), 0]) for s in kv.tolist()]
        n_free, seq = pa.paged_release(table, kv, ints(keep), free, left, page), ints(keep)
        n = n_free.item()
        held = [p for row, s in zip(table.tolist(), keep) for p in row[:-(-s // page)] if p >= 0]
        assert sorted(held + free.tolist()[:n]) == list(range(P))
    assert short > 5


@pytest.mark.parametrize("R", [70, 300])
def test_replayed_release(pa, R):
    # one captured call, of one launch or two, holes in some replays and none in others
    announce(f"paged_release in a graph R={R}")
    page, most = 16, 400
    rng = random.Random(6)
    seq, keep = ints([most * page] * R), ints([16 * (i % 3) for i in range(R)])
    free, n_free = torch.zeros(R * most + 4, dtype=I32, device=DEV), ints([2])
    table, left = torch.zeros(R, most, dtype=I32, device=DEV), ints([0])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pa.paged_release(table, seq, keep, free, n_free, page, n_left=left)
    for holes in (0.0, 0.1, 0.0, 1.0, 0.0):
        rows = [[-1 if rng.random() < holes else rng.randrange(1 << 20) for _ in range(most)]
                for _ in range(R)]
        table.copy_(ints(rows))
        free.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        n, want = release(rows, seq.tolist(), keep.tolist(), [0] * len(free), 2, page)
        assert left.tolist() == [n] and free.tolist()[:n] == want[:n]
