"""Slots as pages of the state cache: counts, copies and compaction against a
plain model, byte for byte."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2608_27513_amd import damp as D
from paper_2608_27513_amd import serving as S

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def pool_of(seed, layers, slots, HV, d, k_hi=8, kind=D.DAMP_STATE_MIXED, fmt=None):
    lay = D.damp_layout_init(d, d, k_hi, kind)
    if fmt is not None:
        lay.hi_dtype, lay.group, lay.meta_dtype, lay.hadamard, lay.code_dtype = fmt
    pool = D.Pool(lay, layers, slots, HV)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pool.buffer.copy_(torch.randint(0, 256, pool.buffer.shape, generator=gen, device="cuda",
                                    dtype=torch.uint8))
    return pool, pool.buffer.view(layers, slots, -1)


LAYOUTS = [dict(d=64), dict(d=16, k_hi=3), dict(d=128, k_hi=16),
           dict(d=64, k_hi=0, kind=D.DAMP_STATE_FP32),
           dict(d=32, fmt=(D.DAMP_DT_FP16, 16, D.DAMP_DT_E4M3, 0, D.DAMP_DT_E2M1)),
           dict(d=64, fmt=(D.DAMP_DT_FP16, 32, D.DAMP_DT_FP16, 1, D.DAMP_DT_U4))]


@pytest.mark.parametrize("lay", range(len(LAYOUTS)))
@pytest.mark.parametrize("HV", [1, 5, 32])
def test_fork(lay, HV):
    print(f"fork {lay} {HV}", flush=True)
    pool, pages = pool_of(lay, 3, 23, HV, **LAYOUTS[lay])
    before = pages.clone()
    S.damp_slots_fork(pool, i32([4, 22, 4, 9]), i32([[0, 1, -1], [5, 23, 6], [7, 8, 10], [-9, 99, -1]]))
    for a, b in ((4, 0), (4, 1), (22, 5), (22, 6), (4, 7), (4, 8), (4, 10)):
        before[:, b] = before[:, a]
    assert torch.equal(pages, before)
    S.damp_slots_fork(pool, i32([3, -1, 23, 2]), i32([11, 12, 13, 14]), layer=1)
    before[1, 11], before[1, 14] = before[1, 3], before[1, 2]
    assert torch.equal(pages, before)


def test_fork_many_and_none():
    print("fork many", flush=True)
    pool, pages = pool_of(9, 2, 400, 2, 32)
    before = pages.clone()
    perm = np.random.RandomState(0).permutation(400)
    S.damp_slots_fork(pool, i32(perm[:40]), i32(perm[40:].reshape(40, 9)))
    for a, row in zip(perm[:40], perm[40:].reshape(40, 9)):
        before[:, row] = before[:, a:a + 1]
    assert torch.equal(pages, before)
    S.damp_slots_fork(pool, i32([]), i32([]))
    S.damp_slots_fork(pool, i32([1]), torch.zeros(1, 0, dtype=torch.int32, device="cuda"))
    assert torch.equal(pages, before)


def test_offsets_beyond_32_bits():
    print("slots offsets", flush=True)
    pool, pages = pool_of(3, 1, 2200, 32, 128, 0, D.DAMP_STATE_FP32)  # 4.6 GB
    want = pages[0, 2199].clone()
    S.damp_slots_fork(pool, i32([2199]), i32([[0, 2198]]))
    assert torch.equal(pages[0, 0], want) and torch.equal(pages[0, 2198], want)
    refs = torch.zeros(2200, dtype=torch.int32, device="cuda")
    refs[2199] = 2
    pages[0, 2199].add_(1)
    want = pages[0, 2199].clone()
    where, live = S.damp_slots_compact(pool, refs)
    assert int(live) == 1 and int(where[2199]) == 0 and torch.equal(pages[0, 0], want)


@pytest.mark.parametrize("slots", [1, 2, 7, 64, 1023, 1024, 1025, 5000])
def test_counts(slots):
    print(f"counts {slots}", flush=True)
    rng = np.random.RandomState(slots)
    refs = rng.randint(0, 3, slots).astype(np.int32)
    dev = i32(refs)
    names = rng.randint(-2, slots + 2, 3000).astype(np.int32)
    inside = names[(names >= 0) & (names < slots)]
    S.damp_slots_retain(dev, i32(names))
    np.add.at(refs, inside, 1)
    assert dev.tolist() == refs.tolist()
    more = np.concatenate([names, names, names])
    S.damp_slots_release(dev, i32(more))
    for s in inside:
        refs[s] -= 3
    refs = np.maximum(refs, 0)
    assert dev.tolist() == refs.tolist()
    for n in (0, 1, slots // 2, slots + 3):
        free = np.flatnonzero(refs == 0)[:n]
        got = S.damp_slots_alloc(dev, n)
        assert got.tolist() == free.tolist() + [-1] * (n - len(free))
        refs[free] = 1
        assert dev.tolist() == refs.tolist()


@pytest.mark.parametrize("slots,share", [(1, 0.0), (1, 1.0), (2, 0.5), (17, 0.3), (64, 0.6),
                                         (64, 0.0), (64, 1.0), (1500, 0.5), (3001, 0.9)])
def test_compact(slots, share):
    print(f"compact {slots} {share}", flush=True)
    rng = np.random.RandomState(slots)
    for layers, HV, d in ((1, 1, 16), (3, 2, 32)):
        pool, pages = pool_of(slots, layers, slots, HV, d, 4)
        refs = np.where(rng.rand(slots) < share, rng.randint(1, 4, slots), 0).astype(np.int32)
        where, new, live, moves = ref.compact(refs)
        before = pages.clone()
        dev = i32(refs)
        got_map, got_live = S.damp_slots_compact(pool, dev)
        assert got_map.tolist() == where.tolist()
        assert dev.tolist() == new.tolist() and int(got_live) == live
        for a, b in moves:
            before[:, b] = before[:, a]
        assert torch.equal(pages, before)


def test_compact_moves_large_slots():
    """More pieces of work than workgroups."""
    print("compact large", flush=True)
    pool, pages = pool_of(5, 6, 40, 32, 128, 16)
    refs = np.array([0, 1] * 20, np.int32)
    where, new, live, moves = ref.compact(refs)
    before = pages.clone()
    dev = i32(refs)
    S.damp_slots_compact(pool, dev)
    for a, b in moves:
        before[:, b] = before[:, a]
    assert torch.equal(pages, before) and dev.tolist() == new.tolist()


def test_graph_replays():
    """Alloc, fork, release and compact in a graph, replayed on fresh counts."""
    print("slots graph", flush=True)
    pool, pages = pool_of(6, 2, 32, 2, 32)
    first, refs0 = pages.clone(), i32([1, 0, 2, 0, 0, 1, 0, 0] * 4)
    refs, ids, src = refs0.clone(), torch.empty(3, dtype=torch.int32, device="cuda"), i32([0, 2, 5])
    where, live = torch.empty(32, dtype=torch.int32, device="cuda"), i32([0])
    ws = torch.empty(S.damp_slots_compact_workspace_bytes(pool), dtype=torch.uint8, device="cuda")

    def turn():
        S.damp_slots_alloc(refs, 3, out=ids)
        S.damp_slots_fork(pool, src, ids)
        S.damp_slots_release(refs, src)
        S.damp_slots_compact(pool, refs, workspace=ws, map_out=where, live=live)

    turn()
    torch.cuda.synchronize()
    want = [t.clone() for t in (refs, ids, where, live, pages)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for i in range(4):
        pages.copy_(first)
        refs.copy_(refs0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((refs, ids, where, live, pages), want)), i


def test_checked_slots(monkeypatch):
    pool, pages = pool_of(7, 1, 8, 1, 16)
    monkeypatch.setenv("DAMP_CHECK_SLOTS", "1")
    before = pages.clone()
    for src, dst, what in (([0, 1], [2, 2], "more than once"), ([0, 1], [1, 3], "read for 1"),
                           ([4], [4], "read for 0")):
        with pytest.raises(D.DampError, match=what):
            S.damp_slots_fork(pool, i32(src), i32(dst))
    assert torch.equal(pages, before)


def test_binding_refusals():
    pool, _ = pool_of(8, 1, 8, 1, 16)
    with pytest.raises(ValueError, match="dst has shape"):
        S.damp_slots_fork(pool, i32([1, 2]), i32([3]))
    with pytest.raises(ValueError, match="src"):
        S.damp_slots_fork(pool, i32([1, 2]).long(), i32([3, 4]))
    with pytest.raises(D.DampError, match="layer"):
        S.damp_slots_fork(pool, i32([1]), i32([3]), layer=1)
    with pytest.raises(ValueError, match="refs has shape"):
        S.damp_slots_compact(pool, i32([1, 2]))
    with pytest.raises(D.DampError, match="workspace"):
        S.damp_slots_compact(pool, i32([1] * 8), workspace=torch.empty(8, dtype=torch.uint8,
                                                                       device="cuda"))
