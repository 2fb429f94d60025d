"""GPU: block tables, slots and positions built from request lengths, against the request-by-request statement; whole numbers, so equal."""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu


def random_step(rng, B, page, longest, prefilling=0, chunk=1, leaving=0, spare=7):
    """A pool in a random state: tables with pages of the requests, the others on the stack, scattered."""
    cached = rng.integers(0, longest + 1, B)
    added = rng.integers(0, 2, B)
    order = rng.permutation(B)
    added[order[:prefilling]] = rng.integers(0, chunk + 1, prefilling)
    added[order[prefilling:prefilling + leaving]] = -1
    width = paged.pages_of(longest + chunk, page)
    held = [paged.pages_of(int(c), page) for c in cached]
    wanted = sum(max(0, paged.pages_of(int(c) + int(a), page) - h) for c, a, h in zip(cached, added, held) if a > 0)
    pages = sum(held) + wanted + spare
    names = rng.permutation(pages)
    table, at = np.full((B, width), -9, dtype=np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = names[at:at + h]
        at += h
    free = np.full(pages, -5, dtype=np.int32)
    free[:pages - at] = names[at:]
    return cached.astype(np.int32), added.astype(np.int32), table, free, pages - at


def run_and_compare(cached, added, page, table, free, count, cap, in_place=False, table_pad=0):
    import torch
    import paper_2601_16032_b200 as sa
    dev = "cuda:0"
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
    c, a, f, n = up(cached), up(added), up(free), torch.tensor([count], dtype=torch.int32, device=dev)
    wide = torch.full((table.shape[0], table.shape[1] + table_pad), -77, dtype=torch.int32, device=dev)
    t = wide[:, :table.shape[1]]
    t.copy_(up(table))
    p = sa.page_plan(c, a, page, t, f, n, cap, seq_len=c if in_place else None, free_count_out=n if in_place else None)
    sa.attn_device_status()
    want = paged.page_plan(cached, added, page, table, free, count, len(free), cap)
    got = dict(table=t, free=f, count=p.free_count, seq_len=p.seq_len, q_start=p.q_start, slot=p.slot, position=p.position, request=p.request, info=p.info)
    for name, g in got.items():
        assert np.array_equal(g.cpu().numpy().reshape(-1), np.asarray(want[name]).reshape(-1)), name
    assert (wide[:, table.shape[1]:] == -77).all()
    if not in_place:
        assert np.array_equal(c.cpu().numpy(), cached) and int(n) == count
    return want


@pytest.mark.parametrize("page", [1, 16, 24, 128])
@pytest.mark.parametrize("B,longest,prefilling,chunk,leaving", [
    (1, 0, 0, 1, 0), (1, 40, 0, 1, 0), (1, 50, 0, 1, 1), (3, 17, 1, 100, 1), (31, 300, 5, 64, 6), (32, 300, 32, 33, 0), (33, 64, 0, 1, 33),
    (257, 500, 20, 40, 30), (1025, 200, 100, 60, 200), (2000, 30, 3, 3000, 500)])
def test_random_steps(page, B, longest, prefilling, chunk, leaving):
    rng = np.random.default_rng(B * 1000 + page)
    for turn in range(2):
        step = random_step(rng, B, page, longest, prefilling, chunk, leaving)
        tokens = int(step[1].clip(0).sum())
        want = run_and_compare(step[0], step[1], page, *step[2:], tokens + (0 if turn else 13), in_place=bool(turn), table_pad=3 * turn)
        assert want["info"][0] == 0


def test_most_requests():
    rng = np.random.default_rng(5)
    step = random_step(rng, 8192, 16, 60, 10, 50, 700)
    run_and_compare(step[0], step[1], 16, *step[2:], 9000)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,longest,leaving", [(700, 1, 1500, 400), (1, 1, 200000, 1), (40, 3, 5000, 40)])
def test_many_pages_given_back(B, page, longest, leaving, in_place):
    """More pages return to the stack than there are threads, and a request's many pages alone."""
    rng = np.random.default_rng(11)
    cached, added, table, free, count = random_step(rng, B, page, longest, leaving=leaving)
    if B == 1:   # the request holds all pages
        cached[0], held = longest, paged.pages_of(longest, page)
        table = rng.permutation(held + 7)[:table.shape[1]].astype(np.int32)[None]
        free, count = np.full(held + 7, -5, dtype=np.int32), 0
    run_and_compare(cached, added, page, table, free, count, int(np.maximum(added, 0).sum()) + 2, in_place=in_place)


@pytest.mark.parametrize("change,state", [
    (dict(cached=-1), 1), (dict(added=-2), 1), (dict(cached=10**6), 1), (dict(added=2**31 - 1), 1), (dict(count=-1), 1), (dict(count=10**6), 1),
    (dict(cap=0), 2), (dict(count=0), 3)])
def test_steps_that_do_not_fit_change_nothing(change, state):
    rng = np.random.default_rng(9)
    cached, added, table, free, count = random_step(rng, 40, 16, 300, 4, 70, 5)
    added[7] = 70
    cap = int(added.clip(0).sum()) + 3
    if "cached" in change:
        cached[11] = change["cached"]
    if "added" in change:
        added[11] = change["added"]
    if state == 3:
        added[added < 0] = 0
    want = run_and_compare(cached, added, 16, table, free, change.get("count", count), change.get("cap", cap))
    assert want["info"][0] == state


def test_token_sums_beyond_32_bits_do_not_fit():
    B, page, width = 64, 16, 1 << 22     # 64 requests of 2^26 tokens: 2^32 in all
    import torch
    import paper_2601_16032_b200 as sa
    dev = "cuda:0"
    zero, many = torch.zeros(B, dtype=torch.int32, device=dev), torch.full((B,), 1 << 26, dtype=torch.int32, device=dev)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    free, count = torch.arange(100, dtype=torch.int32, device=dev), torch.tensor([100], dtype=torch.int32, device=dev)
    p = sa.page_plan(zero, many, page, table, free, count, 50)
    assert p.info.tolist() == [2, 2**31 - 1, B << 22, 0] and (p.slot == -1).all() and p.q_start.sum() == 0 and p.seq_len.sum() == 0
    assert int(p.free_count) == 100


def test_pool_that_cannot_hold_what_is_given_back():
    table = np.array([[4, 5], [6, 7]], dtype=np.int32)
    free = np.array([1, 2, 3, 9], dtype=np.int32)
    want = run_and_compare(np.array([3, 4], np.int32), np.array([-1, -1], np.int32), 2, table, free, 1, 3)
    assert want["info"] == [3, 0, 0, 4]


def test_lifecycle_in_a_graph():
    """One captured step replayed with changing `added`, all state in place: pages are never lost, doubled or shared."""
    import torch
    import paper_2601_16032_b200 as sa
    dev, B, page, width, pages, cap = "cuda:0", 6, 4, 8, 30, 40
    rng = np.random.default_rng(3)
    length, added = torch.zeros(B, dtype=torch.int32, device=dev), torch.zeros(B, dtype=torch.int32, device=dev)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    free, count = torch.arange(pages, dtype=torch.int32, device=dev), torch.tensor([pages], dtype=torch.int32, device=dev)
    step = lambda: sa.page_plan(length, added, page, table, free, count, cap, seq_len=length, free_count_out=count)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p = step()
    state = dict(table=table.cpu().numpy(), free=free.cpu().numpy(), count=pages, seq_len=[0] * B)
    for turn in range(60):
        a = rng.integers(-1, 7, B).astype(np.int32)
        added.copy_(torch.from_numpy(a))
        graph.replay()
        torch.cuda.synchronize()
        state = paged.page_plan(state["seq_len"], a, page, state["table"], state["free"], state["count"], pages, cap)
        assert p.info.tolist() == state["info"] and length.tolist() == [int(x) for x in state["seq_len"]]
        assert int(count) == state["count"] and p.slot.tolist() == state["slot"]
        lengths, n = length.tolist(), int(count)
        held = [int(x) for b in range(B) for x in table[b, :paged.pages_of(lengths[b], page)]] + free[:n].tolist()
        assert sorted(held) == list(range(pages))
