"""How a paged decode is dealt out, replayed on the host: every tile once, equal shares, and parts that the join can find."""
import random

import pytest

import paper_2601_16032_b200 as sa


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    from conftest import nvcc_available
    if not nvcc_available() and not os.path.exists(sa.library_path()):
        pytest.skip("the C-ABI library is not built and there is no nvcc to build it with")


def check(lengths, H, kv_heads, d, max_ctas=0, sm_count=148):
    o = sa.DecodeOpts()
    o.max_ctas = max_ctas
    plan = sa.attn_decode_query_plan(len(lengths), H, kv_heads, d, 0, o, sm_count)
    assert plan.cluster == 0
    group = H // kv_heads
    assert plan.head_blocks == -(-group // 32) and plan.grid <= (max_ctas or 3 * sm_count)
    assert plan.workspace_bytes >= plan.grid * 2 * min(group, 32) * (d + 2) * 4
    trace = sa.attn_decode_trace(lengths, H, kv_heads, d, o, sm_count)
    tiles = [-(-n // plan.tile_tokens) for n in lengths]
    total = sum(tiles) * kv_heads * plan.head_blocks
    seen, load, parts, order = {}, {}, {}, []
    for e in trace:
        assert 0 <= e.cta < plan.grid and e.tile_begin < e.tile_end <= e.n_tiles == tiles[e.request]
        key = (e.request, e.kv_head, e.head_block)
        seen.setdefault(key, []).append(e)
        load[e.cta] = load.get(e.cta, 0) + e.tile_end - e.tile_begin
        order.append((e.cta, key, e.tile_begin))
        whole = e.tile_begin == 0 and e.tile_end == e.n_tiles
        assert (e.part == -1) == whole and e.part < 2 * plan.grid
        if not whole:
            assert e.part not in parts
            parts[e.part] = e
    assert order == sorted(order)
    assert set(seen) == {(b, h, k) for b, n in enumerate(tiles) if n for h in range(kv_heads) for k in range(plan.head_blocks)}
    for key, pieces in seen.items():
        assert [p.tile_begin for p in pieces] == [0] + [p.tile_end for p in pieces[:-1]] and pieces[-1].tile_end == tiles[key[0]]
        assert [p.cta for p in pieces] == list(range(pieces[0].first_cta, pieces[0].last_cta + 1))
        assert len({(p.first_cta, p.last_cta) for p in pieces}) == 1
        if len(pieces) > 1:     # where the join looks: 2 c + 1 of the first CTA, 2 c of the others
            assert [p.part for p in pieces] == [2 * pieces[0].cta + 1] + [2 * p.cta for p in pieces[1:]]
    assert len({p[0].cta for p in seen.values() if len(p) > 1}) == sum(len(p) > 1 for p in seen.values())    # one join a CTA at most
    if total:
        assert max(load.values()) - min(load.values()) <= 1 and sum(load.values()) == total
        assert min(load.values()) >= min(total, plan.min_tiles) - 1 or len(load) == 1
    else:
        assert trace == []


@pytest.mark.parametrize("lengths,H,kv_heads", [
    ([1], 1, 1), ([0], 4, 2), ([0, 0, 5, 0], 4, 2), ([64], 8, 8), ([65, 63, 1], 32, 8), ([1000], 32, 8), ([131072], 32, 8), ([131072], 40, 1),
    ([1 << 24] * 3, 16, 16), ([2**31 - 1, 7], 16, 2), ([700] * 200, 32, 1), (list(range(0, 300, 7)), 7, 7)])
def test_shares(lengths, H, kv_heads):
    if sum(lengths) < 1 << 28:
        for max_ctas in (0, 1, 2, 5, 1000):
            check(lengths, H, kv_heads, 128, max_ctas)
    check(lengths, H, kv_heads, 64)


def test_random_shares():
    rng = random.Random(7)
    for _ in range(300):
        B, kv_heads = rng.randint(1, 40), rng.choice([1, 2, 3, 8])
        longest = rng.choice([3, 100, 1000, 20000])
        check([rng.choice([0, rng.randint(0, longest)]) for _ in range(B)], kv_heads * rng.choice([1, 2, 7, 16, 17, 40]), kv_heads, rng.choice([64, 128]),
              rng.choice([0, 0, 1, 3, 17]), rng.choice([148, 148, 1, 7]))


def test_plan_refusals():
    for args, status in (((0, 4, 2, 128), -1), ((1, 4, 3, 128), -1), ((1, 0, 1, 128), -1), ((1, 4, 2, 96), -2), ((1 << 20, 65536, 1, 128), -1)):
        with pytest.raises(sa.AttnError) as e:
            sa.attn_decode_query_plan(*args, sm_count=148)
        assert e.value.status == status
    with pytest.raises(sa.AttnError):
        sa.attn_decode_trace([-1], 4, 2, 128, sm_count=148)


def test_clusters_for_short_requests():
    """All CTAs fit on the GPU at a time, no CTA has more than a handful of tiles, and a cluster is no larger than there are tiles for."""
    plan = lambda B, kv_heads, d, tokens, **o: sa.attn_decode_query_plan(B, 4 * kv_heads, kv_heads, d, tokens, sa.DecodeOpts(**o), 148)  # noqa: E731
    assert plan(1, 8, 128, 1008).cluster == 8 and plan(1, 8, 128, 131072).cluster == 0 and plan(64, 8, 128, 1008).cluster == 0
    assert plan(1, 8, 128, 64).cluster == 1 and plan(1, 8, 128, 65).cluster == 2 and plan(1, 8, 128, 0).cluster == 0
    assert plan(1, 8, 128, 1008, max_ctas=63).cluster == 4 and plan(1, 8, 128, 1008, max_ctas=7).cluster == 0 and plan(112, 8, 128, 60).cluster == 0 and plan(111, 8, 128, 60).cluster == 1
    for B in (1, 2, 7, 30, 100, 444, 445, 3000):
        for kv_heads in (1, 3, 8):
            for d in (64, 128):
                for tokens in (1, 64, 128, 129, 700, 2048, 2049, 4096, 5000, 1 << 40):
                    p = plan(B, kv_heads, d, tokens)
                    if p.cluster:
                        tiles = -(-tokens // p.tile_tokens)
                        assert p.cluster in (1, 2, 4, 8) and -(-tiles // p.cluster) <= 6
                        assert B * kv_heads * p.cluster <= p.grid or (p.cluster == 1 and B * kv_heads <= 2 * p.grid)
    with pytest.raises(sa.AttnError):
        plan(1, 1, 128, -1)
