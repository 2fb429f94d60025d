"""GPU: attention of one new token over the paged cache, against the 64-bit statement.

Tolerances.  The result is rounded once: half a step of the type.  Before that, with S = scale * sum |q_i k_i| the largest of the
request's tokens: a score is off by at most (d / 16 + 16) 2^-23 S (16 products an instruction, d / 16 instructions, sums cut at 2^-23), a probability by
that twice (numerator and denominator), 2^-22 of 2^x twice and |score| 2^-23 twice, its split into two numbers leaves 2^-18, and sums over n tokens are made of n / 64 + 32
terms a thread: c = 2 (d / 16 + 16 + 1) 2^-23 S + 2^-17 + (n / 64 + 32) 2^-23 of sum p |v| / sum p.  The logarithm of the sum is off by the score's error, the sums' and its own
(2^-22 of itself).
"""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def kinds(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def f64(t):
    return t.detach().double().cpu().numpy()


def make(lengths, H, Hk, d, page, heads_first, kind, seed, spare=3, width=None, spoil=True):
    """q, K, V, table and lengths; what no request may see is NaN, and table entries behind a request's pages point nowhere."""
    import torch
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    held = [paged.pages_of(n, page) for n in lengths]
    pages = sum(held) + spare
    names = rng.permutation(pages)
    table = np.full((len(lengths), width or max(1, max(held))), 2**31 - 1, dtype=np.int32)
    table[:, ::2] = -7
    at = 0
    kv = torch.randn((2, pages, page, Hk, d), generator=g, device=DEV)
    if spoil:
        seen = torch.zeros((pages, page), dtype=torch.bool)
        for b, n in enumerate(lengths):
            table[b, :held[b]] = names[at:at + held[b]]
            for i in range(held[b]):
                seen[int(names[at + i]), :min(page, n - i * page)] = True
            at += held[b]
        kv[:, ~seen.to(DEV)] = float("nan")
        kv[0, ~seen.to(DEV)] = float("inf")
    kv = kv.to(kind)
    if heads_first:
        kv = kv.transpose(2, 3).contiguous()
    q = torch.randn((len(lengths), H, d), generator=g, device=DEV).to(kind)
    return q, kv[0], kv[1], torch.from_numpy(table).to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV)


def check(o, lse, q, k, v, table, lengths, page, heads_first, scale, kind, requests=None):
    import torch
    K, V, Q, T = f64(k), f64(v), f64(q), table.cpu().numpy()
    got, got_lse = f64(o), f64(lse)
    B, H, d = Q.shape
    for b in requests if requests is not None else range(B):
        n = int(lengths[b])
        keys, values = (paged.gather(c, T[b], n, page, heads_first) for c in (K, V))
        want, want_lse = paged.decode(Q[b], keys, values, scale)
        if n == 0:
            assert (got[b] == 0).all() and np.isneginf(got_lse[b]).all()
            continue
        group = H // keys.shape[1]
        for h in range(H):
            kk, vv = keys[:, h // group], values[:, h // group]
            s = scale * (kk @ Q[b, h])
            size = float((np.abs(kk) @ np.abs(Q[b, h])).max() * abs(scale))
            p = np.exp(s - s.max())
            spread = p @ np.abs(vv) / p.sum()
            c = 2 * (d / 16 + 17) * 2.0 ** -23 * size + 2.0 ** -17 + (n / 64 + 32) * 2.0 ** -23
            half = torch.finfo(kind).eps / 2 * np.abs(want[h]) + (2.0 ** -25 if kind == torch.float16 else 0)
            err = np.abs(got[b, h] - want[h])
            assert (err <= half * (1 + 1e-6) + c * spread).all(), (b, h, n, float((err / (half + c * spread)).max()))
            assert abs(got_lse[b, h] - want_lse[h]) <= c + abs(want_lse[h]) * 2.0 ** -22, (b, h, n)


EDGES = [1, 0, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 300, 1000]
HEADS = [(1, 1), (5, 1), (8, 2), (6, 3), (16, 1), (17, 1), (40, 1), (8, 8)]


@pytest.mark.parametrize("H,Hk", HEADS)
@pytest.mark.parametrize("d,kind", [(128, "bf16"), (64, "f16"), (64, "bf16"), (128, "f16")])
def test_lengths_around_the_tiles(H, Hk, d, kind):
    import paper_2601_16032_b200 as sa
    kind = kinds(kind)
    for page, heads_first, max_ctas in ((16, False, 0), (1, True, 3), (24, False, 1), (128, True, 7), (64, False, 40)):
        q, k, v, table, lengths = make(EDGES, H, Hk, d, page, heads_first, kind, H * 100 + page)
        layout = sa.LAYOUT_BHND if heads_first else sa.LAYOUT_BNHD
        o, lse = sa.decode_paged(q, k, v, table, lengths, cache_layout=layout, return_lse=True, max_ctas=max_ctas)
        sa.attn_device_status()
        check(o, lse, q, k, v, table, lengths, page, heads_first, d ** -0.5, kind)


@pytest.mark.parametrize("length", [1, 2, 64, 4097, 20000])
@pytest.mark.parametrize("H,Hk,d,kind", [(4, 1, 128, "bf16"), (2, 2, 64, "f16")])
def test_one_request_split_over_the_gpu(length, H, Hk, d, kind):
    import torch
    import paper_2601_16032_b200 as sa
    kind = kinds(kind)
    q, k, v, table, lengths = make([length], H, Hk, d, 16, False, kind, length)
    o, lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    sa.attn_device_status()
    check(o, lse, q, k, v, table, lengths, 16, False, d ** -0.5, kind)
    again, _ = sa.decode_paged(q, k, v, table, lengths)
    assert torch.equal(o, again)


def test_many_requests():
    import paper_2601_16032_b200 as sa
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 40, 700).tolist()
    q, k, v, table, lengths = make(lens, 4, 2, 64, 8, False, kinds("bf16"), 11)
    o, lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    sa.attn_device_status()
    check(o, lse, q, k, v, table, lengths, 8, False, 0.125, kinds("bf16"))


@pytest.mark.parametrize("scale", [0.0, -0.09, 3.0])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_scales_that_spread_or_level_the_scores(scale, kind):
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([200, 3, 2500], 4, 1, 128, 16, False, kinds(kind), 21)
    o, lse = sa.decode_paged(q, k, v, table, lengths, scale=scale, return_lse=True)
    sa.attn_device_status()
    check(o, lse, q, k, v, table, lengths, 16, False, scale, kinds(kind))


def test_invariants():
    """Values of one give one; a dominant key gives its value; the order of the pages does not matter to more than rounding."""
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([500, 77], 8, 2, 128, 16, False, torch.float16, 5)
    o, _ = sa.decode_paged(q, k, torch.ones_like(v), table, lengths)
    assert (o == 1).all()
    k[table[0, 7], 3] = 0
    k[table[0, 7], 3, :, 0] = 100
    q[0, :, 0] = 60
    o, lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    assert torch.equal(o[0].view(2, 4, 128), v[table[0, 7], 3][:, None].expand(2, 4, 128))


def test_special_values_inside_the_length():
    """A score of -infinity takes no part; NaN and +infinity give NaN, in their head only."""
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([300, 300, 300], 4, 4, 64, 16, False, torch.bfloat16, 6)
    clean, clean_lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    q[:, :, 0] = 1
    k[:, :, :, 0] = 0
    base, base_lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    k2, v2 = k.clone(), v.clone()
    k2[table[0, 2], 5, 1, 0] = -float("inf")
    k2[table[1, 3], 0, 2, 0] = float("nan")
    k2[table[2, 0], 9, 3, 0] = float("inf")
    o, lse = sa.decode_paged(q, k2, v2, table, lengths, return_lse=True)
    touched = torch.zeros(3, 4, dtype=torch.bool, device=DEV)
    touched[0, 1] = touched[1, 2] = touched[2, 3] = True
    assert torch.equal(o[~touched], base[~touched]) and torch.equal(lse[~touched], base_lse[~touched])
    assert torch.isfinite(o[0, 1]).all() and o[1, 2].isnan().all() and o[2, 3].isnan().all()
    keep = torch.arange(300) != 2 * 16 + 5
    keys, values = (f64(c[table[0, :19].long()].reshape(-1, 4, 64)[:300][keep.to(DEV)]) for c in (k, v))
    want, want_lse = paged.decode(f64(q[0]), keys, values, 0.125)
    assert np.abs(f64(o[0, 1]) - want[1]).max() <= 2.0 ** -8 * np.abs(want[1]).max() and abs(float(lse[0, 1]) - want_lse[1]) < 1e-4
    k2 = torch.full_like(k, 0)
    k2[..., 0] = -float("inf")                      # nothing left: 0 / 0, as in the definition
    o, lse = sa.decode_paged(q, k2, v, table, lengths, return_lse=True)
    assert o.isnan().all() and torch.isneginf(lse).all()


def test_strided_queries_outputs_and_caches():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([100, 0, 33], 6, 2, 64, 16, False, torch.float16, 8)
    want, want_lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    wide = torch.zeros((3, 10, 72), dtype=torch.float16, device=DEV)
    q2 = wide[:, 2:8, 8:]
    q2.copy_(q)
    pool = torch.full((k.shape[0], 16, 2, 2, 80), float("nan"), dtype=torch.float16, device=DEV)   # K and V of a token side by side
    pool[:, :, 0, :, :64], pool[:, :, 1, :, :64] = k, v
    out = torch.full((3, 6, 2, 64), 5.0, dtype=torch.float16, device=DEV)
    big_table = torch.full((3, 50), -1, dtype=torch.int32, device=DEV)
    big_table[:, 10:10 + table.shape[1]] = table
    o, lse = sa.decode_paged(q2, pool[:, :, 0, :, :64], pool[:, :, 1, :, :64], big_table[:, 10:10 + table.shape[1]], lengths, out=out[:, :, 1], return_lse=True)
    sa.attn_device_status()
    assert torch.equal(o, want) and torch.equal(lse, want_lse) and (out[:, :, 0] == 5).all()


def test_pages_beyond_32_bit_offsets():
    import torch
    import paper_2601_16032_b200 as sa
    page, d, far = 16, 128, 5
    stride = (1 << 29) + 4096                       # elements between pages: the last one starts beyond 2^31
    buf = torch.empty(2, far * stride, dtype=torch.bfloat16, device=DEV)
    k, v = (buf[i].as_strided((far, page, 2, d), (stride, 2 * d, d, 1)) for i in (0, 1))
    small = torch.randn((2, far, page, 2, d), device=DEV).bfloat16()
    k.copy_(small[0])
    v.copy_(small[1])
    table = torch.tensor([[4, 0, 3], [2, 1, 4]], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([40, 48], dtype=torch.int32, device=DEV)
    q = torch.randn((2, 4, d), device=DEV).bfloat16()
    o, _ = sa.decode_paged(q, k, v, table, lengths)
    want, _ = sa.decode_paged(q, small[0], small[1], table, lengths)
    assert torch.equal(o, want)
    # and the append writes there
    slot = torch.tensor([4 * page + 15, 3], device=DEV)
    new = torch.randn((2, 2, d), device=DEV).bfloat16()
    sa.qk_norm_rope(q, new, new, k_cache=k, v_cache=v, slot=slot)
    assert torch.equal(k[4, 15], new[0]) and torch.equal(v[0, 3], new[1])


@pytest.mark.parametrize("page_number", [-1, 12345, 2**31 - 1, -2**31])
def test_a_bad_page_number_reads_as_zeros_and_is_reported(page_number):
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([100, 90], 4, 2, 64, 16, False, torch.bfloat16, 9)
    want, _ = sa.decode_paged(q, k, v, table, lengths)
    sa.attn_device_status()
    table[0, 3] = page_number
    o, _ = sa.decode_paged(q, k, v, table, lengths)
    with pytest.raises(sa.AttnError) as e:
        sa.attn_device_status()
    assert e.value.status == -7 and torch.equal(o[1], want[1]) and torch.isfinite(o[0]).all()
    sa.attn_device_status()


def test_lengths_out_of_range_are_cut_and_reported():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([96, 90, 96], 4, 2, 64, 16, False, torch.bfloat16, 10)
    want, want_lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    lengths[0], lengths[2] = 2**31 - 1, -5
    o, lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    with pytest.raises(sa.AttnError) as e:
        sa.attn_device_status()
    assert e.value.status == -7
    assert torch.equal(o[:2], want[:2]) and (o[2] == 0).all() and torch.isneginf(lse[2]).all()


def test_the_longest_length():
    """2^31 - 1 tokens, cut to the most there can be: one page again and again, so the result is that of the page alone."""
    import math

    import torch
    import paper_2601_16032_b200 as sa
    page, d = 65536, 64
    k, v = (torch.randn((1, page, 1, d), device=DEV).bfloat16() for _ in range(2))
    q = torch.randn((1, 2, d), device=DEV).bfloat16()
    table = torch.zeros((1, 32768), dtype=torch.int32, device=DEV)
    lengths = torch.tensor([page], dtype=torch.int32, device=DEV)
    want, want_lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    sa.attn_device_status()
    lengths.fill_(2**31 - 1)
    o, lse = sa.decode_paged(q, k, v, table, lengths, return_lse=True)
    with pytest.raises(sa.AttnError) as e:
        sa.attn_device_status()
    assert e.value.status == -7
    # a thread's sums have 2^31 / (444 * 4 * 8) terms, each addition off by 2^-24 of the sum: 2^-6.7 at most
    assert (lse - want_lse - math.log(32768)).abs().max() <= 1e-2
    assert (o.float() - want.float()).abs().max() <= 1e-2 * v.float().abs().max()


def test_workspace_contents_do_not_matter_and_its_end_is_kept():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([3000, 1, 700], 8, 2, 128, 16, False, torch.bfloat16, 12)
    want, _ = sa.decode_paged(q, k, v, table, lengths)
    n = sa.attn_decode_query_plan(3, 8, 2, 128).workspace_bytes
    for fill in (0, 0xff, 0x7f):
        ws = torch.full((n + 256,), fill, dtype=torch.uint8, device=DEV)
        o, _ = sa.decode_paged(q, k, v, table, lengths, workspace=ws[:n])
        assert torch.equal(o, want) and (ws[n:] == fill).all()
    with pytest.raises(sa.AttnError):
        sa.decode_paged(q, k, v, table, lengths, workspace=ws[:n - 16])


def test_captured_with_lengths_that_change():
    import torch
    import paper_2601_16032_b200 as sa
    full = [2000, 700, 64, 1]
    q, k, v, table, lengths = make(full, 8, 2, 128, 16, False, torch.bfloat16, 13)
    ws = torch.empty(sa.attn_decode_query_plan(4, 8, 2, 128).workspace_bytes, dtype=torch.uint8, device=DEV)
    call = lambda: sa.decode_paged(q, k, v, table, lengths, return_lse=True, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = call()
    for lens in ([1, 0, 0, 0], [0, 0, 0, 0], [2000, 700, 64, 1], [1999, 650, 63, 0], [64, 64, 64, 1]):
        lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = call()
        assert torch.equal(o, want) and torch.equal(lse, want_lse)
        check(o, lse, q, k, v, table, lengths, 16, False, 128 ** -0.5, torch.bfloat16)


def test_two_streams_at_once_with_a_workspace_each():
    import torch
    import paper_2601_16032_b200 as sa
    cases = [make([5000, 300], 8, 2, 128, 16, False, torch.bfloat16, s) for s in (14, 15)]
    want = [sa.decode_paged(*c)[0] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(sa.decode_paged(*c)[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_wrapper_refuses():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, table, lengths = make([40, 50], 4, 2, 64, 16, False, torch.bfloat16, 16)
    for change in (dict(q=q.float()), dict(q=q.half()), dict(q=q[..., ::2]), dict(k=k[:, :, :1]), dict(v=v.half()), dict(table=table.long()), dict(table=table[:1]),
                   dict(lengths=lengths.long()), dict(lengths=lengths[:1]), dict(q=q.cpu()), dict(q=q[0]), dict(k=k.transpose(0, 1), v=v),
                   dict(q=q[:, :3].contiguous()), dict(k=k[:1].expand_as(k), v=v[:1].expand_as(v), bad=False)):
        a = dict(q=q, k=k, v=v, table=table, lengths=lengths)
        a.update({n: x for n, x in change.items() if n != "bad"})
        if change.get("bad", True):
            with pytest.raises(sa.AttnError):
                sa.decode_paged(a["q"], a["k"], a["v"], a["table"], a["lengths"])
        else:       # pages that share memory may be read
            sa.decode_paged(a["q"], a["k"], a["v"], a["table"], a["lengths"])
    sa.attn_device_status()
    cache = sa.KVCache(k.data_ptr(), v.data_ptr(), k.shape[0], 0, 0, 0, 16, 2, 64, sa.BF16, sa.LAYOUT_BNHD)
    ws = torch.empty(1 << 25, dtype=torch.uint8, device=DEV)
    with pytest.raises(sa.AttnError) as e:          # more tiles than the kernel counts: refused before anything is launched
        sa.attn_decode_paged(q.data_ptr(), cache, table.data_ptr(), 0, 2**31 - 1, lengths.data_ptr(), ws.data_ptr() + (1 << 24), 1 << 25, 4, 0.1,
                             ws.data_ptr(), 1 << 24, torch.cuda.current_stream().cuda_stream)
    assert e.value.status == -1 and "more work" in str(e.value)
    empty, lse = sa.decode_paged(q[:0], k, v, table[:0], lengths[:0], return_lse=True)
    assert empty.shape == (0, 4, 64) and lse.shape == (0, 4)
