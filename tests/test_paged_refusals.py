"""What the entry points around the paged cache refuse, without a device: every check comes before the first use of one."""
import ctypes

import pytest

import paper_2601_16032_b200 as sa

P = 1 << 20      # stands for device addresses, never read on the host


def at(i):
    return P + (i << 30)


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    from conftest import nvcc_available
    if not nvcc_available() and not os.path.exists(sa.library_path()):
        pytest.skip("the C-ABI library is not built and there is no nvcc to build it with")


def refused(call, status=-1):
    with pytest.raises(sa.AttnError) as e:
        call()
    assert e.value.status == status, str(e.value)
    return str(e.value)


def plan_call(**change):
    a = dict(table=at(0), stride=10, free=at(1), count=at(2), count_out=at(3), width=10, capacity=100, page=16, cached=at(4), added=at(5), B=4,
             seq_len=at(6), q_start=at(7), slot=at(8), position=at(9), request=at(10), cap=20, info=at(11))
    a.update(change)
    pool = sa.PagePool(a["table"], a["stride"], a["free"], a["count"], a["count_out"], a["width"], a["capacity"], a["page"])
    return lambda: sa.attn_page_plan(pool, a["cached"], a["added"], a["B"], a["seq_len"], a["q_start"], a["slot"], a["position"], a["request"], a["cap"], a["info"])


@pytest.mark.parametrize("change,status", [
    (dict(table=0), -1), (dict(free=0), -1), (dict(count=0), -1), (dict(count_out=0), -1), (dict(cached=0), -1), (dict(added=0), -1), (dict(seq_len=0), -1),
    (dict(q_start=0), -1), (dict(slot=0), -1), (dict(info=0), -1), (dict(B=0), -1), (dict(B=8193), -1), (dict(cap=-1), -1), (dict(page=0), -1),
    (dict(page=65537), -1), (dict(width=0), -1), (dict(capacity=-1), -1), (dict(stride=9), -1), (dict(stride=1 << 60), -1), (dict(width=1 << 28, stride=1 << 28), -1),
    (dict(cached=at(4) + 2), -3), (dict(slot=at(8) + 4), -3), (dict(position=at(9) + 1), -3),
    (dict(seq_len=at(4) + 4), -1), (dict(seq_len=at(5)), -1), (dict(position=at(10)), -1), (dict(info=at(1) + 4), -1), (dict(count_out=at(0) + 4 * 39), -1),
    (dict(slot=at(0)), -1), (dict(q_start=at(2) - 16), -1)])
def test_page_plan(change, status):
    refused(plan_call(**change), status)


def rope_call(backward=False, opts=None, cache=None, **change):
    a = dict(q=at(0), k=at(1), v=0, q_out=at(3), k_out=at(4), T=10, H=4, Hk=2, d=128, dtype=sa.BF16, wq=at(5), wk=at(6), eps=1e-6, position=at(7),
             freq=at(8), rot=128, style=0, dq=at(9), dk=at(10), dwq=at(11), dwk=at(12), ws=at(13), ws_bytes=1 << 22)
    a.update(change)
    o = sa.RopeOpts()
    for name, value in (opts or {}).items():
        setattr(o, name, value)
    if cache is not None:
        c = dict(k=at(14), v=at(15), num_pages=100, page_size=16, kv_heads=2, d=128, dtype=sa.BF16)
        c.update(cache)
        desc = sa.KVCache(**c)
        o.cache = ctypes.pointer(desc)
    if backward:
        return lambda: sa.attn_qk_norm_rope_bwd(a["q_out"], a["k_out"], a["q"], a["k"], a["dq"], a["dk"], a["dwq"], a["dwk"], a["T"], a["H"], a["Hk"], a["d"],
                                                a["dtype"], a["wq"], a["wk"], a["eps"], a["position"], a["freq"], a["rot"], a["style"], a["ws"], a["ws_bytes"], 0, o)
    return lambda: sa.attn_qk_norm_rope(a["q"], a["k"], a["v"], a["q_out"], a["k_out"], a["T"], a["H"], a["Hk"], a["d"], a["dtype"], a["wq"], a["wk"], a["eps"],
                                        a["position"], a["freq"], a["rot"], a["style"], 0, o)


COMMON = [
    (dict(q=0), -1), (dict(k=0), -1), (dict(q_out=0), -1), (dict(T=-1), -1), (dict(H=0), -1), (dict(Hk=0), -1), (dict(d=96), -2), (dict(dtype=2), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(rot=8), -1), (dict(rot=144), -1), (dict(rot=-16), -1),
    (dict(style=2), -1), (dict(position=0), -1), (dict(freq=0), -1), (dict(freq=at(8) + 4), -3), (dict(wq=at(5) + 2), -3), (dict(q=at(0) + 8), -3),
    (dict(opts=dict(q_token=4)), -1), (dict(opts=dict(q_token=-8)), -1), (dict(opts=dict(q_token=1 << 60)), -1), (dict(opts=dict(k_token=1 << 31, k_head=128)), -1), (dict(opts=dict(q_token=128, q_head=1 << 28)), -1), (dict(opts=dict(weight_f32=2)), -1),
    (dict(opts=dict(check_mode=3)), -1)]


@pytest.mark.parametrize("change,status", COMMON + [
    (dict(k_out=0), -1), (dict(v=at(2)), -1), (dict(opts=dict(slot=at(16))), -1), (dict(v=at(2), opts=dict(slot=at(16))), -1),
    (dict(q_out=at(0) + 256), -1), (dict(q_out=at(1)), -1), (dict(k_out=at(0)), -1), (dict(k_out=at(3) + 1024), -1),
    (dict(opts=dict(q_out_token=512, q_out_head=64)), -1), (dict(opts=dict(q_out_token=256, q_out_head=128)), -1)])
def test_rope_forward(change, status):
    refused(rope_call(**change), status)


@pytest.mark.parametrize("cache,more,status", [
    (dict(k=0), {}, -1), (dict(v=at(14)), {}, -1), (dict(num_pages=0), {}, -1), (dict(page_size=0), {}, -1), (dict(page_size=65537), {}, -1),
    (dict(kv_heads=4), {}, -1), (dict(d=64), {}, -1), (dict(dtype=sa.F16), {}, -1), (dict(layout=2), {}, -1), (dict(k=at(14) + 2), {}, -3),
    (dict(page_stride=4096, token_stride=256, head_stride=100), {}, -1), (dict(page_stride=4096, token_stride=128, head_stride=128), {}, -1),
    (dict(page_stride=2048, token_stride=256, head_stride=128), {}, -1), (dict(page_stride=-4096, token_stride=256, head_stride=128), {}, -1),
    (dict(page_stride=1 << 54, token_stride=256, head_stride=128), {}, -1), (dict(page_stride=1 << 30, token_stride=128, head_stride=1 << 28), {}, -1), ({}, dict(v=0), -1), ({}, dict(slot=0), -1), ({}, dict(slot=at(16) + 4), -3),
    (dict(k=at(3)), {}, -1), (dict(v=at(0)), {}, -1)])
def test_rope_cache(cache, more, status):
    refused(rope_call(cache=cache, v=more.get("v", at(2)), opts=dict(slot=more.get("slot", at(16)))), status)


@pytest.mark.parametrize("change,status", COMMON + [
    (dict(dq=0), -1), (dict(dk=0), -1), (dict(dwq=0), -1), (dict(wk=0), -1), (dict(dwk=at(12) + 2), -3), (dict(ws=0), -1), (dict(ws_bytes=1000), -1),
    (dict(ws=at(13) + 4), -3), (dict(dq=at(0)), -1), (dict(dk=at(1)), -1), (dict(dq=at(4)), -1), (dict(dk=at(9)), -1), (dict(ws=at(9)), -1),
    (dict(opts=dict(slot=at(16))), -1), (dict(k_out=0), -1)])
def test_rope_backward(change, status):
    refused(rope_call(backward=True, **change), status)


def decode_call(cache=None, opts=None, **change):
    a = dict(q=at(0), table=at(1), stride=64, pages=64, lens=at(2), o=at(3), B=4, H=8, scale=0.1, ws=at(4), ws_bytes=1 << 26)
    a.update(change)
    c = dict(k=at(14), v=at(15), num_pages=100, page_size=16, kv_heads=2, d=128, dtype=sa.BF16)
    c.update(cache or {})
    o = sa.DecodeOpts()
    for name, value in (opts or {}).items():
        setattr(o, name, value)
    return lambda: sa.attn_decode_paged(a["q"], sa.KVCache(**c), a["table"], a["stride"], a["pages"], a["lens"], a["o"], a["B"], a["H"], a["scale"], a["ws"],
                                        a["ws_bytes"], 0, o)


@pytest.mark.parametrize("change,status", [
    (dict(q=0), -1), (dict(table=0), -1), (dict(lens=0), -1), (dict(o=0), -1), (dict(ws=0), -1), (dict(ws=at(4) + 8), -3), (dict(B=0), -1), (dict(H=7), -1),
    (dict(H=0), -1), (dict(pages=0), -1), (dict(stride=-1), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(scale=3e38), -1), (dict(q=at(0) + 4), -3),
    (dict(lens=at(2) + 2), -3), (dict(opts=dict(lse=at(5) + 2)), -3), (dict(opts=dict(max_ctas=-1)), -1), (dict(opts=dict(check_mode=2)), -1),
    (dict(opts=dict(q_head=4)), -1), (dict(opts=dict(o_request=64, o_head=128)), -1), (dict(cache=dict(d=80)), -2), (dict(cache=dict(k=0)), -1),
    (dict(cache=dict(v=at(14))), -1), (dict(cache=dict(page_size=0)), -1), (dict(cache=dict(kv_heads=3)), -1), (dict(cache=dict(dtype=4)), -1),
    (dict(cache=dict(k=at(14) + 8)), -3), (dict(cache=dict(page_stride=4, token_stride=8, head_stride=8)), -1)])
def test_decode(change, status):
    refused(decode_call(**change), status)


def test_queries_and_keys_may_lie_side_by_side():
    """Interleaved parts of one array do not overlap: the call gets as far as looking for a device."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses stand for nothing")
    row = 8 * 128
    call = rope_call(q=at(0), k=at(0) + 2 * 4 * 128, q_out=at(0), k_out=at(0) + 2 * 4 * 128, opts=dict(
        q_token=row, q_head=128, k_token=row, k_head=128, q_out_token=row, q_out_head=128, k_out_token=row, k_out_head=128))
    refused(call, -4)
    refused(rope_call(), -4)
    refused(rope_call(backward=True), -4)
    refused(rope_call(cache={}, v=at(2), opts=dict(slot=at(16))), -4)
    refused(plan_call(seq_len=at(4), count_out=at(2), position=0, request=0), -4)
    refused(decode_call(), -4)


def test_status_of_an_index_out_of_range_has_a_text():
    assert "out of range" in sa.attn_status_string(-7)
