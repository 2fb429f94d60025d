"""GPU: head norm, position rotation and cache append, and their gradients, against the 64-bit statement.

Tolerances.  An output is rounded once: half a step, eps / 2 of its value, or half the smallest fp16 subnormal (2^-25).  Before that
everything is 32-bit: the mean of squares (8 terms in a lane, 4 shuffle steps, relative error at most 12 * 2^-24, halved by
the root), rsqrtf (2^-22), two products, the angle (pi * 2^-24 for the rounding of the part of a turn), the sine and cosine
(2^-22), and a two-term sum of |a| + |b|: below 2^-20 of |a| + |b| together.  2^-19 is allowed.  Gradients pass through the same
chain with one more mean: 2^-18 of the terms' sizes.  A weight's gradient is a 32-bit sum of N terms added up in a tree whose longest chain is
a thread's rows, then 32, 32 and 32: with up to 60 rows a thread under 160 * 2^-24 < 2^-16 of the sum of the terms' sizes.
"""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def kinds(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def half_step(kind, y):
    import torch
    return torch.finfo(kind).eps / 2 * np.abs(y) + (2.0 ** -25 if kind == torch.float16 else 0)


def f64(t):
    return t.detach().double().cpu().numpy()


def parts(x, inv_freq, adjacent):
    """|a| + |b| of the pair each element belongs to (|x| where nothing turns)."""
    size = np.abs(x)
    if inv_freq is not None and len(inv_freq):
        a, b = paged._pair_index(2 * len(inv_freq), adjacent)
        s = size[..., a] + size[..., b]
        size[..., a] = size[..., b] = s
    return size


def make(T, H, Hk, d, kind, rot, far, seed, weight_kind=None):
    import torch
    g = torch.Generator(device=DEV).manual_seed(seed)
    qkv = torch.randn((T, H + 2 * Hk, d), generator=g, device=DEV, dtype=torch.float32).to(kind)
    w = [(1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(weight_kind or kind) for _ in range(2)]
    position = torch.randint(0, far, (T,), generator=g, device=DEV, dtype=torch.int32)
    freq = (1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).to(DEV) if rot else None
    return qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], w[0], w[1], position, freq


def check_forward(y, x, w, eps, position, freq, adjacent, kind):
    pos, fr = position.tolist(), None if freq is None else freq.tolist()
    want = paged.norm_rope(f64(x), None if w is None else f64(w), eps, pos, fr, adjacent)
    n = paged.norm_rope(f64(x), None if w is None else f64(w), eps, pos, None, adjacent)
    err = np.abs(f64(y) - want)
    assert (err <= half_step(kind, want) * (1 + 1e-6) + 2.0 ** -19 * parts(n, fr, adjacent)).all(), err.max()


SHAPES = [(1, 1, 1, 128), (1, 32, 8, 128), (3, 5, 1, 64), (7, 7, 7, 64), (65, 12, 4, 128), (301, 8, 2, 128), (1300, 4, 4, 64)]


@pytest.mark.parametrize("T,H,Hk,d", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_forward_into_dense_outputs(T, H, Hk, d, kind, adjacent):
    import paper_2601_16032_b200 as sa
    kind = kinds(kind)
    for rot in (d, d // 2, 16, 0):
        q, k, v, wq, wk, pos, freq = make(T, H, Hk, d, kind, rot, 1 << 20, T + rot)
        yq, yk = sa.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, eps=1e-6, position=pos, inv_freq=freq, interleaved=adjacent)
        sa.attn_device_status()
        check_forward(yq, q, wq, 1e-6, pos, freq, adjacent, kind)
        check_forward(yk, k, wk, 1e-6, pos, freq, adjacent, kind)


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("page", [1, 16, 24])
@pytest.mark.parametrize("d,kind", [(128, "bf16"), (64, "f16")])
def test_append_to_the_cache(heads_first, page, d, kind):
    """Padded rows (slot -1) are left alone, every other row of the cache keeps its bits, v arrives unchanged."""
    import torch
    import paper_2601_16032_b200 as sa
    kind, T, H, Hk, pages = kinds(kind), 150, 6, 3, 400 // page + 2
    q, k, v, wq, wk, pos, freq = make(T, H, Hk, d, kind, d, 5000, 77)
    shape = (pages, Hk, page, d) if heads_first else (pages, page, Hk, d)
    both = torch.randn((2,) + shape, device=DEV).to(kind)
    kc, vc = both[0], both[1]
    kc0, vc0 = kc.clone(), vc.clone()
    slot = torch.randperm(pages * page, device=DEV)[:T]
    slot[[0, 17, T - 1]] = -1
    q_out = torch.full((T, H, d), 7.0, dtype=kind, device=DEV)
    k_out = torch.full((T, Hk, d), 7.0, dtype=kind, device=DEV)
    layout = sa.LAYOUT_BHND if heads_first else sa.LAYOUT_BNHD
    for with_dense in (False, True):
        kc.copy_(kc0)
        vc.copy_(vc0)
        _, got = sa.qk_norm_rope(q, k, v, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq, k_cache=kc, v_cache=vc, cache_layout=layout, slot=slot,
                                 q_out=q_out, k_out=k_out if with_dense else None)
        sa.attn_device_status()
        assert (got is None) == (not with_dense)
        live = slot >= 0
        yq, yk = sa.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)
        assert torch.equal(q_out[live], yq[live]) and (q_out[~live] == 7).all()
        if with_dense:
            assert torch.equal(k_out[live], yk[live]) and (k_out[~live] == 7).all()
        for cache, before, rows in ((kc, kc0, yk), (vc, vc0, v)):
            want = before.clone()
            flat = want.transpose(1, 2) if heads_first else want
            flat[slot[live] // page, slot[live] % page] = rows[live]
            assert torch.equal(cache.view(torch.int16), want.view(torch.int16))


def test_slot_beyond_the_cache_is_not_written_and_is_reported():
    import torch
    import paper_2601_16032_b200 as sa
    kind = torch.bfloat16
    q, k, v, wq, wk, pos, freq = make(4, 2, 1, 64, kind, 64, 100, 5)
    buf = torch.zeros((2, 12, 4, 1, 64), dtype=kind, device=DEV)     # two guard pages at each end
    kc, vc = buf[0, 2:10], buf[1, 2:10]
    slot = torch.tensor([3, 32, 1 << 40, 31], device=DEV)
    sa.qk_norm_rope(q, k, v, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq, k_cache=kc, v_cache=vc, slot=slot)
    with pytest.raises(sa.AttnError) as e:
        sa.attn_device_status()
    assert e.value.status == -7
    sa.attn_device_status()
    written = (buf != 0).any(-1).any(-1).view(2, -1).nonzero()
    assert written.tolist() == [[i, 8 + s] for i in (0, 1) for s in (3, 31)]


def test_no_norm_one_norm_and_fp32_weights():
    import torch
    import paper_2601_16032_b200 as sa
    for wq_on, wk_on in ((False, False), (True, False), (False, True)):
        q, k, v, wq, wk, pos, freq = make(33, 3, 2, 128, torch.bfloat16, 64, 1000, 6, torch.float32)
        wq, wk = wq if wq_on else None, wk if wk_on else None
        yq, yk = sa.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, eps=1e-5, position=pos, inv_freq=freq)
        check_forward(yq, q, wq, 1e-5, pos, freq, False, torch.bfloat16)
        check_forward(yk, k, wk, 1e-5, pos, freq, False, torch.bfloat16)
        gq, gk = torch.randn_like(yq), torch.randn_like(yk)
        dq, dk, dwq, dwk = sa.qk_norm_rope_backward(gq, gk, q, k, q_weight=wq, k_weight=wk, eps=1e-5, position=pos, inv_freq=freq)
        assert (dwq is None) == (not wq_on) and (dwk is None) == (not wk_on)
        check_backward(dq, dwq, gq, q, wq, 1e-5, pos, freq, False, torch.bfloat16)
        check_backward(dk, dwk, gk, k, wk, 1e-5, pos, freq, False, torch.bfloat16)


def test_rows_that_are_special():
    """Zero rows, rows of one huge value, rows with NaN or infinity: each row's result is its own."""
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, wq, wk, pos, freq = make(64, 4, 4, 64, torch.bfloat16, 64, 1000, 8)
    q, k = q.clone(), k.clone()
    clean, _ = sa.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)
    q[3, 1] = 0
    q[5, 0, 7] = 1e18
    q[9, 2, 1] = float("nan")
    q[11, 3, 60] = float("inf")
    y, _ = sa.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)
    assert (y[3, 1] == 0).all() and torch.isfinite(y[5, 0]).all() and y[9, 2].isnan().any() and y[11, 3].isnan().any()
    same = torch.ones(64, 4, dtype=torch.bool)
    for i in ((3, 1), (5, 0), (9, 2), (11, 3)):
        same[i] = False
    assert torch.equal(y[same.to(DEV)], clean[same.to(DEV)])
    check_forward(y[5:6, 0:1], q[5:6, 0:1], wq, 1e-6, pos[5:6], freq, False, torch.bfloat16)


def test_in_place_strided_and_far_positions():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, wq, wk, pos, freq = make(50, 4, 2, 128, torch.float16, 128, 2**31 - 1, 9)
    want_q, want_k = sa.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)
    check_forward(want_q, q, wq, 1e-6, pos, freq, False, torch.float16)
    big = torch.zeros((50, 3, 8, 136), dtype=torch.float16, device=DEV)
    q2, k2 = big[:, 0, :4, :128], big[:, 1, 2:6:2, 8:136]
    q2.copy_(q)
    k2.copy_(k)
    rest = big.clone()
    rest[:, 0, :4, :128] = 0
    rest[:, 1, 2:6:2, 8:136] = 0
    yq, yk = sa.qk_norm_rope(q2, k2, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq, q_out=q2, k_out=k2)
    assert torch.equal(yq, want_q) and torch.equal(yk, want_k)
    now = big.clone()
    now[:, 0, :4, :128] = 0
    now[:, 1, 2:6:2, 8:136] = 0
    assert torch.equal(now, rest)
    one = torch.randn((1, 4, 128), device=DEV).half().expand(50, 4, 128)     # the same queries at all positions
    y, _ = sa.qk_norm_rope(one, k, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)
    check_forward(y, one, wq, 1e-6, pos, freq, False, torch.float16)


def check_backward(dx, dw, dy, x, w, eps, position, freq, adjacent, kind):
    pos, fr = position.tolist(), None if freq is None else freq.tolist()
    X, DY, W = f64(x), f64(dy), None if w is None else f64(w)
    want, want_w = paged.norm_rope_grad(DY, X, W, eps, pos, fr, adjacent)
    size = parts(DY, fr, adjacent)
    if W is not None:
        r = 1 / np.sqrt((X * X).mean(-1, keepdims=True) + eps)
        term_w = (size * np.abs(X) * r).sum((0, 1))
        assert (np.abs(f64(dw) - want_w) <= 2.0 ** -16 * term_w).all()
        g = size * np.abs(W)
        size = r * (g + np.abs(X) * r * (g * np.abs(X) * r).mean(-1, keepdims=True))
    err = np.abs(f64(dx) - want)
    assert (err <= half_step(kind, want) * (1 + 1e-6) + 2.0 ** -18 * size).all(), err.max()


@pytest.mark.parametrize("T,H,Hk,d", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_backward(T, H, Hk, d, kind, adjacent):
    import torch
    import paper_2601_16032_b200 as sa
    kind = kinds(kind)
    for rot in (d, d // 2, 0):
        q, k, v, wq, wk, pos, freq = make(T, H, Hk, d, kind, rot, 10000, T + rot + 1)
        gq, gk = torch.randn((T, H, d), device=DEV).to(kind), torch.randn((T, Hk, d), device=DEV).to(kind)
        args = dict(q_weight=wq, k_weight=wk, eps=1e-6, position=pos, inv_freq=freq, interleaved=adjacent)
        out = sa.qk_norm_rope_backward(gq, gk, q, k, **args)
        again = sa.qk_norm_rope_backward(gq, gk, q, k, **args)
        sa.attn_device_status()
        assert all(torch.equal(a, b) for a, b in zip(out, again))
        check_backward(out[0], out[2], gq, q, wq, 1e-6, pos, freq, adjacent, kind)
        check_backward(out[1], out[3], gk, k, wk, 1e-6, pos, freq, adjacent, kind)
        into = sa.qk_norm_rope_backward(gq, gk, q, k, dq=gq, dk=gk, **args)          # in place of the incoming gradients
        assert all(torch.equal(a, b) for a, b in zip(out, into)) and into[0] is gq


def test_backward_against_differences():
    """The kernel's gradient against differences of the 64-bit forward pass."""
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, wq, wk, pos, freq = make(5, 2, 1, 64, torch.float16, 64, 300, 31)
    gq, gk = torch.randn((5, 2, 64), device=DEV).half(), torch.randn((5, 1, 64), device=DEV).half()
    dq, dk, dwq, dwk = sa.qk_norm_rope_backward(gq, gk, q, k, q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)
    X, W, G = f64(q), f64(wq), f64(gq)
    loss = lambda X, W: float((paged.norm_rope(X, W, 1e-6, pos.tolist(), freq.tolist(), False) * G).sum())  # noqa: E731
    rng, h = np.random.default_rng(1), 1e-5
    for _ in range(30):
        i = tuple(rng.integers(0, n) for n in X.shape)
        e = np.zeros_like(X)
        e[i] = h
        slope = (loss(X + e, W) - loss(X - e, W)) / (2 * h)
        assert abs(float(dq[i]) - slope) <= 2.0 ** -11 * abs(slope) + 1e-5      # half a step, 32-bit and difference errors
        e = np.zeros_like(W)
        e[i[2]] = h
        assert abs(float(dwq[i[2]]) - (loss(X, W + e) - loss(X, W - e)) / (2 * h)) <= 1e-4


def test_zero_eps_and_no_tokens():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, wq, wk, pos, freq = make(9, 3, 1, 128, torch.bfloat16, 128, 300, 32)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    out = sa.qk_norm_rope_backward(gq, gk, q, k, q_weight=wq, k_weight=wk, eps=0.0, position=pos, inv_freq=freq)
    check_backward(out[0], out[2], gq, q, wq, 0.0, pos, freq, False, torch.bfloat16)
    out = sa.qk_norm_rope_backward(gq[:0], gk[:0], q[:0], k[:0], q_weight=wq, k_weight=wk, position=pos[:0], inv_freq=freq)
    assert out[0].shape == (0, 3, 128) and (out[2] == 0).all() and (out[3] == 0).all()
    yq, yk = sa.qk_norm_rope(q[:0], k[:0], q_weight=wq, k_weight=wk, position=pos[:0], inv_freq=freq)
    assert yq.shape == (0, 3, 128) and yk.shape == (0, 1, 128)


def test_captured_and_on_another_stream():
    import torch
    import paper_2601_16032_b200 as sa
    q, k, v, wq, wk, pos, freq = make(40, 4, 2, 64, torch.bfloat16, 64, 300, 33)
    q, k = q.clone(), k.clone()
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    ws = torch.empty(sa.attn_rope_bwd_workspace_bytes(64), dtype=torch.uint8, device=DEV)
    args = dict(q_weight=wq, k_weight=wk, position=pos, inv_freq=freq)

    def both():
        return (*sa.qk_norm_rope(q, k, **args), *sa.qk_norm_rope_backward(gq, gk, q, k, workspace=ws, **args))

    both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    q.normal_()
    gk.normal_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, both()):
        assert torch.equal(a, b)
