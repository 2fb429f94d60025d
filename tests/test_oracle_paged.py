"""Pins of the plain statements in oracle/paged.py: closed forms, invariants and differences."""
import numpy as np
import pytest

from oracle import paged


def test_plan_by_hand():
    table = np.array([[5, 6, -1, -1], [7, -1, -1, -1], [8, 9, -1, -1]])
    free = np.array([1, 2, 3, 0, 0, 0, 0, 0])
    # request 0 grows from 7 to 10 tokens (pages of 4): one page; request 1 ends with one page; request 2 grows by nothing
    p = paged.page_plan([7, 3, 8], [3, -1, 0], 4, table, free, 3, 8, 5)
    assert p["info"] == [0, 3, 1, 1] and p["count"] == 3
    assert p["table"][0].tolist() == [5, 6, 7, -1]        # the page request 1 gave back was on top
    assert p["slot"] == [27, 28, 29, -1, -1] and p["position"] == [7, 8, 9, 0, 0] and p["request"] == [0, 0, 0, -1, -1]
    assert p["seq_len"] == [10, 0, 8] and p["q_start"] == [0, 3, 3, 3]
    assert p["free"][:3].tolist() == [1, 2, 3]
    assert paged.page_plan([7, 3, 8], [3, -1, 0], 4, table, free, 3, 8, 2)["info"] == [2, 3, 1, 1]
    assert paged.page_plan([7, 3, 8], [9, 9, 8], 4, table, free, 3, 8, 99)["info"] == [3, 26, 6, 0]
    assert paged.page_plan([7, 3, 8], [10, 0, 0], 4, table, free, 3, 8, 99)["info"] == [1, 0, 0, 0]


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_invariants(adjacent):
    rng = np.random.default_rng(1)
    x, freq = rng.standard_normal((4, 2, 32)), 1e4 ** (-np.arange(8) / 8)
    pos = [0, 1, 77, 123456]
    y = paged.rotate(x, pos, freq, adjacent)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 16:], x[..., 16:])
    assert np.allclose((y * y).sum(-1), (x * x).sum(-1))
    assert np.allclose(paged.rotate(y, pos, freq, adjacent, back=True), x)
    # the product of a query and a key depends on the distance of their positions only
    q, k = x[0:1], x[1:2]
    dot = [(paged.rotate(q, [a], freq, adjacent) * paged.rotate(k, [a + 5], freq, adjacent)).sum() for a in (0, 3, 1000)]
    assert np.allclose(dot, dot[0])


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 32])
def test_gradient_against_differences(adjacent, rot):
    rng = np.random.default_rng(2)
    x, w, dy = rng.standard_normal((3, 2, 32)), rng.standard_normal(32), rng.standard_normal((3, 2, 32))
    freq, pos = 1e4 ** (-np.arange(rot // 2) / 16), [0, 5, 900]

    def loss(x, w):
        return float((paged.norm_rope(x, w, 1e-6, pos, freq, adjacent) * dy).sum())

    dx, dw = paged.norm_rope_grad(dy, x, w, 1e-6, pos, freq, adjacent)
    h = 1e-6
    for _ in range(20):
        i = tuple(rng.integers(0, n) for n in x.shape)
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-7
        e = np.zeros_like(w)
        e[i[2]] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[i[2]]) < 1e-7


def test_decode_is_the_last_row_of_causal_attention():
    from oracle import attention as ora
    rng = np.random.default_rng(3)
    k, v, q = rng.standard_normal((37, 2, 16)), rng.standard_normal((37, 2, 16)), rng.standard_normal((4, 16))
    o, lse = paged.decode(q, k, v, 0.25)
    for h in range(4):
        full = ora.attention_head(np.concatenate([np.zeros((36, 16)), q[h:h + 1]]), k[:, h // 2].copy(), v[:, h // 2].copy(), 0.25, True)
        assert np.allclose(o[h], full[-1], atol=1e-12)
    o, lse = paged.decode(q, k[:0], v[:0], 0.25)
    assert (o == 0).all() and np.isneginf(lse).all()


def test_gather_follows_the_table():
    cache = np.arange(5 * 4 * 2 * 3).reshape(5, 4, 2, 3)
    row = [3, 0, 4]
    got = paged.gather(cache, row, 9, 4, False)
    assert np.array_equal(got[5], cache[0, 1]) and np.array_equal(got[8], cache[4, 0])
    assert np.array_equal(paged.gather(cache.transpose(0, 2, 1, 3), row, 9, 4, True), got)
