"""Pins of the oracle's embedding, head and clipping definitions: Python integers, the plaintext that three parties' shares open
to, and the gradients against the formula's and against differences (exact in the ring, where everything is linear or bilinear)."""
import math

import numpy as np
import pytest

from oracle import ring_oracle as ro
from paper_2104_10949_amd import workloads as wl

MOD = 1 << 64


def ints(a):
    return [int(v) for v in np.asarray(a).reshape(-1)]


def shares(x, seed):
    return ro.share(x, wl.draw_ring(x.shape, seed), wl.draw_ring(x.shape, seed + 1))


def opened(zs):
    return ro.reconstruct(*zs)


def parties(*sharings):
    """The operands of each party: both components of every sharing."""
    return [[c for s in sharings for c in (s[i], s[(i + 1) % 3])] for i in range(3)]


def test_embedding_by_integers():
    T, ids = wl.draw_ring((5, 3), 1), np.array([[4, -1, 0], [5, 4, 2]])
    z = ro.embedding(T, ids, -3)
    for at in np.ndindex(2, 3):
        v = int(ids[at])
        want = [(-3 * int(t)) % MOD for t in T[v]] if 0 <= v < 5 else [0, 0, 0]
        assert ints(z[at]) == want


def test_embedding_gradient_is_the_adjoint_and_accumulates():
    """sum over z of g * lookup(T) = sum over T of T * gradient(g), for every table: the formula's own definition."""
    ids = np.array([3, 0, 3, -2, 7, 3, 6])
    T, G, old = wl.draw_ring((7, 4), 2), wl.draw_ring((7, 4), 3), wl.draw_ring((7, 4), 4)
    d = ro.embedding_grad(G, ids, 7, 11)
    left = sum(a * b for a, b in zip(ints(G), ints(ro.embedding(T, ids, 11)))) % MOD
    assert left == sum(a * b for a, b in zip(ints(T), ints(d))) % MOD
    assert np.array_equal(ro.embedding_grad(G, ids, 7, 11, old), old + d)
    assert not d[[1, 2, 4, 5]].any()


def test_embedding_of_shares_opens_to_the_plain_one():
    X, ids = ro.encode(wl.draw_reals((9, 6), ("normal", 0.0, 1.0), 5)), np.array([8, 8, 9, 1])
    zs = [ro.embedding(s, ids, 5) for s in shares(X, 6)]
    assert np.array_equal(opened(zs), ro.embedding(X, ids, 5))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_by_integers_and_back(interleaved):
    f, dim, half = 14, 7, 2
    angle = np.array([[0.0, 0.0], [0.3, 1.9]])
    cos, sin = (ro.encode(fn(angle), f) for fn in (np.cos, np.sin))
    U, pos = wl.draw_ring((3, 2, dim), 8), np.array([1, 0, 2])
    z = ro.rotate(U, cos, sin, pos, f, interleaved)
    pairs = [(0, 1), (2, 3)] if interleaved else [(0, 2), (1, 3)]
    for t in range(2):
        for h in range(2):
            u = ints(U[t, h])
            for p, (d1, d2) in enumerate(pairs):
                c, s = int(cos[pos[t], p]), int(sin[pos[t], p])
                assert int(z[t, h, d1]) == (u[d1] * c - u[d2] * s) % MOD and int(z[t, h, d2]) == (u[d1] * s + u[d2] * c) % MOD
            assert ints(z[t, h, 4:]) == [(v << f) % MOD for v in u[4:]]
    assert not z[2].any()                                                # a position outside the table
    # angle 0 is a plain shift; the turn back is the transposed map: <g, R u> = <R^T g, u>
    assert np.array_equal(z[1], U[1] << np.uint64(f))
    g = wl.draw_ring(U.shape, 9)
    back = ro.rotate(g, cos, sin, pos, f, interleaved, back=True)
    assert sum(a * b for a, b in zip(ints(g), ints(z))) % MOD == sum(a * b for a, b in zip(ints(back), ints(U))) % MOD


def test_heads_of_shares_open_to_the_normed_and_turned_plaintext():
    """In reals: a head of norm 1 after the product with its inverse norm, turned by its angle.  Each of the three fixed-point
    factors is off by at most 2^-17 (t = 16; 2^-15 for the angles' 14 bits), of values below 1, 8 and 1."""
    t, f, rows, heads, dim = 16, 14, 4, 3, 8
    X = wl.draw_reals((rows, heads, dim), ("normal", 0.0, 1.0), 10)
    norm = 1.0 / np.sqrt((X ** 2).sum(-1))
    angle = np.arange(6)[:, None] * np.array([1.0, 0.1, 0.01])
    pos = np.array([5, 0, 3, 1])
    cos, sin = (ro.encode(fn(angle), f) for fn in (np.cos, np.sin))
    sx, sr = shares(ro.encode(X, t), 11), shares(ro.encode(norm, t), 13)
    z = opened([ro.head_norm_rotate(*ops, cos, sin, pos, f) for ops in parties(sx, sr)])
    c, s, u = np.cos(angle)[pos][:, None], np.sin(angle)[pos][:, None], X * norm[..., None]
    want = np.concatenate([u[..., :3] * c - u[..., 3:6] * s, u[..., :3] * s + u[..., 3:6] * c, u[..., 6:]], -1)
    # |x r - enc| <= 2^-17 |x| + 2^-17 |r| + 2^-34, |x| < 8, |r| < 8; two terms, plus two angles off by 2^-15 on |u| <= 1
    assert np.abs(ro.decode(z, 2 * t + f) - want).max() < 2 * (16 * 2.0 ** -17 + 2.0 ** -34) + 2 * 2.0 ** -15
    sq = opened([ro.head_sq_sum(*ops) for ops in parties(sx)])
    assert np.array_equal(sq, (ro.encode(X, t) ** np.uint64(2)).sum(-1, dtype=np.uint64))


@pytest.mark.parametrize("interleaved", [False, True])
def test_head_gradients_open_to_the_differences(interleaved):
    """The result is linear in x and in r: L(x + e) - L(x) is the gradient times e, exactly, for L = <g, z>."""
    f, rows, heads, dim = 10, 2, 2, 6
    angle = np.array([[0.7, 2.0], [0.1, 0.4], [1.0, 3.0]])
    cos, sin = (ro.encode(fn(angle), f) for fn in (np.cos, np.sin))
    pos = np.array([2, 0])
    X, R, G = wl.draw_ring((rows, heads, dim), 14), wl.draw_ring((rows, heads), 15), wl.draw_ring((rows, heads, dim), 16)
    sx, sr, sg = shares(X, 17), shares(R, 19), shares(G, 21)
    got = [ro.head_norm_rotate_grad(*ops, cos, sin, pos, f, interleaved) for ops in parties(sg, sx, sr)]
    dx, dr = (opened([g[k] for g in got]) for k in range(2))

    def loss(x, r):
        zero = np.zeros_like
        return sum(a * b for a, b in zip(ints(G), ints(ro.head_norm_rotate(x, zero(x), r, zero(r), cos, sin, pos, f, interleaved)))) % MOD
    base = loss(X, R)
    for at in [(0, 0, 0), (1, 1, 3), (0, 1, 5)]:
        for step in (1, 12345):
            x = X.copy()
            x[at] += np.uint64(step)
            assert (loss(x, R) - base) % MOD == int(dx[at]) * step % MOD
    for at in [(0, 0), (1, 1)]:
        r = R.copy()
        r[at] += np.uint64(777)
        assert (loss(X, r) - base) % MOD == int(dr[at]) * 777 % MOD


def test_squared_norm_of_shares_opens_to_the_plain_one():
    gs = [ro.encode(wl.draw_reals(s, ("normal", 0.0, 1.0), 30 + k)) for k, s in enumerate([(3, 5), (7,), (1,)])]
    sh = [shares(g, 40 + 2 * k) for k, g in enumerate(gs)]
    zs = [ro.sq_norm([(s[i], s[(i + 1) % 3]) for s in sh]) for i in range(3)]
    assert sum(zs) % MOD == sum(int(np.int64(v)) ** 2 for g in gs for v in g.view(np.int64).reshape(-1))


@pytest.mark.parametrize("S,max_norm,f", [(0, 0, 16), (0, 5, 16), (99, 9, 16), (100, 9, 16), (MOD - 1, 1 << 20, 16), ((1 << 32) + 1, 1 << 16, 0),
                                          (1 << 62, (1 << 31) - 1, 20), (1 << 62, 1 << 31, 20), (5, 0, 62)])
def test_clip_factor(S, max_norm, f):
    c = ro.clip_factor(S, max_norm, f)
    N = math.isqrt(S)
    assert c == (1 << f) if N <= max_norm else c * N <= max_norm << f < (c + 1) * N
