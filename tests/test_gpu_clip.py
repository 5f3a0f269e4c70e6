"""Global gradient norm, clip factor and clipping on the GPU against the oracle, bit for bit; and one party's step from the
embedding to the clipped gradients, as a program runs it, with what the three parties open to."""
import numpy as np
import pytest

from tests.gpu_util import first_mismatch, say
from tests.test_gpu_embedding import Guarded, place

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2104_10949_amd import binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def ro():
    from oracle import ring_oracle
    return ring_oracle


@pytest.fixture(scope="module")
def wl():
    from paper_2104_10949_amd import workloads
    return workloads


LISTS = [[], [0], [1], [2], [255, 0, 1], [4096], [4097, 3], [8191, 8193, 1, 1, 64], [100003], [1] * 300, [3000 + 7 * k for k in range(130)], [5 + 3 * (k % 90) for k in range(161)], [64] * 97, [3 * 8192, 1], [4 * 8192 + 1], [9000, 0, 16384],
         [1 << 21, 5, (1 << 20) + 1], [0] * 100 + [77], list(range(200))]


@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
@pytest.mark.parametrize("words", [0, 1])
def test_norm_and_clip_of_lists(cg, ro, wl, sizes, words):
    say(f"norm and clip of {len(sizes)} tensors, the largest {max(sizes, default=0)}, {words} words off")
    host = [[wl.draw_ring((n,), 300 + 2 * k + c) for k, n in enumerate(sizes)] for c in range(2)]
    dev = [[place(cg, a, words) for a in part] for part in host]
    out = [[Guarded((n,), words) for n in sizes] for _ in range(2)]
    x, y = cg.ShareList(*dev), cg.ShareList(*([g.t for g in part] for part in out))
    z = Guarded((1,), words)
    z.t.fill_(99)
    cg.cg_share_sq_norm(x, z_i=z.t)
    assert int(z.host()[0]) == ro.sq_norm(zip(*host))
    c = 0xA5A5A5A512345677
    factor = cg.to_device(np.array([c], np.uint64))
    cg.cg_share_clip(x, factor, y)
    for part, got in zip(host, out):
        for a, g in zip(part, got):
            assert np.array_equal(g.host(), a * np.uint64(c)), first_mismatch(g.host(), a * np.uint64(c))
    cg.cg_share_clip(x, factor)                         # in place
    for part, got in zip(host, dev):
        for a, t in zip(part, got):
            assert np.array_equal(cg.to_host(t), a * np.uint64(c))


def test_views_of_one_buffer_one_after_the_other(cg, ro, wl):
    """Gradients as a program keeps them, odd sizes without gaps: every alignment of 8 bytes."""
    sizes = [5, 8, 1, 300, 7, 4096, 9001, 2]
    flat = [wl.draw_ring((sum(sizes),), 320 + c) for c in range(2)]
    dev = [cg.to_device(a) for a in flat]
    x = cg.ShareList(*(t.split(sizes) for t in dev))
    assert int(cg.to_host(cg.cg_share_sq_norm(x))[0]) == ro.sq_norm([flat])
    factor = torch.tensor([7], device="cuda")
    cg.cg_share_clip(x, factor)
    for a, t in zip(flat, dev):
        assert np.array_equal(cg.to_host(t), a * np.uint64(7))


def test_tensors_of_more_than_2_to_the_31_words(cg):
    """Behind 2^34 bytes, and cut into two entries of a launch."""
    n = (1 << 31) + 1029
    say(f"norm and clip of a tensor of {n} words")
    a, b = (torch.full((n,), v, dtype=torch.int64, device="cuda") for v in (3, 5))
    for at in (0, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1):
        a[at] = 1000
    x = cg.ShareList([a[:7], a[7:]], [b[:7], b[7:]])
    assert int(cg.cg_share_sq_norm(x)) == (n - 5) * 3 * 13 + 5 * 1000 * 1010
    cg.cg_share_clip(x, torch.tensor([2], device="cuda"))
    assert int(a.sum()) == (n - 5) * 6 + 5 * 2000 and int(b.min()) == int(b.max()) == 10


def test_lists_in_any_order(cg, wl):
    """Outputs that descend, lie between the inputs or are the inputs of their own position are all fine."""
    host = [wl.draw_ring((100,), 330 + k) for k in range(4)]
    buffer = torch.zeros(1000, dtype=torch.int64, device="cuda")
    a0, a1, b0, b1 = (buffer[200 * k:200 * k + 100] for k in range(4))
    for t, h in zip((a0, a1, b0, b1), host):
        t.copy_(cg.to_device(h))
    y0, y1 = buffer[900:1000], buffer[100:200]
    factor = torch.tensor([3], device="cuda")
    cg.cg_share_clip(cg.ShareList([a0, a1], [b0, b1]), factor, cg.ShareList([y0, y1], [b0, b1]))
    for t, h in zip((y0, y1, b0, b1), host):
        assert np.array_equal(cg.to_host(t), h * np.uint64(3))
    assert np.array_equal(cg.to_host(a0), host[0]) and not bool(buffer[300:400].any())


def test_lists_that_write_a_word_twice_are_refused(cg, wl):
    t = [torch.ones(64, dtype=torch.int64, device="cuda") for _ in range(2)]
    factor = torch.tensor([2], device="cuda")
    with pytest.raises(cg.CgError) as e:
        cg.cg_share_clip(cg.ShareList([t[0], t[0]], [t[1], t[1]]), factor)          # a tied weight listed twice
    assert e.value.status == cg.CG_ERR_ALIAS
    with pytest.raises(cg.CgError) as e:
        cg.cg_share_clip(cg.ShareList([t[0][:32], t[0][31:]], [t[1][:32], t[1][31:]]), factor)
    assert e.value.status == cg.CG_ERR_ALIAS
    torch.cuda.synchronize()
    assert all(bool((a == 1).all()) for a in t)


S_VALUES = [0, 1, 2, 3, 4, 99, 100, (1 << 32) - 1, 1 << 32, (1 << 52) + 3, (3037000499 ** 2) - 1, 3037000499 ** 2, (1 << 63) - 1, 1 << 63, (1 << 64) - 1,
            (4294967295 ** 2) - 1, 4294967295 ** 2]


@pytest.mark.parametrize("max_norm,f", [(0, 16), (1, 62), (9, 16), (1 << 16, 16), (10 << 16, 20), ((1 << 32) - 1, 31), ((1 << 48) - 1, 16), ((1 << 64) - 1, 0)])
def test_clip_factor(cg, ro, wl, max_norm, f):
    for S in S_VALUES:
        s0, s1 = (int(v) for v in wl.draw_ring((2,), S % 1000))
        words = [cg.to_device(np.array([v % (1 << 64)], np.uint64)) for v in (s0, s1, S - s0 - s1)]
        got = int(cg.to_host(cg.cg_clip_factor(*words, max_norm, f))[0])
        assert got == ro.clip_factor(S, max_norm, f), (S, max_norm, f)
        cg.cg_clip_factor(*words, max_norm, f, factor=words[1])                       # over one of the shares
        assert int(cg.to_host(words[1])[0]) == got


def test_norm_and_clip_in_a_graph(cg, ro, wl):
    sizes = [3000, 17, 9999, 1]
    dev = [[torch.zeros(n, dtype=torch.int64, device="cuda") for n in sizes] for _ in range(2)]
    out = [[torch.zeros(n, dtype=torch.int64, device="cuda") for n in sizes] for _ in range(2)]
    x, y = cg.ShareList(*dev), cg.ShareList(*out)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    cg.cg_share_sq_norm(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = cg.cg_share_sq_norm(x)
        c = cg.cg_clip_factor(z, zero, zero, 5 << 32, 16)
        cg.cg_share_clip(x, c, y)
    for turn in range(4):
        host = [[wl.draw_ring((n,), 340 + 20 * turn + 2 * k + p) for k, n in enumerate(sizes)] for p in range(2)]
        for part, ts in zip(host, dev):
            for a, t in zip(part, ts):
                t.copy_(cg.to_device(a))
        graph.replay()
        _ = cg.cg_share_sq_norm(y)
        if turn % 2:
            torch.cuda.synchronize()
        S = ro.sq_norm(zip(*host))
        want = ro.clip_factor(S, 5 << 32, 16)
        assert int(cg.to_host(z)[0]) == S and int(cg.to_host(c)[0]) == want
        for part, ts in zip(host, out):
            for a, t in zip(part, ts):
                assert np.array_equal(cg.to_host(t), a * np.uint64(want))


def test_a_private_step_from_the_embedding_to_the_clipped_gradients(cg, ro, wl):
    """Three parties, each with its own calls, messages as plain assignments: lookup, query and key projection, norms and rotation
    (the inverse norms dealt as fresh shares, in place of the protocol), then backward to the projection and the table, the
    opened norm and the clipping.  Everything opens to what the same steps give on the plain words of the ring."""
    n, V, D, heads, dim, P, f = 30, 12, 16, 3, 8, 20, 10
    ids = np.array([3, -1, 5] * 10)
    pos = np.arange(n) % P
    plain = {"T": wl.draw_ring((V, D), 400), "W": wl.draw_ring((heads * dim, D), 401), "r": wl.draw_ring((n, heads), 402),
             "g": wl.draw_ring((n, heads, dim), 403)}
    cos, sin = wl.draw_ring((P, dim // 2), 404), wl.draw_ring((P, dim // 2), 405)
    sh = {k: ro.share(v, wl.draw_ring(v.shape, 410 + 2 * i), wl.draw_ring(v.shape, 411 + 2 * i)) for i, (k, v) in enumerate(plain.items())}
    dev = {k: [cg.to_device(s) for s in v] for k, v in sh.items()}
    dids, dpos, dcos, dsin = torch.from_numpy(ids).cuda(), torch.from_numpy(pos).cuda().int(), cg.to_device(cos), cg.to_device(sin)
    turn = dict(cos=dcos, sin=dsin, pos=dpos, frac_bits=f)
    keys = [bytes([k] * 16) for k in range(3)]

    def pair(s, i):
        return s[i], s[(i + 1) % 3]

    def reshare(zs, nonce):
        return [cg.cg_reshare(z, keys[i], keys[(i - 1) % 3], nonce) for i, z in enumerate(zs)]

    def open_(zs):
        return cg.to_host(cg.cg_reconstruct(*zs))

    # forward
    X = [cg.cg_share_embedding(*pair(dev["T"], i), dids, 5) for i in range(3)]
    assert all(torch.equal(X[i][1], X[(i + 1) % 3][0]) for i in range(3))             # linear: the pairs stay replicated
    x = [p[0] for p in X]
    qk = reshare([cg.cg_share_matmul(*pair(x, i), *pair(dev["W"], i)).view(n, heads, dim) for i in range(3)], 1)
    sq = [cg.cg_share_head_sq_sum(*pair(qk, i)) for i in range(3)]
    z = [cg.cg_share_head_norm_rotate(*pair(qk, i), *pair(dev["r"], i), **turn) for i in range(3)]
    px = ro.embedding(plain["T"], ids, 5)
    pqk = ro.matmul(px, plain["W"]).reshape(n, heads, dim)
    assert np.array_equal(open_(sq), (pqk * pqk).sum(-1, dtype=np.uint64))
    assert np.array_equal(open_(z), ro.rotate(pqk * plain["r"][..., None], cos, sin, pos, f, False))
    # backward
    back = [cg.cg_share_head_norm_rotate_grad(*pair(dev["g"], i), *pair(qk, i), *pair(dev["r"], i), **turn) for i in range(3)]
    dqk, dr = reshare([b[0] for b in back], 2), [b[1] for b in back]
    pv = ro.rotate(plain["g"], cos, sin, pos, f, False, back=True)
    pdqk = pv * plain["r"][..., None]
    assert np.array_equal(open_(dqk), pdqk) and np.array_equal(open_(dr), (pqk * pv).sum(-1, dtype=np.uint64))
    flat = [t.view(n, heads * dim) for t in dqk]
    dx = reshare([cg.cg_share_matmul_t(*pair(flat, i), *pair(dev["W"], i), False, True) for i in range(3)], 3)
    dW = reshare([cg.cg_share_matmul_t(*pair(flat, i), *pair(x, i), True, True) for i in range(3)], 4)
    dT = [cg.cg_share_embedding_grad(*pair(dx, i), dids, V, 5) for i in range(3)]
    pflat = pdqk.reshape(n, heads * dim)
    pdW = ro.matmul(np.ascontiguousarray(pflat.T), np.ascontiguousarray(px.T))
    pdT = ro.embedding_grad(ro.matmul(pflat, np.ascontiguousarray(plain["W"].T)), ids, V, 5)
    assert np.array_equal(open_(dW), pdW) and np.array_equal(open_([p[0] for p in dT]), pdT)
    # norm and clipping
    lists = [cg.ShareList([pair(dW, i)[0].clone(), dT[i][0]], [pair(dW, i)[1].clone(), dT[i][1]]) for i in range(3)]
    norm = [cg.cg_share_sq_norm(x) for x in lists]
    S = int((pdW * pdW).sum(dtype=np.uint64)) + int((pdT * pdT).sum(dtype=np.uint64))
    assert int(open_(norm)[0]) == S % (1 << 64)
    factors = [cg.cg_clip_factor(*norm, 3 << 16, 20) for _ in range(3)]
    want = ro.clip_factor(S, 3 << 16, 20)
    assert all(int(cg.to_host(c)[0]) == want for c in factors)
    for x, c in zip(lists, factors):
        cg.cg_share_clip(x, c)
    for k, plain_grad in enumerate((pdW, pdT)):
        assert np.array_equal(open_([x.a[k] for x in lists]), plain_grad * np.uint64(want))
