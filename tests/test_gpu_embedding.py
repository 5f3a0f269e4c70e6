"""Embedding lookup and its gradient on the GPU against the oracle: every bit of every row, at the sizes, ids and alignments where
the kernels change their way of working, and nothing written beside the outputs."""
import numpy as np
import pytest

from tests.gpu_util import first_mismatch, say

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


def draw_ids(kind, n, V, seed):
    rng = np.random.default_rng(seed)
    if kind == "one":                                    # every token the same
        return np.full(n, V - 1, np.int64)
    if kind == "padding":
        return np.full(n, -1, np.int64)
    if kind == "rank":                                   # frequencies as of words: the first id half of the time
        return (np.exp(rng.random(n) * np.log(V + 1)) - 1).astype(np.int64).clip(0, V - 1)
    if kind == "bucket":                                 # rows that the same block looks after
        return (rng.integers(0, 8, n) + rng.integers(0, max(1, V // 1024), n) * 1024).clip(0, V - 1)
    if kind == "position":
        return np.arange(n) % V
    ids = rng.integers(0, V, n)
    if kind == "mixed":                                  # padding of every kind among them
        bad = rng.random(n) < 0.3
        ids[bad] = rng.choice([-1, V, V + 7, -2 ** 31, 2 ** 31 - 1], bad.sum())
    return ids


def place(cg, a, words=0):
    """The words of `a` on the GPU, `words` behind a 256-byte boundary."""
    flat = torch.empty(a.size + words, dtype=torch.int64, device="cuda")
    t = flat[words:].view(a.shape)
    t.copy_(cg.to_device(a) if a.size else t)
    return t


GUARD = 0x5A5A5A5A5A5A5A5A


class Guarded:
    """An output with guard words on both sides of it."""

    def __init__(self, shape, words=0, fill=None):
        size = int(np.prod(shape))
        self.flat = torch.full((size + 64 + words,), GUARD, dtype=torch.int64, device="cuda")
        self.lo, self.size = 32 + words, size
        self.t = self.flat[self.lo:self.lo + size].view(shape)
        if fill is not None:
            self.t.copy_(torch.from_numpy(fill.view(np.int64)))

    def host(self):
        flat = self.flat.cpu().numpy()
        assert (flat[:self.lo] == GUARD).all() and (flat[self.lo + self.size:] == GUARD).all(), "written beside the output"
        return flat[self.lo:self.lo + self.size].view(np.uint64).reshape(tuple(self.t.shape))


LOOKUPS = [(1, 1, 1), (1, 10, 512), (2, 3, 2), (3, 2, 515), (65, 50, 7), (64, 50, 8), (257, 100, 64), (1000, 33, 130), (5, 9, 1024), (3, 4, 4098),
           (33, 1000, 2049), (4097, 64, 16), (100, 300, 768)]


@pytest.mark.parametrize("n,V,D", LOOKUPS)
@pytest.mark.parametrize("dtype,words", [(torch.int64, 0), (torch.int32, 0), (torch.int32, 1)])
def test_lookup(cg, ro, wl, n, V, D, dtype, words):
    say(f"lookup n={n} V={V} D={D} {dtype} {words} words off")
    ids, alpha = draw_ids("mixed", n, V, n + V), 0x123456789ABCDEF1
    T = [wl.draw_ring((V, D), 100 + k) for k in range(2)]
    z = [Guarded((n, D), words) for _ in range(2)]
    dev = torch.from_numpy(ids).to("cuda").to(dtype)
    cg.cg_share_embedding(place(cg, T[0], words), place(cg, T[1], words), dev, alpha, za=z[0].t, zb=z[1].t)
    for t, out in zip(T, z):
        want = ro.embedding(t, ids, alpha)
        assert np.array_equal(out.host(), want), first_mismatch(out.host(), want)


def test_lookup_of_a_batch_and_of_nothing(cg, ro, wl):
    T = [wl.draw_ring((20, 24), 110 + k) for k in range(2)]
    ids = draw_ids("uniform", 42, 20, 5).reshape(2, 3, 7)
    z = cg.cg_share_embedding(*(cg.to_device(t) for t in T), torch.from_numpy(ids).cuda())
    assert z[0].shape == (2, 3, 7, 24)
    for t, out in zip(T, z):
        assert np.array_equal(cg.to_host(out), ro.embedding(t, ids))
    none = torch.empty((0, 4), dtype=torch.int64, device="cuda")
    z = cg.cg_share_embedding(*(cg.to_device(t) for t in T), none)
    assert z[0].shape == (0, 4, 24)


def test_lookup_beyond_32_bit_offsets(cg):
    """A table whose last rows lie behind 2^32 bytes, and whose words lie behind 2^29."""
    V, D = (1 << 20) + 3, 520
    say(f"lookup in a table of {V} x {D} words")
    T = torch.arange(V, dtype=torch.int64, device="cuda")[:, None] * 1000003 + torch.arange(D, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2, 1 << 20], device="cuda")
    za, zb = cg.cg_share_embedding(T, T, ids, 3)
    want = (ids[:, None] * 1000003 + torch.arange(D, device="cuda")) * 3
    assert torch.equal(za, want) and torch.equal(zb, want)


# (n, V, D): one token to many, rows shorter and longer than a wave's piece, tables smaller and larger than the batch
GRADS = [(1, 1, 1), (1, 700, 512), (2, 5, 3), (63, 7, 16), (64, 64, 64), (65, 1000, 30), (128, 300, 514), (129, 300, 514), (100, 40, 1031), (500, 3, 515), (777, 1531, 130), (1024, 2000, 257), (1025, 100, 260), (1024, 3, 70000), (600, (1 << 18) + 5, 4), (600, 1 << 18, 4), (2048, 60, 512), (2048, 60, 513), (2049, 60, 8), (4096, 9, 40), (20480, 1200, 6), (20481, 1200, 6), (20480, 300, 9), (20480, 1000, 700), (5000, 1 << 20, 2), (5000, (1 << 20) + 1, 2), (9000, 130 * 1024, 5), (2048, 100, 258),
         (4096, 300, 8), (4097, 40, 64), (5000, 5000, 20), (3000, 9, 1030), (9001, 2000, 33), (20000, 700, 34), (16384, 16384, 6), (40000, 50, 18)]


@pytest.mark.parametrize("n,V,D", GRADS)
@pytest.mark.parametrize("kind", ["rank", "mixed", "one", "position", "bucket"])
@pytest.mark.parametrize("scratch", [True, False])
def test_gradient(cg, ro, wl, n, V, D, kind, scratch):
    say(f"gradient n={n} V={V} D={D} {kind}, scratch memory {scratch}")
    ids, alpha, words = draw_ids(kind, n, V, n + D), 0xFEDCBA9876543210 + n, int(kind == "mixed")
    G = [wl.draw_ring((n, D), 120 + k) for k in range(2)]
    dev = torch.from_numpy(ids).to("cuda").to(torch.int32 if kind == "rank" else torch.int64)
    g = [place(cg, t, words) for t in G]
    d = [Guarded((V, D), words) for _ in range(2)]
    need = max(cg.cg_share_embedding_grad_workspace_bytes(n, V, D, acc) for acc in (False, True)) if scratch else 0
    memory = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    ws = memory[256:256 + need]                              # without: none of it is used
    cg.cg_share_embedding_grad(*g, dev, V, alpha, da=d[0].t, db=d[1].t, workspace=ws)
    want = [ro.embedding_grad(t, ids, V, alpha) for t in G]
    for w, out in zip(want, d):
        assert np.array_equal(out.host(), w), first_mismatch(out.host(), w)
    cg.cg_share_embedding_grad(*g, dev, V, alpha, da=d[0].t, db=d[1].t, accumulate=True, workspace=ws)     # and once more on top
    for w, out in zip(want, d):
        assert np.array_equal(out.host(), w + w), first_mismatch(out.host(), w + w)
    assert bool((memory[:256] == 0x5A).all()) and bool((memory[256 + need:] == 0x5A).all())


@pytest.mark.parametrize("n", [0, 40, 5000, 20000, 30000])
def test_gradient_of_padding_alone(cg, wl, n):
    say(f"gradient of {n} tokens of padding")
    V, D = 31, 22
    g = [cg.to_device(wl.draw_ring((n, D), 130 + k)) for k in range(2)]
    ids = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    old = wl.draw_ring((V, D), 132)
    d = [Guarded((V, D), fill=old) for _ in range(2)]
    cg.cg_share_embedding_grad(*g, ids, V, 5, da=d[0].t, db=d[1].t, accumulate=True)
    assert all(np.array_equal(t.host(), old) for t in d)
    cg.cg_share_embedding_grad(*g, ids, V, 5, da=d[0].t, db=d[1].t)
    assert all(not t.host().any() for t in d)


@pytest.mark.parametrize("n", [300, 3000, 20000, 30000])
def test_gradient_on_another_stream_and_of_changing_ids(cg, ro, wl, n):
    """Calls one after the other on one stream with ids and gradients overwritten in between, each checked."""
    say(f"gradient on a stream of its own, n={n}")
    V, D = 150, 40
    s = torch.cuda.Stream()
    ids = torch.empty(n, dtype=torch.int64, device="cuda")
    g = [torch.empty((n, D), dtype=torch.int64, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    results, wants = [], []
    with torch.cuda.stream(s):
        for k, kind in enumerate(("rank", "one", "mixed", "uniform")):
            host = draw_ids(kind, n, V, k)
            G = [wl.draw_ring((n, D), 140 + 2 * k + c) for c in range(2)]
            ids.copy_(torch.from_numpy(host).cuda())
            for t, h in zip(g, G):
                t.copy_(cg.to_device(h))
            results.append(cg.cg_share_embedding_grad(*g, ids, V, 7, stream=s if k % 2 else None))
            wants.append([ro.embedding_grad(h, host, V, 7) for h in G])
    s.synchronize()
    for got, want in zip(results, wants):
        for a, w in zip(got, want):
            assert np.array_equal(cg.to_host(a), w), first_mismatch(cg.to_host(a), w)


@pytest.mark.parametrize("n", [500, 3000, 20000, 30000])
def test_gradients_on_two_streams_at_once(cg, ro, wl, n):
    """Calls under way at the same time on two streams, scratch memory from the allocator for each."""
    say(f"two gradients of {n} tokens at once")
    V, D = 400, 64
    jobs = []
    for k in range(2):
        host = draw_ids("rank", n, V, k)
        G = [wl.draw_ring((n, D), 180 + 2 * k + c) for c in range(2)]
        jobs.append((torch.cuda.Stream(), torch.from_numpy(host).cuda(), [cg.to_device(h) for h in G], host, G))
    torch.cuda.synchronize()
    results = [[], []]
    for _ in range(6):
        for k, (s, ids, g, _, _) in enumerate(jobs):
            with torch.cuda.stream(s):
                results[k].append(cg.cg_share_embedding_grad(*g, ids, V, 3))
    torch.cuda.synchronize()
    for k, (_, _, _, host, G) in enumerate(jobs):
        want = [ro.embedding_grad(h, host, V, 3) for h in G]
        for got in results[k]:
            for a, w in zip(got, want):
                assert np.array_equal(cg.to_host(a), w), first_mismatch(cg.to_host(a), w)


def test_gradient_added_as_a_numpy_truth_value_says(cg, ro, wl):
    n, V, D = 5000, 60, 12
    host = draw_ids("uniform", n, V, 3)
    ids, G = torch.from_numpy(host).cuda(), [wl.draw_ring((n, D), 230 + c) for c in range(2)]
    g, d = [cg.to_device(h) for h in G], [torch.ones((V, D), dtype=torch.int64, device="cuda") for _ in range(2)]
    cg.cg_share_embedding_grad(*g, ids, V, da=d[0], db=d[1], accumulate=np.bool_(True))
    for t, h in zip(d, G):
        assert np.array_equal(cg.to_host(t), ro.embedding_grad(h, host, V, 1) + np.uint64(1))


@pytest.mark.parametrize("n", [300, 3000, 20000, 30000])
def test_gradient_in_two_graphs(cg, ro, wl, n):
    """Two captured calls, replayed in turn with new inputs and the program's own work in between."""
    say(f"gradient in two graphs, n={n}")
    V, D = 90, 36
    state, graphs = [], []
    for k in range(2):
        ids = torch.from_numpy(draw_ids("rank", n, V, k)).cuda()
        # the second graph has scratch memory of its own, the first none
        ws = torch.empty(cg.cg_share_embedding_grad_workspace_bytes(n, V, D, True) if k else 0, dtype=torch.uint8, device="cuda")
        g = [cg.to_device(wl.draw_ring((n, D), 160 + c)) for c in range(2)]
        d = [torch.zeros((V, D), dtype=torch.int64, device="cuda") for _ in range(2)]
        cg.cg_share_embedding_grad(*g, ids, V, 3, da=d[0], db=d[1], workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cg.cg_share_embedding_grad(*g, ids, V, 3, da=d[0], db=d[1], workspace=ws)
            cg.cg_share_embedding_grad(*g, ids, V, 3, da=d[0], db=d[1], accumulate=True, workspace=ws)
        state.append((ids, g, d, ws))
        graphs.append(graph)
    for turn in range(4):
        for k in range(2):
            ids, g, d, _ = state[k]
            host = draw_ids(["rank", "one", "mixed", "uniform"][turn], n, V, 10 * turn + k)
            G = [wl.draw_ring((n, D), 170 + 10 * turn + 2 * k + c) for c in range(2)]
            ids.copy_(torch.from_numpy(host))
            for t, h in zip(g, G):
                t.copy_(cg.to_device(h))
            for t in d:
                t.fill_(turn)
            graphs[k].replay()
            _ = cg.cg_share_embedding_grad(*state[1 - k][1], state[1 - k][0], V)      # the program's own work
            if turn % 2:
                torch.cuda.synchronize()
            for t, h in zip(d, G):
                want = ro.embedding_grad(h, host, V, 6)
                assert np.array_equal(cg.to_host(t), want), first_mismatch(cg.to_host(t), want)


@pytest.mark.parametrize("n", [500, 3000, 9000])
def test_calls_captured_as_they_are(cg, ro, wl, n):
    """Lookup and gradient captured without a word about scratch memory: nothing is allocated inside the call for it."""
    say(f"lookup and gradient of {n} tokens in a graph")
    V, D = 70, 18
    T = [wl.draw_ring((V, D), 190 + c) for c in range(2)]
    G = [wl.draw_ring((n, D), 192 + c) for c in range(2)]
    table, g = [cg.to_device(t) for t in T], [cg.to_device(t) for t in G]
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    cg.cg_share_embedding_grad(*g, ids, V, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = cg.cg_share_embedding(*table, ids, 9)
        d = cg.cg_share_embedding_grad(*g, ids, V, 3)
    for turn, kind in enumerate(("rank", "mixed", "one", "position")):
        host = draw_ids(kind, n, V, turn).clip(-5, V + 5)
        ids.copy_(torch.from_numpy(host))
        graph.replay()
        _ = cg.cg_share_embedding_grad(*g, ids, V, 3)
        for a, t in zip(z, T):
            assert np.array_equal(cg.to_host(a), ro.embedding(t, host, 9))
        for a, h in zip(d, G):
            assert np.array_equal(cg.to_host(a), ro.embedding_grad(h, host, V, 3))


def test_gradient_of_many_words(cg):
    """Gradients behind 2^32 bytes and a table of as many: rows of ones, so that every sum is a count."""
    n, V, D = 1 << 16, (1 << 17) + 1, 8200
    say(f"gradient n={n} V={V} D={D}")
    g = torch.ones((n, D), dtype=torch.int64, device="cuda")
    ids = torch.full((n,), V - 1, dtype=torch.int64, device="cuda")
    ids[::2] = torch.arange(0, n, 2, device="cuda") * 2
    da, db = cg.cg_share_embedding_grad(g, g, ids, V, 2)
    count = torch.bincount(ids, minlength=V) * 2
    for d in (da, db):
        assert torch.equal(d[:, 0], count) and torch.equal(d[:, D - 1], count) and torch.equal(d[V - 1], count[V - 1].expand(D))
        assert int(d.sum(0).ne(2 * n).sum()) == 0
