"""Sums of squares, norm with rotation, and their gradient on the GPU against the oracle, bit for bit."""
import numpy as np
import pytest

from tests.gpu_util import first_mismatch, say
from tests.test_gpu_embedding import GUARD, Guarded

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


def packed(cg, a, extra, words=0):
    """[rows, heads, dim] words as the first heads of rows that are `extra` words longer, `words` behind a boundary."""
    rows, heads, dim = a.shape
    ld = heads * dim + extra
    flat = torch.full((rows * ld + words,), GUARD, dtype=torch.int64, device="cuda")
    t = flat[words:].as_strided((rows, heads, dim), (ld, dim, 1), words)
    t.copy_(cg.to_device(a))
    return t


class GuardedRows:
    """An output whose rows lie apart: what is between them stays as it is."""

    def __init__(self, rows, heads, dim, extra, words=0):
        self.shape, self.ld, self.words = (rows, heads, dim), heads * dim + extra, words
        self.flat = torch.full((rows * self.ld + words + 64,), GUARD, dtype=torch.int64, device="cuda")
        self.t = self.flat.as_strided((rows, heads, dim), (self.ld, dim, 1), words)

    def host(self):
        rows, heads, dim = self.shape
        flat = self.flat.cpu().numpy()
        body = flat[self.words:self.words + rows * self.ld].reshape(rows, self.ld)
        assert (flat[:self.words] == GUARD).all() and (flat[self.words + rows * self.ld:] == GUARD).all() and (body[:, heads * dim:] == GUARD).all()
        return body[:, :heads * dim].reshape(rows, heads, dim).view(np.uint64)


# rows, heads, dim, rot, words between the rows, words behind a boundary
SHAPES = [(1, 1, 1, 0, 0, 0), (1, 1, 2, 2, 0, 0), (1, 16, 64, 64, 256, 0), (3, 2, 5, 4, 1, 0), (7, 3, 6, 2, 0, 1), (2, 5, 16, 8, 16, 0), (5, 1, 80, 40, 0, 0),
          (33, 7, 80, 40, 2, 0), (9, 4, 128, 128, 64, 0), (4, 3, 128, 126, 0, 0), (3, 3, 130, 66, 2, 0), (2, 2, 256, 256, 0, 0), (2, 2, 515, 512, 3, 0),
          (1, 2, 1024, 1024, 0, 0), (130, 1, 32, 32, 0, 0), (64, 9, 96, 48, 0, 2), (3, 2, 64, 62, 0, 0), (257, 5, 12, 12, 4, 0), (2, 1, 1300, 650, 0, 1)]
FRAC = 14


def case(cg, wl, rows, heads, dim, rot, extra, words, seed, P=50, pos32=False):
    x = [wl.draw_ring((rows, heads, dim), seed + k) for k in range(2)]
    g = [wl.draw_ring((rows, heads, dim), seed + 2 + k) for k in range(2)]
    r = [wl.draw_ring((rows, heads), seed + 4 + k) for k in range(2)]
    angles, dev = {}, {}
    if rot:
        rng = np.random.default_rng(seed)
        pos = rng.integers(0, P, rows)
        pos[rng.random(rows) < 0.15] = rng.choice([-1, P, -2 ** 31, 2 ** 31 - 1])
        angles = {"cos": wl.draw_ring((P, rot // 2), seed + 6), "sin": wl.draw_ring((P, rot // 2), seed + 7), "pos": pos}
        dev = {k: cg.to_device(angles[k]) for k in ("cos", "sin")}
        dev["pos"] = torch.from_numpy(pos).cuda().to(torch.int32 if pos32 else torch.int64)
    return x, g, r, angles, dev


@pytest.mark.parametrize("rows,heads,dim,rot,extra,words", SHAPES)
def test_sums_of_squares(cg, ro, wl, rows, heads, dim, rot, extra, words):
    say(f"sums of squares {rows} x {heads} x {dim}, {extra} between rows, {words} off")
    x = [wl.draw_ring((rows, heads, dim), 200 + k) for k in range(2)]
    z = Guarded((rows, heads), words)
    cg.cg_share_head_sq_sum(*(packed(cg, a, extra, words) for a in x), z_i=z.t)
    want = ro.head_sq_sum(*x)
    assert np.array_equal(z.host(), want), first_mismatch(z.host(), want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,rot,extra,words", SHAPES)
def test_norm_and_rotation(cg, ro, wl, rows, heads, dim, rot, extra, words, interleaved):
    say(f"norm and rotation {rows} x {heads} x {dim}, {rot} turned, {extra} between rows, {words} off, interleaved {interleaved}")
    x, _, r, angles, dev = case(cg, wl, rows, heads, dim, rot, extra, words, 210, pos32=interleaved)
    z = GuardedRows(rows, heads, dim, extra + (dim == 96), words)
    cg.cg_share_head_norm_rotate(*(packed(cg, a, extra, words) for a in x), *(cg.to_device(a) for a in r), **dev, frac_bits=FRAC,
                                 interleaved=interleaved, z_i=z.t)
    want = ro.head_norm_rotate(*x, *r, **angles, frac_bits=FRAC, interleaved=interleaved)
    assert np.array_equal(z.host(), want), first_mismatch(z.host(), want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,rot,extra,words", SHAPES)
def test_gradient(cg, ro, wl, rows, heads, dim, rot, extra, words, interleaved):
    say(f"head gradient {rows} x {heads} x {dim}, {rot} turned, {extra} between rows, {words} off, interleaved {interleaved}")
    x, g, r, angles, dev = case(cg, wl, rows, heads, dim, rot, extra, words, 220, pos32=not interleaved)
    dx, dr = GuardedRows(rows, heads, dim, extra, words), Guarded((rows, heads), words)
    cg.cg_share_head_norm_rotate_grad(*(packed(cg, a, 2 * extra, words) for a in g), *(packed(cg, a, extra, words) for a in x),
                                      *(cg.to_device(a) for a in r), **dev, frac_bits=FRAC, interleaved=interleaved, dx_i=dx.t, dr_i=dr.t)
    want = ro.head_norm_rotate_grad(*g, *x, *r, **angles, frac_bits=FRAC, interleaved=interleaved)
    for got, w in zip((dx.host(), dr.host()), want):
        assert np.array_equal(got, w), first_mismatch(got, w)


@pytest.mark.parametrize("frac", [0, 1, 40, 63])
def test_without_angles_and_at_every_scale(cg, ro, wl, frac):
    x, g, r, _, _ = case(cg, wl, 6, 3, 10, 0, 0, 0, 230)
    dev = [[cg.to_device(a) for a in pair] for pair in (g, x, r)]
    assert np.array_equal(cg.to_host(cg.cg_share_head_norm_rotate(*dev[1], *dev[2], frac_bits=frac)), ro.head_norm_rotate(*x, *r, frac_bits=frac))
    for got, want in zip(cg.cg_share_head_norm_rotate_grad(*dev[0], *dev[1], *dev[2], frac_bits=frac), ro.head_norm_rotate_grad(*g, *x, *r, frac_bits=frac)):
        assert np.array_equal(cg.to_host(got), want)


def test_no_rows(cg):
    none = torch.empty((0, 3, 8), dtype=torch.int64, device="cuda")
    r = torch.empty((0, 3), dtype=torch.int64, device="cuda")
    cos = torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    pos = torch.empty(0, dtype=torch.int64, device="cuda")
    assert cg.cg_share_head_sq_sum(none, none).shape == (0, 3)
    assert cg.cg_share_head_norm_rotate(none, none, r, r, cos, cos, pos).shape == (0, 3, 8)
    assert cg.cg_share_head_norm_rotate_grad(none, none, none, none, r, r, cos, cos, pos)[1].shape == (0, 3)


def test_rows_beyond_32_bit_offsets(cg):
    """Rows that lie so far apart that the last ones begin behind 2^33 bytes."""
    rows, heads, dim, ld = 5, 2, 8, 1 << 28
    say("heads in rows of 2^31 bytes")
    flat = torch.zeros((rows * ld,), dtype=torch.int64, device="cuda")
    x = flat.as_strided((rows, heads, dim), (ld, dim, 1))
    x.copy_(torch.arange(rows * heads * dim, device="cuda").view(rows, heads, dim))
    want = (x * (3 * x)).sum(-1)
    assert torch.equal(cg.cg_share_head_sq_sum(x, x), want)
    r = torch.full((rows, heads), 7, dtype=torch.int64, device="cuda")
    assert torch.equal(cg.cg_share_head_norm_rotate(x, x, r, r), x * 21)
    dx, dr = cg.cg_share_head_norm_rotate_grad(x, x, x, x, r, r)
    assert torch.equal(dx, x * 21) and torch.equal(dr, want)


def test_heads_in_a_graph(cg, ro, wl):
    """Forward and gradient captured on a stream, replayed with new inputs and the program's own work in between."""
    rows, heads, dim, rot = 12, 5, 64, 32
    x, g, r, angles, dev = case(cg, wl, rows, heads, dim, rot, 0, 0, 240)
    t = [[cg.to_device(a) for a in pair] for pair in (x, g, r)]
    kw = dict(dev, frac_bits=FRAC, interleaved=True)
    cg.cg_share_head_norm_rotate_grad(*t[1], *t[0], *t[2], **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sq, z = cg.cg_share_head_sq_sum(*t[0]), cg.cg_share_head_norm_rotate(*t[0], *t[2], **kw)
        dx, dr = cg.cg_share_head_norm_rotate_grad(*t[1], *t[0], *t[2], **kw)
    for turn in range(4):
        x, g, r, _, _ = case(cg, wl, rows, heads, dim, rot, 0, 0, 250 + 10 * turn)
        for pair, host in zip(t, (x, g, r)):
            for a, h in zip(pair, host):
                a.copy_(cg.to_device(h))
        graph.replay()
        _ = cg.cg_share_head_sq_sum(*t[1])
        if turn % 2:
            torch.cuda.synchronize()
        kh = dict(angles, frac_bits=FRAC, interleaved=True)
        wants = (ro.head_sq_sum(*x), ro.head_norm_rotate(*x, *r, **kh), *ro.head_norm_rotate_grad(*g, *x, *r, **kh))
        for got, want in zip((sq, z, dx, dr), wants):
            assert np.array_equal(cg.to_host(got), want), first_mismatch(cg.to_host(got), want)
