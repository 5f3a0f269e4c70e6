"""Calls so large that a grid is capped and its blocks go round again: embedding lookup, its gradient (sums and both ways of
clearing) and the heads' calls, every word checked against plain 64-bit arithmetic on the GPU."""
import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

CHUNK = 1 << 20   # rows that are checked at a time


@pytest.fixture(scope="module")
def cg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2104_10949_amd import binding
    return binding


@pytest.fixture(autouse=True)
def memory_goes_back():
    yield
    if torch.cuda.is_available():
        torch.cuda.empty_cache()


def words(*shape):
    """Words that differ, each, from every other."""
    n = 1
    for s in shape:
        n *= s
    return torch.arange(1, n + 1, dtype=torch.int64, device="cuda").mul_(0x1E3779B97F4A7C15).view(shape)


def spread(n, V):
    """n ids, all different and in no order, n <= V."""
    step = 7919
    while V % step == 0:
        step += 2
    return torch.arange(n, dtype=torch.int64, device="cuda").mul_(step).remainder_(V)


# rows of 33 words take a wave each, four to a block: 2^22 blocks have 2^24 rows
def test_lookup_of_more_rows_than_the_grid_has(cg):
    n, V, D = (1 << 24) + 70001, 1000, 33
    say(f"lookup of {n} rows")
    T = words(2, V, D)
    ids = spread(V, V).repeat(n // V + 1)[:n].int()
    ids[1::1000] = -1
    za, zb = cg.cg_share_embedding(T[0], T[1], ids, 5)
    for t, z in zip(T, (za, zb)):
        t = torch.cat((t * 5, torch.zeros_like(t[:1])))   # the last row is padding's
        for at in range(0, n, CHUNK):
            assert torch.equal(z[at:at + CHUNK], t[ids[at:at + CHUNK].long()])


# (n, V, D): few and middling tokens, in tables of 16-byte and of 8-byte accesses, of more than 2048 blocks' clearing
@pytest.mark.parametrize("n,V,D", [(700, 200001, 400), (700, 200001, 201), (3000, 200003, 700), (3000, 200003, 351)])
def test_clearing_of_large_tables(cg, n, V, D):
    say(f"gradient of {n} tokens of {V} x {D}")
    assert V * (D // 2 if D % 2 == 0 else D) > 2048 * (512 if n <= 1024 else 1024) // 64 * 2048
    g, ids = words(2, n, D), spread(n, V)
    ids[n // 2:] = (ids[:n - n // 2] + (torch.arange(n - n // 2, device="cuda") % 3 == 0)).clamp(max=V - 1)   # rows of several tokens
    ids = torch.where(torch.arange(n, device="cuda") % 11 == 0, V - 1, ids)
    d = [torch.full((V, D), 77, dtype=torch.int64, device="cuda") for _ in range(2)]
    ws = torch.empty(cg.cg_share_embedding_grad_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    cg.cg_share_embedding_grad(g[0], g[1], ids, V, 3, da=d[0], db=d[1], workspace=ws)
    for rows, out in zip(g, d):
        want = torch.zeros((V, D), dtype=torch.int64, device="cuda")
        for j, v in enumerate(ids.tolist()):
            want[v] += rows[j] * 3
        assert torch.equal(out, want)


# (n, D): a wave per row and piece, two pieces; half a wave per row.  2^22 blocks have 2^24 waves, 2^25 halves.
@pytest.mark.parametrize("n,D", [((1 << 23) + 5003, 129), ((1 << 25) + 5003, 33)])
def test_more_sums_than_the_grid_has(cg, n, D):
    V = n + 3
    say(f"gradient of {n} tokens of {V} x {D}")
    buffer = words(n * D + 1)
    g, ids = [buffer[c:c + n * D].view(n, D) for c in range(2)], spread(n, V)
    d = [torch.full((V, D), 77, dtype=torch.int64, device="cuda") for _ in range(2)]
    ws = torch.empty(cg.cg_share_embedding_grad_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    cg.cg_share_embedding_grad(*g, ids, V, 3, da=d[0], db=d[1], workspace=ws)
    empty = torch.ones(V, dtype=torch.bool, device="cuda")
    empty[ids] = False
    assert int(empty.sum()) == 3
    for rows, out in zip(g, d):
        assert not bool(out[empty].any())
        for at in range(0, n, CHUNK):
            assert torch.equal(out[ids[at:at + CHUNK]], rows[at:at + CHUNK] * 3)


# 129 words take a wave each: 2^22 blocks have 2^24 heads
def test_more_heads_to_sum_than_the_grid_has(cg):
    rows, heads, dim = (1 << 23) + 2001, 2, 129
    say(f"sums of squares of {rows} x {heads} x {dim}")
    x = words(rows, heads, dim)
    z = cg.cg_share_head_sq_sum(x, x)
    for at in range(0, rows, CHUNK):
        c = x[at:at + CHUNK]
        assert torch.equal(z[at:at + CHUNK], (c * c).sum(-1) * 3)


def test_more_heads_to_scale_than_the_grid_has(cg):
    rows, heads, dim, f = (1 << 23) + 2001, 2, 33, 7
    say(f"product of {rows} x {heads} x {dim} and a word per head")
    x, r = words(rows, heads, dim), words(2, rows, heads)
    z = cg.cg_share_head_norm_rotate(x, x, r[0], r[1], frac_bits=f)
    for at in range(0, rows, CHUNK):
        part = slice(at, at + CHUNK)
        assert torch.equal(z[part], x[part] * (2 * r[0, part] + r[1, part])[..., None] * (1 << f))


def test_more_head_gradients_than_the_grid_has(cg):
    rows, heads, dim, P = (1 << 23) + 2001, 2, 66, 11
    half = dim // 2
    say(f"gradient of {rows} x {heads} x {dim}, all turned")
    x, r, angles = words(rows, heads, dim), words(2, rows, heads), words(2, P, half)
    pos = torch.arange(rows, device="cuda").remainder_(P).int()
    dx, dr = cg.cg_share_head_norm_rotate_grad(x, x, x, x, r[0], r[1], angles[0], angles[1], pos, frac_bits=3)
    for at in range(0, rows, CHUNK):
        part = slice(at, at + CHUNK)
        c, s = (a[pos[part].long()][:, None] for a in angles)
        x1, x2 = x[part, :, :half], x[part, :, half:]
        v = torch.cat((x1 * c + x2 * s, x2 * c - x1 * s), -1)
        assert torch.equal(dx[part], v * (2 * r[0, part] + r[1, part])[..., None])
        assert torch.equal(dr[part], (x[part] * v).sum(-1) * 3)
