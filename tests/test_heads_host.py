"""Refusals of the embedding, head and clipping entry points, before any HIP call.  No GPU is used."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    from paper_2104_10949_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2104_10949_amd import build
        build.build()
    binding.lib()
    return binding


P = 1 << 32   # fake "device" addresses, far apart; never dereferenced


def test_embedding_validation(b):
    f = b.lib().cg_share_embedding
    ok = dict(ta=P, tb=2 * P, ids=3 * P, w=8, alpha=1, za=4 * P, zb=5 * P, n=4, V=10, D=6)

    def call(**kw):
        return f(*{**ok, **kw}.values(), None)
    for name in ("ta", "tb", "ids", "za", "zb"):
        assert call(**{name: 0}) == b.CG_ERR_NULL
        assert call(**{name: 3 * P + (4 if name == "ids" else 4)}) == b.CG_ERR_ALIGN
    assert call(ids=3 * P + 2, w=4) == b.CG_ERR_ALIGN
    for bad in (dict(V=0), dict(D=0), dict(w=2), dict(w=0), dict(n=1 << 40, D=1 << 40), dict(V=1 << 40, D=1 << 30)):
        assert call(**bad) == b.CG_ERR_SHAPE
    assert call(n=1 << 31, D=1) == b.CG_ERR_UNSUPPORTED
    assert call(V=1 << 31, D=1) == b.CG_ERR_UNSUPPORTED
    assert call(D=(1 << 22) + 1) == b.CG_ERR_UNSUPPORTED
    for bad in (dict(za=P + 8), dict(zb=2 * P + 10 * 6 * 8 - 8), dict(za=5 * P), dict(za=5 * P + 4 * 6 * 8 - 8), dict(zb=3 * P + 24)):
        assert call(**bad) == b.CG_ERR_ALIAS
    assert call(n=0, ids=0, za=0, zb=0, ta=0, tb=0) == b.CG_OK
    assert call(n=0, V=0) == b.CG_ERR_SHAPE


def test_embedding_gradient_validation(b):
    f = b.lib().cg_share_embedding_grad
    ok = dict(ga=P, gb=2 * P, ids=3 * P, w=4, alpha=1, da=4 * P, db=5 * P, n=4, V=10, D=6, acc=0, ws=0, bytes=0)

    def call(**kw):
        return f(*{**ok, **kw}.values(), None)
    for name in ("ga", "gb", "ids", "da", "db"):
        assert call(**{name: 0}) == b.CG_ERR_NULL
        assert call(**{name: 6 * P + 2}) == b.CG_ERR_ALIGN
    for bad in (dict(V=0), dict(D=0), dict(w=1), dict(acc=2), dict(acc=-1), dict(V=1 << 40, D=1 << 40)):
        assert call(**bad) == b.CG_ERR_SHAPE
    assert call(n=1 << 31, D=1) == b.CG_ERR_UNSUPPORTED
    for bad in (dict(da=P), dict(db=2 * P + 4 * 6 * 8 - 8), dict(da=5 * P + 8), dict(da=3 * P + 8)):
        assert call(**bad) == b.CG_ERR_ALIAS
    assert call(n=0, acc=1, da=0) == b.CG_ERR_NULL
    # scratch memory that would be used and lies in an operand
    need = b.cg_share_embedding_grad_workspace_bytes
    n, V, D = 20000, 500, 6
    assert need(n, V, D) > 8 * n
    for where in (P, 2 * P + n * D * 8 - 16, 3 * P + 16, 4 * P, 5 * P - need(n, V, D) + 16):
        assert call(n=n, V=V, D=D, ws=where, bytes=need(n, V, D)) == b.CG_ERR_ALIAS
    assert need(0, 5, 5) == need(5000, 0, 5) == need(5000, 5, 0) == need(1 << 31, 5, 5) == need(5000, 5, (1 << 22) + 1) == 0
    assert need(1024, 1 << 18, 5) == 0 < min(need(1025, 5, 5), need(1024, (1 << 18) + 1, 5))
    assert need(2048, 5, 512, True) == need(1, 1 << 30, 9, True) == 0 < min(need(2049, 5, 5, True), need(2048, 5, 513, True))


def desc(b, **kw):
    base = dict(rows=4, heads=3, dim=8, rot=6, ld_x=24, ld_g=24, ld_out=24, positions=16, pos_bytes=8, frac_bits=14, interleaved=0)
    return ctypes.byref(b.HeadDesc(**{**base, **kw}))


BAD_DESC = [dict(rows=-1), dict(heads=0), dict(dim=0), dict(rot=5), dict(rot=10), dict(rot=-2), dict(ld_x=23), dict(ld_out=23), dict(positions=0),
            dict(positions=1 << 60), dict(pos_bytes=2), dict(frac_bits=64), dict(frac_bits=-1), dict(interleaved=2), dict(ld_x=1 << 62), dict(ld_out=-24),
            dict(rows=1 << 40, heads=1 << 30)]


def test_head_validation(b):
    L = b.lib()
    f, g, q = L.cg_share_head_norm_rotate, L.cg_share_head_norm_rotate_grad, L.cg_share_head_sq_sum
    fw = [k * P for k in range(1, 9)]     # x_i x_ip1 r_i r_ip1 cos sin pos z
    bw = [k * P for k in range(1, 12)]    # g_i g_ip1 x_i x_ip1 r_i r_ip1 cos sin pos dx dr
    for call, ptrs in ((f, fw), (g, bw)):
        assert call(*ptrs, None, None) == b.CG_ERR_NULL
        for k in range(len(ptrs)):
            assert call(*ptrs[:k], 0, *ptrs[k + 1:], desc(b), None) == b.CG_ERR_NULL
            assert call(*ptrs[:k], ptrs[k] + 4, *ptrs[k + 1:], desc(b), None) == b.CG_ERR_ALIGN
        for bad in BAD_DESC:
            assert call(*ptrs, desc(b, **bad), None) == b.CG_ERR_SHAPE, bad
        assert call(*ptrs, desc(b, rows=1 << 30, heads=2, ld_x=24, ld_out=24), None) == b.CG_ERR_UNSUPPORTED
        assert call(*ptrs, desc(b, rows=0), None) == b.CG_OK
        assert call(*[0] * len(ptrs), desc(b, rows=0), None) == b.CG_OK
        outs = range(len(ptrs) - (2 if call is g else 1), len(ptrs))
        for o in outs:
            for k in range(len(ptrs)):
                if k != o:                 # an output that begins at any other operand
                    assert call(*ptrs[:o], ptrs[k], *ptrs[o + 1:], desc(b), None) == b.CG_ERR_ALIAS, (o, k)
    assert g(*bw, desc(b, ld_g=23), None) == b.CG_ERR_SHAPE
    # the extent of rows that lie apart counts to the last word
    assert f(*fw[:7], P + (3 * 100 + 24) * 8 - 8, desc(b, ld_x=100), None) == b.CG_ERR_ALIAS
    assert q(P, 2 * P, 0, 4, 3, 8, 24, None) == b.CG_ERR_NULL
    assert q(P, 2 * P + 4, 3 * P, 4, 3, 8, 24, None) == b.CG_ERR_ALIGN
    assert q(P, 2 * P, P + 8, 4, 3, 8, 24, None) == b.CG_ERR_ALIAS
    assert q(P, 2 * P, 3 * P, 4, 3, 8, 23, None) == b.CG_ERR_SHAPE
    assert q(P, 2 * P, 3 * P, 4, 0, 8, 24, None) == b.CG_ERR_SHAPE
    assert q(P, 2 * P, 3 * P, 1 << 30, 2, 1, 2, None) == b.CG_ERR_UNSUPPORTED
    assert q(0, 0, 0, 0, 3, 8, 24, None) == b.CG_OK


def arrays(*lists):
    return [(ctypes.c_void_p * len(v))(*v) for v in lists]


def sizes(*n):
    return (ctypes.c_size_t * len(n))(*n)


def test_norm_and_clip_validation(b):
    L = b.lib()
    norm, clip, factor = L.cg_share_sq_norm, L.cg_share_clip, L.cg_clip_factor
    xa, xb, za, zb = arrays([P, 2 * P], [3 * P, 4 * P], [5 * P, 6 * P], [7 * P, 8 * P])
    n = sizes(10, 20)
    assert norm(xa, xb, n, 2, 0, None) == b.CG_ERR_NULL
    assert norm(xa, xb, n, 2, 9 * P + 4, None) == b.CG_ERR_ALIGN
    assert norm(None, xb, n, 2, 9 * P, None) == b.CG_ERR_NULL
    assert norm(xa, xb, None, 2, 9 * P, None) == b.CG_ERR_NULL
    assert norm(xa, arrays([3 * P, 0])[0], n, 2, 9 * P, None) == b.CG_ERR_NULL
    assert norm(xa, arrays([3 * P, 4 * P + 2])[0], n, 2, 9 * P, None) == b.CG_ERR_ALIGN
    assert norm(xa, xb, n, 2, 4 * P + 19 * 8, None) == b.CG_ERR_ALIAS
    assert norm(xa, xb, sizes(10, 1 << 62), 2, 9 * P, None) == b.CG_ERR_SHAPE
    assert clip(xa, xb, 0, za, zb, n, 2, None) == b.CG_ERR_NULL
    assert clip(xa, xb, 9 * P + 1, za, zb, n, 2, None) == b.CG_ERR_ALIGN
    assert clip(xa, xb, 9 * P, None, zb, n, 2, None) == b.CG_ERR_NULL
    assert clip(xa, xb, 6 * P + 8, za, zb, n, 2, None) == b.CG_ERR_ALIAS                          # the factor inside an output
    for bad in ([5 * P, 5 * P + 72], [5 * P, 5 * P], [5 * P, 7 * P], [5 * P, P + 8], [P + 8, 6 * P], [3 * P, 6 * P], [2 * P, 6 * P]):
        assert clip(xa, xb, 9 * P, arrays(bad)[0], zb, n, 2, None) == b.CG_ERR_ALIAS, bad
    assert clip(*arrays([P, P], [3 * P, 4 * P]), 9 * P, *arrays([P, P], [7 * P, 8 * P]), sizes(10, 10), 2, None) == b.CG_ERR_ALIAS  # twice in place
    # in place over the other entry's input, an output before the one in front of it, inputs between outputs
    assert clip(*arrays([P, 2 * P], [3 * P, 4 * P]), 9 * P, *arrays([2 * P, P], [7 * P, 8 * P]), n, 2, None) == b.CG_ERR_ALIAS
    assert clip(*arrays([P, 2 * P], [3 * P, 4 * P]), 9 * P, *arrays([6 * P, 6 * P - 152], [7 * P, 8 * P]), n, 2, None) == b.CG_ERR_ALIAS
    assert clip(*arrays([P, 2 * P], [3 * P, 4 * P]), 9 * P, *arrays([P, 2 * P], [3 * P + 8, 8 * P]), n, 2, None) == b.CG_ERR_ALIAS
    assert clip(*arrays([P, 2 * P], [3 * P, 4 * P]), 9 * P, *arrays([P, 2 * P], [P + 80 - 8, 8 * P]), n, 2, None) == b.CG_ERR_ALIAS
    assert clip(None, None, 9 * P, None, None, None, 0, None) == b.CG_OK
    assert clip(xa, xb, 9 * P, za, zb, sizes(0, 0), 2, None) == b.CG_OK
    assert factor(P, 2 * P, 3 * P, 1, 16, 0, None) == b.CG_ERR_NULL
    assert factor(P, 2 * P, 3 * P + 4, 1, 16, 4 * P, None) == b.CG_ERR_ALIGN
    for bad in ((1, 63), (1, -1), (1 << 48, 16), ((1 << 64) - 1, 1)):
        assert factor(P, 2 * P, 3 * P, *bad, 4 * P, None) == b.CG_ERR_SHAPE


def test_binding_refuses_what_the_library_cannot_see(b, monkeypatch):
    i64 = dict(dtype=torch.int64)
    t, ids = torch.zeros((4, 6), **i64), torch.zeros(3, **i64)
    for call in (lambda: b.cg_share_embedding(t, t, ids), lambda: b.cg_share_embedding_grad(t[:3], t[:3], ids, 4),
                 lambda: b.cg_share_head_sq_sum(torch.zeros((2, 3, 4), **i64), torch.zeros((2, 3, 4), **i64)),
                 lambda: b.ShareList([t], [t])):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):      # CPU tensors
            call()
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(b, "_device", lambda: 1)

    class Elsewhere:
        device = "cuda:0"

        def get_device(self):
            return 0
    with pytest.raises(ValueError, match="current GPU"):
        b._current(Elsewhere())
    with pytest.raises(ValueError, match="current GPU"):
        b._ptrs(t)
    with pytest.raises(TypeError):
        b._index_ptr(torch.zeros(3, dtype=torch.int16))
    with pytest.raises(ValueError):
        b.cg_share_embedding(t, t[:3], ids)
    with pytest.raises(ValueError):
        b.cg_share_embedding_grad(t, t, ids, 4)                              # 4 rows of gradient for 3 ids
    with pytest.raises(ValueError):
        b.cg_share_embedding_grad(t[:3], t[:3], ids, 4, accumulate=True)     # nothing to add to
    x = torch.zeros((2, 3, 4), **i64)
    with pytest.raises(TypeError):
        monkeypatch.setattr(b, "_current", lambda *tensors: None)
        b._ring_ptrs(x, x.int())
    for bad in (x.transpose(0, 1), x[..., ::2], x.reshape(6, 4)):
        with pytest.raises(ValueError):
            b._pair_step(bad, bad, bad.shape)
    with pytest.raises(ValueError):
        b._pair_step(x, torch.zeros((2, 5, 4), **i64)[:, :3], x.shape)       # rows not equally far apart
    with pytest.raises(ValueError):
        b._pair_step(x, x[:1], x.shape)
    assert b._row_step(torch.zeros((2, 5, 4), **i64)[:, 1:4]) == 20
    assert b._row_step(torch.zeros((1, 5, 4), **i64)[:, 1:4]) == 12          # one row: nothing to be apart from
    with pytest.raises(ValueError):
        b.ShareList([t], [t[:2]])
    with pytest.raises(ValueError):
        b.cg_clip_factor(t[0, :1], t[0, :1], t[0, :2], 1, 16)


def test_small_scratch_is_taken_without_asking_how_much_is_free(b, monkeypatch):
    asked, real_empty = [], torch.empty
    monkeypatch.setattr(b, "_scratch_fits", lambda nbytes, device: asked.append(nbytes) or True)
    monkeypatch.setattr(b, "_exchange_capture_mode", lambda mode: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch, "empty", lambda n, dtype=None, device=None: real_empty(n, dtype=dtype))
    device = torch.device("cuda", 0)
    assert b._scratch(b.SCRATCH_SMALL, device, None).numel() == b.SCRATCH_SMALL and asked == []
    assert b._scratch(b.SCRATCH_SMALL + 1, device, None) is not None and asked == [b.SCRATCH_SMALL + 1]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert b._scratch(b.SCRATCH_SMALL, device, None) is None
