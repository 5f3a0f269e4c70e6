"""The gradient norm opened the way a program has to: every party blinds its share before it is sent."""
import numpy as np
import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("sizes", [[1], [5, 0, 300], [70000, 3]])
def test_the_norm_opened_from_blinded_shares(sizes):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from oracle import ring_oracle as ro
    from paper_2104_10949_amd import binding as cg, workloads as wl
    say(f"blinded norm of {sizes}")
    keys, nonce, max_norm, f = [bytes([k + 1] * 16) for k in range(3)], 77, 3 << 16, 20
    plain = [wl.draw_ring((n,), 620 + k) for k, n in enumerate(sizes)]
    shared = [ro.share(p, wl.draw_ring(p.shape, 630 + 2 * k), wl.draw_ring(p.shape, 631 + 2 * k)) for k, p in enumerate(plain)]
    dev = [[cg.to_device(s) for s in sharing] for sharing in shared]
    lists = [cg.ShareList([d[i].clone() for d in dev], [d[(i + 1) % 3].clone() for d in dev]) for i in range(3)]
    own = [cg.cg_share_sq_norm(x) for x in lists]
    sent = [cg.cg_reshare(z, keys[i], keys[(i - 1) % 3], nonce) for i, z in enumerate(own)]
    for i, (z, s) in enumerate(zip(own, sent)):
        raw = ro.sq_norm([(a[i], a[(i + 1) % 3]) for a in shared])
        assert int(cg.to_host(z)[0]) == raw
        assert int(cg.to_host(s)[0]) == int(ro.reshare(np.array([raw], np.uint64), keys[i], keys[(i - 1) % 3], nonce, 0)[0]) != raw
    S = sum(int((p * p).sum(dtype=np.uint64)) for p in plain) % (1 << 64)
    want = ro.clip_factor(S, max_norm, f)
    for x in lists:
        c = cg.cg_clip_factor(*sent, max_norm, f)
        assert int(cg.to_host(c)[0]) == want
        cg.cg_share_clip(x, c)
    for k, p in enumerate(plain):
        if p.size:
            assert np.array_equal(cg.to_host(cg.cg_reconstruct(*(x.a[k] for x in lists))), p * np.uint64(want))
