"""The calls over heads without a turn, and on pairs whose components lie in memory in different ways that come to the same row step, against the
oracle, bit for bit."""
import numpy as np
import pytest

from tests.gpu_util import say
from tests.test_heads_strides_host import heads

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("rows,count,dim,first,second", [
    (1, 5, 8, dict(step=40 + 24), {}),                  # the next token: a slice of wider rows beside a whole tensor
    (1, 3, 5, {}, dict(step=16)),
    (6, 1, 8, {}, dict(head=100)),                      # one head
    (6, 1, 7, dict(step=9, head=50), dict(step=9)),
])
def test_components_that_lie_differently(rows, count, dim, first, second):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from oracle import ring_oracle as ro
    from paper_2104_10949_amd import binding as cg, workloads as wl
    say(f"heads {rows} x {count} x {dim}, {first} beside {second}")
    x, g = ([wl.draw_ring((rows, count, dim), seed + k) for k in range(2)] for seed in (500, 502))
    r = [wl.draw_ring((rows, count), 504 + k) for k in range(2)]
    cos, sin = (wl.draw_ring((10, dim // 2), 506 + k) for k in range(2))
    pos = np.arange(rows) % 10

    def place(pair, how):
        out = []
        for a, kw in zip(pair, how):
            t = heads(rows, count, dim, **kw)
            stored = torch.zeros(t.untyped_storage().nbytes() // 8, dtype=torch.int64, device="cuda").as_strided(t.shape, t.stride())
            stored.copy_(cg.to_device(a))
            out.append(stored)
        return out
    dx, dg = place(x, (first, second)), place(g, (second, first))
    dr = [cg.to_device(a) for a in r]
    dev = dict(cos=cg.to_device(cos), sin=cg.to_device(sin), pos=torch.from_numpy(pos).cuda())
    kw = dict(cos=cos, sin=sin, pos=pos, frac_bits=9)
    got = (cg.cg_share_head_sq_sum(*dx), cg.cg_share_head_norm_rotate(*dx, *dr, **dev, frac_bits=9),
           *cg.cg_share_head_norm_rotate_grad(*dg, *dx, *dr, **dev, frac_bits=9))
    want = (ro.head_sq_sum(*x), ro.head_norm_rotate(*x, *r, **kw), *ro.head_norm_rotate_grad(*g, *x, *r, **kw))
    for a, w in zip(got, want):
        assert np.array_equal(cg.to_host(a), w)


def test_angles_of_no_pairs_read_no_position():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from oracle import ring_oracle as ro
    from paper_2104_10949_amd import binding as cg, workloads as wl
    say("heads with angles of no pairs")
    x, r = [wl.draw_ring((4, 2, 6), 510 + k) for k in range(2)], [wl.draw_ring((4, 2), 512 + k) for k in range(2)]
    none, pos = torch.empty((9, 0), dtype=torch.int64, device="cuda"), torch.tensor([0, -1, 9, 3], device="cuda")
    dx, dr = [cg.to_device(a) for a in x], [cg.to_device(a) for a in r]
    z = cg.cg_share_head_norm_rotate(*dx, *dr, none, none, pos, frac_bits=5)
    assert np.array_equal(cg.to_host(z), ro.head_norm_rotate(*x, *r, frac_bits=5))
    for got, want in zip(cg.cg_share_head_norm_rotate_grad(*dx, *dx, *dr, none, none, pos, frac_bits=5), ro.head_norm_rotate_grad(*x, *x, *r, frac_bits=5)):
        assert np.array_equal(cg.to_host(got), want)
