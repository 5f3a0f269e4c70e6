"""The embedding gradient's own scratch memory, of less than a megabyte, where memory is short: the call goes without it."""
import numpy as np
import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("n", [1500, 4096, 20000])
def test_embedding_gradient_where_memory_is_short(monkeypatch, n):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from oracle import ring_oracle as ro
    from paper_2104_10949_amd import binding as cg, workloads as wl
    say(f"embedding gradient of {n} tokens where memory is short")
    V, D = 100, 16
    host, G = np.random.default_rng(n).integers(-1, V + 1, n), [wl.draw_ring((n, D), 600 + c) for c in range(2)]
    g, ids, d = [cg.to_device(h) for h in G], torch.from_numpy(host).cuda(), [torch.empty((V, D), dtype=torch.int64, device="cuda") for _ in range(2)]
    want = [ro.embedding_grad(h, host, V, 3) for h in G]
    need = cg.cg_share_embedding_grad_workspace_bytes(n, V, D)
    assert 0 < need <= cg.SCRATCH_SMALL

    def taken():
        for t in d:
            t.fill_(77)
        before, stats = torch.cuda.memory_allocated(), torch.cuda.memory_stats()
        torch.cuda.reset_peak_memory_stats()
        cg.cg_share_embedding_grad(*g, ids, V, 3, da=d[0], db=d[1])
        bytes_taken, after = torch.cuda.max_memory_allocated() - before, torch.cuda.memory_stats()
        assert all(after[k] == stats[k] for k in ("num_alloc_retries", "num_ooms"))
        for t, w in zip(d, want):
            assert np.array_equal(cg.to_host(t), w)
        return bytes_taken

    assert taken() >= need   # there is room
    total = torch.cuda.mem_get_info()[1]
    try:
        torch.cuda.set_per_process_memory_fraction(0.9)
        assert taken() == 0
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "mem_get_info", lambda device=None: (total // 8, total))
        assert taken() == 0
    assert taken() >= need
