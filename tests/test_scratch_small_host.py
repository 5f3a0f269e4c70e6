"""Small scratch memory where memory is short: what the allocator would have to take for it, decided on the host.  No GPU is used."""
import pytest

from tests.test_scratch_host import TOTAL, card, takes  # noqa: F401

torch = pytest.importorskip("torch")

SIZES = [256, 5 << 10, 300 << 10, 1 << 20]


@pytest.fixture
def used(card, monkeypatch):  # noqa: F811
    """The card of a program that has begun to use it."""
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    return card


@pytest.mark.parametrize("nbytes", SIZES)
def test_small_scratch_is_taken_where_it_is_free(used, nbytes):
    assert takes(used, nbytes)
    used["free"] = TOTAL // 8 + (2 << 20)          # what the allocator takes from the card for small tensors
    assert takes(used, nbytes)


@pytest.mark.parametrize("nbytes", SIZES)
def test_no_small_scratch_is_asked_for_where_memory_is_short(used, nbytes):
    """The allocator would synchronise and release its whole cache before it says that there is none."""
    for free in (TOTAL // 8 + (2 << 20) - 1, TOTAL // 8, nbytes, 0):
        used["free"] = free
        assert not takes(used, nbytes)


@pytest.mark.parametrize("nbytes", SIZES)
def test_no_small_scratch_is_asked_for_by_a_program_that_limits_its_share(used, nbytes):
    used["fraction"] = 0.5
    assert not takes(used, nbytes)


def test_an_embedding_gradient_takes_none_where_memory_is_short(used):
    """The call that most often asks for little."""
    from paper_2104_10949_amd import binding as b
    need = b.cg_share_embedding_grad_workspace_bytes(4096, 100, 16)
    assert 0 < need <= b.SCRATCH_SMALL
    used["free"] = 1 << 20
    assert not takes(used, need)
