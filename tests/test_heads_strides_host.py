"""Which strides the calls over heads take: where a dimension has one entry, its stride says nothing.  No GPU is used."""
import pytest

torch = pytest.importorskip("torch")


def heads(rows, count, dim, step=None, head=None):
    """[rows, heads, dim] words with `step` words from a row to the next and `head` from a head to the next."""
    step, head = count * dim if step is None else step, dim if head is None else head
    size = max(0, rows - 1) * step + max(0, count - 1) * head + dim
    return torch.zeros(size, dtype=torch.int64).as_strided((rows, count, dim), (step, head, 1))


@pytest.mark.parametrize("first,second,want", [
    (heads(1, 5, 4, step=32), heads(1, 5, 4), 20),            # the next token: a slice of the packed projection beside a whole tensor
    (heads(1, 5, 4), heads(1, 5, 4, step=32), 20),
    (heads(6, 1, 4), heads(6, 1, 4, head=99), 4),             # one head
    (heads(6, 1, 4, step=12, head=7), heads(6, 1, 4, step=12), 12),
    (heads(1, 1, 4, step=9, head=8), heads(1, 1, 4), 4),
    (heads(0, 3, 4, step=50), heads(0, 3, 4), 12),            # no rows
    (heads(3, 2, 1, step=8), heads(3, 2, 1, step=8).as_strided((3, 2, 1), (8, 1, 5)), 8),   # heads of one word
    (heads(3, 2, 4, step=16), heads(3, 2, 4, step=16), 16),
])
def test_pairs_whose_rows_are_equally_far_apart(first, second, want):
    from paper_2104_10949_amd import binding as b
    assert b._pair_step(first, second, first.shape) == want


@pytest.mark.parametrize("first,second", [
    (heads(2, 5, 4, step=32), heads(2, 5, 4)),                # two rows: they do lie differently far apart
    (heads(6, 1, 4), heads(6, 1, 4, step=5)),
    (heads(2, 3, 4), heads(2, 3, 4, step=24, head=8)),        # the second component's heads lie apart
    (heads(2, 3, 4, step=24, head=8), heads(2, 3, 4)),
    (heads(1, 3, 4), heads(1, 3, 4, head=8)),
    (heads(2, 3, 4), heads(2, 3, 8)[..., ::2]),
    (heads(2, 3, 4), heads(2, 4, 3)),
])
def test_pairs_that_no_single_step_describes(first, second):
    from paper_2104_10949_amd import binding as b
    with pytest.raises(ValueError):
        b._pair_step(first, second, first.shape)
