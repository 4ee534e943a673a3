"""Windows and lengths as large as their type holds."""
import pytest
import torch

from test_gpu_attend import TYPES, World, compare, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30, 17])
@pytest.mark.parametrize("counts,lengths", [([4, 0, 40, 1], [0, 10, 3, 0]), ([1, 1], [500, 1]), ([150, 333], [100, 320])], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_windows_of_any_size_beside_queries_before_the_first_token(dtype, counts, lengths, window):
    w = World(lengths, 1, 64, 20)
    w.queries(counts, 2, dtype)
    w.check(True, window)


@pytest.mark.parametrize("counts", [[1], [150]], ids=str)
@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 65])
def test_a_length_beyond_all_pages(length, counts):
    """Tokens without a page do not exist: those of the table are seen, whatever the sequence's length is said to be."""
    w = World([500], 2, 64, 21)
    w.queries(counts, 4, torch.float32)
    q, t, s = w.q.cuda(), ints(w.table.tolist()), ints(w.starts.tolist())
    w.lengths = [512]                                    # the whole last page
    out, lse = w.c.attend(q, t, s, ints([length]), counts[0], length)
    compare(out, lse, *w.want(False), w)
    out, lse = w.c.attend(q, t, s, ints([length]), counts[0], length, causal=True)
    compare(out, lse, *w.want(False), w)
