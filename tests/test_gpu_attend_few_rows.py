"""17 to 64 rows over few and many sequences, on both sides of the choice between blocks of 16 and of 128 rows."""
import pytest
import torch

from test_gpu_attend import TYPES, World

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", [32, 64, 80, 96, 128, 192])
@pytest.mark.parametrize("seqs,kv,heads", [(3, 2, 4), (150, 4, 8)])
def test_few_rows(seqs, kv, heads, dim, dtype):
    w = World([1 + 37 * i % 200 for i in range(seqs)], kv, dim, 23)
    w.queries([1 + 5 * i % 16 for i in range(seqs)], heads, dtype)           # up to 32 rows
    w.check(True)
    w.queries([20 + i % 13 for i in range(seqs)], heads, dtype)              # up to 64
    w.check(True, 50)
    w.check(False)
