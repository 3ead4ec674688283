"""The block operators on the GPU where care is called for: vectors that should not matter and are not finite, gates far below zero, launches of the largest size."""
import pytest
import torch

from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_zz_most_rows_of_wide_norms():
    """So many rows of more than 4096 columns that one launch would have 2^32 threads and more: each row is taken once."""
    T, D, step = (1 << 23) + 3, 4104, 1 << 20
    x = torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    mark = (torch.arange(T, device=DEV) % 255 + 1).to(torch.bfloat16)[:, None]
    for i in range(0, T, step):
        x[i:i + step] = mark[i:i + step]
    rtl.residual_norm(x, alpha=0.5, out=(x, None))
    for i in range(0, T, step):
        assert bool((x[i:i + step] == mark[i:i + step] * 0.5).all())
    del x
    torch.cuda.empty_cache()
