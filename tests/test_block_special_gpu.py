"""The block operators on the GPU where care is called for: vectors that should not matter and are not finite, gates far below zero, launches of the largest size."""
import pytest
import torch

from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
BAD = [float("inf"), float("-inf"), float("nan")]


def normal(seed, *shape, dtype=torch.bfloat16, std=1.0, mean=0.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)


def spoilt(seed, *shape, bad):
    """A vector with one value that is not finite in each of its rows."""
    t = normal(seed, *shape)
    t[..., 5] = bad
    return t


# two sequences with rows and one without, as in a batch of fixed size that is not full; D of one wave, and of several
OFFSETS = [0, 7, 7, 20]


@pytest.mark.parametrize("D", [64, 1032])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("wide", [False, True])
def test_no_branch_no_gate(D, bad, wide):
    """Without y x' is alpha x whatever gate and w_post hold, the sign of a zero too."""
    x = normal(1, 20, D, dtype=torch.float32 if wide else torch.bfloat16)
    x[3] = -0.0
    offsets = torch.tensor(OFFSETS, dtype=torch.int32, device=DEV)
    how = dict(offsets=offsets, post="rms", pre="rms", alpha=0.5, eps=EPS)
    want = rtl.residual_norm(x, **how)
    got = rtl.residual_norm(x, gate=spoilt(2, 3, D, bad=bad), w_post=spoilt(3, D, bad=bad), **how)
    assert torch.equal(got[0], x * 0.5) and bool(torch.signbit(got[0][3]).all())
    assert torch.equal(got[1], want[1]) and bool(torch.isfinite(got[1]).all())


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
