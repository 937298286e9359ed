"""ssn_logprobs where the ends decide: rows whose weight lies in their first and last columns, beside the borders between the
lanes', waves' and workgroups' shares, or in the reference class, so that a class lost or counted twice there moves the results by
more than roundings do.  The comparison and its tolerances are those of test_gpu_logprobs.py: log-sum-exp to (C / 64 + 64) u, 1.3e-4
at 131077 classes and 2.5e-4 at 262147, where the least that one of the heavy classes weighs is 2.8e-4."""
import numpy as np
import pytest
import torch

from paper_1802_09113_amd.binding import ssn_logprobs, ssn_logprobs_grad
from tests.test_gpu_logprobs import DTYPES, check, some_labels

pytestmark = pytest.mark.gpu


# one wave to a row, four, eight, sixteen, and rows of several workgroups; C odd, not a multiple of any vector
@pytest.mark.parametrize("n,C", [(6, 517), (2100, 3001), (600, 9001), (300, 9001), (200, 9001), (6, 40003), (6, 70001), (6, 131077), (6, 262147)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_ends(dtype, n, C):
    rng = np.random.default_rng(C)
    dt = DTYPES[dtype]
    for reference in (False, True):
        width = C - reference
        tail = 1 + rng.integers(0, 7, n)                             # columns at the end that a partial vector may hold
        h = np.full((n, width), -40.0) + rng.integers(-8, 9, (n, width)) / 4
        edge = np.zeros(width, dtype=bool)
        edge[::128], edge[127::128] = True, True                     # beside every border between shares: multiples of 128
        if C < 135000:
            h[0::6, edge] = rng.integers(-4, 5, (len(h[0::6]), edge.sum())) / 8
        else:
            h[0::6, edge] = np.where(np.arange(edge.sum()) % 2, -40.0, rng.integers(-4, 5, (len(h[0::6]), edge.sum())) / 8)
        for i in range(1, n):
            if i % 6 == 1:
                h[i, -tail[i]:] = rng.integers(-8, 9, tail[i]) / 8   # the last columns
            elif i % 6 == 2:
                h[i, :tail[i]] = rng.integers(-8, 9, tail[i]) / 8    # the first ones
            elif i % 6 == 3 and reference:
                h[i] -= 10.0                                         # the reference class alone
            elif i % 6 == 4:
                h[i, -1] = 1.0                                       # the last column against the first
                h[i, 0] = 0.5
        mask = np.ones((n, C), dtype=bool)
        mask[5::6, :] = False                                        # only the last classes may be answered with
        for i in range(5, n, 6):
            mask[i, -tail[i]:] = True
        Zh = torch.from_numpy(h).to(dt).double().numpy()
        Zd = torch.from_numpy(h).to(dt).cuda()
        y = some_labels(n, 3, C, rng)
        y[:, 0], y[:, 1] = C - 1, C - tail
        check(Zd, Zh, y, 9, reference, None, grad=n <= 300)
        check(Zd, Zh, y, 0, reference, mask, grad=n <= 300)


@pytest.mark.parametrize("n,C", [(3, 400), (3, 5000), (2, 70001), (300, 9000)])
def test_alternatives_of_rows_full_of_ties_in_double(n, C):
    rng = np.random.default_rng(12)
    h = rng.integers(-3, 3, (n, C)).astype(np.float64)
    check(torch.from_numpy(h).cuda(), h, some_labels(n, 1, C, rng), min(64, C), False, None, grad=False)


@pytest.mark.parametrize("C", [9, 300, 3000])
def test_an_index_that_is_no_class_in_a_row_without_a_class(C):
    """The row's gradient is zero, at its allowed classes too; in a row with a class it is NaN."""
    Z = torch.randn(3, C, device="cuda")
    Z[0] = -float("inf")
    mask = torch.full((3, -(-C // 32)), -1, dtype=torch.int32, device="cuda")
    mask[1] = 0
    lab = torch.full((3, 2), C, dtype=torch.int32, device="cuda")
    out = ssn_logprobs(Z, lab, allowed=mask)
    assert bool(torch.isnan(out["logp"]).all())
    dZ = ssn_logprobs_grad(Z, lab, out, dlogp=torch.ones(3, 2, device="cuda"), dlse=torch.ones(3, device="cuda"), allowed=mask)
    assert bool((dZ[:2] == 0).all()) and bool(torch.isnan(dZ[2]).all())
