"""Blocks of so many classes that the threads of one launch over them would pass 2^32: laid out and multiplied stretch by stretch.

Weights are six times a power of two, whose scale and code are exact, and rows hold small integers: margins are exact.  Of two
weights in one group the smaller goes to the magnitude nearest to its share of the scale, by the header's rule."""
import pytest
import torch

from paper_1802_09113_amd.binding import ssn_q4_margins, ssn_q4_quantize

pytestmark = pytest.mark.gpu


def weight_of(c):
    return torch.where(c % 3 == 1, -6.0, 6.0) * torch.exp2((c % 7).float())


def weights_of(c, p):
    """The weights of the first and the last feature that classes c are multiplied with."""
    first, end = weight_of(c), weight_of(c + 2)
    if p <= 128:                                         # one group of 128 features: the scale is the larger one's
        s = torch.maximum(first.abs(), end.abs()) / 6
        sizes = torch.tensor([6, 3, 1.5, 1, 0.5, 0, 0], device=c.device)      # of 6, 3, 1.5, 0.75 (a tie), 0.375, 0.1875, 0.09375
        first, end = (torch.sign(w) * s * sizes[torch.log2(6 * s / w.abs()).round().long()] for w in (first, end))
    return first, end


# classes; n = 16 takes 512 threads for 64 classes, n = 40 in float 256 for 16 rows by 128 classes
@pytest.mark.parametrize("K,p,dtype,rows", [((1 << 29) + 37, 1, "bf16", (1, 9)), ((1 << 26) + 37, 128, "f32", (3, 40)),
                                            ((1 << 26) + 37, 130, "f16", (6, 20))])
def test_more_classes_than_one_launch(K, p, dtype, rows):
    if torch.cuda.mem_get_info()[0] < 80e9:
        pytest.skip("needs 80 GB of device memory")
    dt, last, step = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)[dtype], p - 1, 1 << 26
    W = torch.zeros(p if p == 1 else 2, K, device="cuda", dtype=dt)
    for lo in range(0, K, step):
        c = torch.arange(lo, min(lo + step, K), device="cuda")
        W[0, lo:lo + step] = weight_of(c).to(dt)
        if p > 1:
            W[1, lo:lo + step] = weight_of(c + 2).to(dt)
    if p > 1:                                            # features between the first and the last: zero, in memory once
        full = torch.zeros(p, K, device="cuda", dtype=dt)
        full[0], full[last] = W[0], W[1]
        W = full
    block = ssn_q4_quantize(W, 128)
    del W
    for n in rows:
        print(f"[case] n={n} p={p} K={K} {dtype}", flush=True)
        X = torch.randint(-3, 4, (n, p), device="cuda").to(dt)
        Z = torch.full((n + 1, K), 7.0, device="cuda", dtype=dt)
        ssn_q4_margins(block, X, Z[:n])
        for lo in range(0, K, step):
            c = torch.arange(lo, min(lo + step, K), device="cuda")
            first, end = weights_of(c, p) if p > 1 else (weight_of(c), None)
            for i in range(n):
                want = X[i, 0].float() * first + (X[i, last].float() * end if p > 1 else 0)
                assert torch.equal(Z[i, lo:lo + step].float(), want), (i, lo)
        assert bool((Z[n] == 7).all())
        del Z
    del block
    torch.cuda.empty_cache()
