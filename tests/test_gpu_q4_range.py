"""ssn_q4_margins over the whole range of its features' types: the largest, the smallest, subnormal ones.

Tolerances: those of test_gpu_q4.py (`group` additions in the matrix cores, one rounding or two per group, a few to join, none
off by more than a step 2^-23 of sum |x| |w|), and at the lower end what the header states: bits of a float feature below 2^-133
are not seen, and a margin's sum is rounded to multiples of 2^-139, once for each group and a few times more."""
import pytest
import torch

from paper_1802_09113_amd.binding import Q4Block, ssn_q4_margins, ssn_q4_quantize

pytestmark = pytest.mark.gpu

F = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
# every form of the kernels: rows, features, classes
SHAPES = [(1, 256, 64), (2, 300, 20500), (3, 20000, 40), (6, 300, 8300), (7, 256, 24704), (13, 256, 64), (16, 256, 16500),
          (40, 384, 100), (100, 300, 5200), (70, 9000, 40), (257, 256, 20480)]


def weights(block):
    """The weights that a block stands for, K x p in 64 bits, by the documented layout."""
    tiles, blocks = block.packed.shape[:2]
    c = torch.stack([block.packed & 15, block.packed >> 4], -1).view(tiles, blocks, 4, 16, 4, 4, 2)
    c = c.permute(0, 3, 1, 4, 2, 5, 6).reshape(tiles * 16, -1).long()
    v = torch.where(c >= 8, -1.0, 1.0) * SIZES.to(c.device)[c % 8]
    s = block.scales.double().permute(0, 2, 1, 3).reshape(tiles * 16, -1)
    return (v.view(tiles * 16, -1, block.group) * s[..., None]).view(tiles * 16, -1)[:block.K, :block.p]


def check(dtype, n, p, K, group, size, wsize, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    block = ssn_q4_quantize((wsize * torch.randn(p, K, generator=g, device="cuda", dtype=torch.float64)), group)
    X = (size * torch.randn(n, p, generator=g, device="cuda", dtype=torch.float64).clamp(-3, 3)).to(F[dtype])
    assert bool(torch.isfinite(X).all())
    print(f"[case] n={n} p={p} K={K} group={group} {dtype} size={size:g} weights {wsize:g}", flush=True)
    got = ssn_q4_margins(block, X, torch.empty(n, K, device="cuda")).double()
    W, x = weights(block), X.double()
    want, total = x @ W.t().contiguous(), x.abs() @ W.abs().t().contiguous()
    steps = group + p / group + 80
    lost = (2.0 ** -133 * W.abs().sum(1) if dtype == "f32" else 0) + (p / group + 16) * 2.0 ** -139
    err, tol = (got - want).abs(), steps * 2.0 ** -23 * total + lost
    assert bool((err <= tol).all()), (float((err / tol).max()), int((~torch.isfinite(got)).sum()))


@pytest.mark.parametrize("n,p,K", SHAPES)
@pytest.mark.parametrize("dtype,group", [("bf16", 32), ("bf16", 128), ("f32", 64), ("f32", 32)])
def test_largest_features(dtype, group, n, p, K):
    """Margins of the order of 1e35 from features of the order of 1e38: a group's sum of code numbers times features is beyond
    the largest float."""
    check(dtype, n, p, K, group, 1e38, 1e-5, n)


@pytest.mark.parametrize("n,p,K", SHAPES)
@pytest.mark.parametrize("dtype,group", [("bf16", 64), ("f32", 32), ("f32", 128), ("f16", 32)])
def test_smallest_features(dtype, group, n, p, K):
    for size in (1e-4, 1e-6, 1e-7) if dtype == "f16" else (1e-30, 1e-34, 1e-36, 1e-38, 1e-40):
        check(dtype, n, p, K, group, size, 0.02, n)
        check(dtype, n, p, K, group, size, 1e30 if dtype != "f16" else 1e-4, n + 1)


# float rows on both sides of the class counts where another form takes over (256 compute units)
@pytest.mark.parametrize("n,K", [(6, 8192), (6, 8193), (12, 8192), (12, 8193), (16, 16384), (16, 16385), (4, 14336), (8, 24576)])
def test_float_rows_at_the_borders(n, K):
    check("f32", n, 300, K, 64, 1.0, 0.02, n)


@pytest.mark.parametrize("dtype", list(F))
def test_largest_scales(dtype):
    """The largest scales that there are, at features that make the margins finite, and classes whose codes are all zero."""
    block = ssn_q4_quantize(torch.ones(256, 20, device="cuda"), 32)
    scales = torch.full_like(block.scales, torch.finfo(torch.bfloat16).max)
    packed = block.packed.clone()
    packed[:, :, 3::16] = 0                              # class 3 of each tile of 16
    block = Q4Block(packed, scales, 256, 20, 32)
    size = 2.0 ** -14 if dtype == "f16" else 2.0 ** -120
    for n in (1, 7, 16, 100):
        X = torch.full((n, 256), size, device="cuda", dtype=F[dtype])
        got = ssn_q4_margins(block, X, torch.empty(n, 20, device="cuda")).double()
        want = X.double() @ weights(block).t().contiguous()
        finite = want.abs() < torch.finfo(torch.float32).max
        assert bool((got[:, [3, 19]] == 0).all()) and not bool(torch.isnan(got).any())
        assert bool(((got - want).abs()[finite] <= 1e-5 * want.abs()[finite]).all())
