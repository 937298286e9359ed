"""ssn_logprobs on rows that a confident model gives: a few classes far above all others.

Tolerances are for the root mean square over many rows.  A row's sum s passes `count` roundings: the additions of a lane's
margins, the exchanges of 64 lanes and 16 waves (ten additions), and about sixteen more in exponentials and rescalings, each off
by at most u = 2^-24 of s and as likely up as down: the root mean square of their sum is at most sqrt(count) u, and L = log s
is off by that.  The entropy L - t / s has the same count on each of its terms, the second of the size of H - L, at most
H + 1 here."""
import pytest
import torch

from paper_1802_09113_amd.binding import ssn_logprobs

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


def exact(Z):
    """logpart and entropy in 64 bits."""
    z = Z.double()
    d = z - z.amax(1, keepdim=True)
    L = d.exp().sum(1).log()
    p = (d - L[:, None]).exp()
    return L, L - (p * d).sum(1)


# rows, classes and the most margins that a lane adds up: one wave, four, eight and sixteen to a row, and rows of several
# workgroups
@pytest.mark.parametrize("n,C,lane", [(300, 768, 16), (2100, 3001, 64), (600, 9001, 80), (300, 32003, 80), (256, 65536, 136),
                                      (100, 50000, 80), (4, 131077, 64), (300, 400, 8)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_entropy_of_peaked_rows(dtype, n, C, lane):
    g = torch.Generator(device="cuda")
    g.manual_seed(C)
    count = lane + 10 + 16
    for gap in (4, 9, 12.5, 20):                         # above normal margins; over and below what a lane may lag behind
        Z = torch.randn(n, C, generator=g, device="cuda")
        at = torch.randint(C, (n, 4), generator=g, device="cuda")
        Z.scatter_(1, at, gap + 3 * torch.rand(n, 4, generator=g, device="cuda"))
        Z = Z.to(DTYPES[dtype])
        print(f"[case] n={n} C={C} {dtype} gap={gap}", flush=True)
        out, (L, H) = ssn_logprobs(Z), exact(Z)
        eL = float((out["logpart"] - L).square().mean().sqrt())
        # the entropy's error in units of its size: |H - L| <= H + 1
        eH = float(((out["entropy"] - H) / (2 + H + L)).square().mean().sqrt())
        print(f"   L {eL / U:.2f} u, H {eH / U:.2f} u, sqrt(count) {count ** 0.5:.2f}", flush=True)
        assert eL <= (count ** 0.5 + float(L.max())) * U and eH <= count ** 0.5 * U


@pytest.mark.parametrize("n,C", [(300, 1000), (2100, 3001), (600, 9001), (300, 32003), (256, 65536), (3, 131077)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_a_best_class_behind_margins_of_the_same_lane(dtype, n, C):
    """One class above all, and before it, at every distance of a wave's load of 16 bytes a lane, margins 3 to 12.8 below it,
    which the lane has met first.  Nothing else weighs anything, so that few roundings are left: two exponentials of the best
    class's term (3 u each, with its argument), at most two rescalings (3 u each), ten additions that join lanes and waves, the
    logarithm (2 u): 24 on L, and as many again on t / s."""
    dt = DTYPES[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(C)
    step = 1024 // torch.empty((), dtype=dt).element_size()
    square, seen = torch.zeros(2, dtype=torch.float64, device="cuda"), 0
    for _ in range(max(1, 256 // n)):
        best = torch.randint(C, (n, 1), generator=g, device="cuda")
        v = 3 * torch.rand(n, 1, generator=g, device="cuda")
        gap = 3 + 9.8 * torch.rand(n, 1, generator=g, device="cuda")
        c = torch.arange(C, device="cuda")
        Z = torch.where((c < best) & ((best - c) % step == 0), v - gap, -60.0)
        Z = Z.scatter_(1, best, v).to(dt)
        out, (L, H) = ssn_logprobs(Z), exact(Z)
        assert bool((out["maxpart"] == Z.amax(1).float()).all())
        square += torch.stack([(out["logpart"] - L).square().sum(), (out["entropy"] - H).square().sum()])
        seen += n
    eL, eH = ((square / seen).sqrt() / U).tolist()
    print(f"[case] n={n} C={C} {dtype}: L {eL:.2f} u, H {eH:.2f} u", flush=True)
    assert eL <= 24 ** 0.5 and eH <= 48 ** 0.5


@pytest.mark.parametrize("n,C", [(4096, 300), (4096, 700), (3000, 5000), (600, 9001), (100, 40000), (3, 131077)])
@pytest.mark.parametrize("dtype", list(DTYPES) + ["f64"])
def test_signs(dtype, n, C):
    """logpart >= 0, entropy >= 0 and no log probability above zero, exactly: rows of one class, or of a class that has all the
    weight, at every size of its margin."""
    dt = DTYPES.get(dtype, torch.float64)
    g = torch.Generator(device="cuda")
    g.manual_seed(C)
    for scale in (1.0, 30.0, 3000.0):
        best = torch.randint(C, (n, 1), generator=g, device="cuda")
        Z = scale * torch.randn(n, C, generator=g, device="cuda") - 40 * scale
        Z = Z.scatter_(1, best, scale * torch.randn(n, 1, generator=g, device="cuda"))
        Z[::3] = torch.where(torch.arange(C, device="cuda") == best[::3], Z[::3], -float("inf"))
        out = ssn_logprobs(Z.to(dt), best.to(torch.int32), k=2)
        print(f"[case] n={n} C={C} {dtype} scale={scale} lowest logpart {float(out['logpart'].min()):.3g}", flush=True)
        assert bool((out["logpart"] >= 0).all()) and bool((out["entropy"] >= 0).all())
        assert bool((out["logp"] <= 0).all()) and bool((out["top_logp"] <= 0).all())
        assert bool((out["top_ids"][:, :1] == best).all())
