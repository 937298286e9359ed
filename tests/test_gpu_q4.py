"""Weight blocks in 4 bits: ssn_q4_quantize bit for bit against its rule on the host, ssn_q4_margins against a product in 64
bits, and the run of calls that a trained layer is answered with, against the framework's own objective and gradient.

Tolerances: products are exact in fp32.  A margin's sum passes through at most `group` additions inside the matrix cores, one
multiplication and addition per group and a few to join waves and parts, none of them off by more than a step 2^-23 of the
largest partial sum, itself at most sum |x| |w|; then one rounding to the output's type."""
import numpy as np
import pytest
import torch

from paper_1802_09113_amd import binding, synth
from paper_1802_09113_amd.binding import (Context, Q4Block, SsnError, ssn_logprobs, ssn_logprobs_grad, ssn_q4_margins,
                                          ssn_q4_quantize)

pytestmark = pytest.mark.gpu

F = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f64": torch.float64}
SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16_up(v):
    """The smallest bfloat16 number >= v (v >= 0, float64 host array), as float64."""
    f = v.astype(np.float32)
    f = np.where(f.astype(np.float64) < v, np.nextafter(f, np.float32(np.inf)), f)        # smallest float >= v
    b = f.view(np.uint32)
    b = np.where(b & 0xffff, (b | 0xffff) + np.uint32(1), b).astype(np.uint32)
    return b.view(np.float32).astype(np.float64)


def rule(W, group):
    """Codes and scales of W (p x K float64) by the rule, padded; NaN scales where a group is not finite."""
    p, K = W.shape
    P, Kp = -(-p // 128) * 128, -(-K // 16) * 16
    w = np.zeros((Kp, P))
    w[:K, :p] = W.T
    w = w.reshape(Kp, P // group, group)
    a = np.abs(w)
    most = a.max(2)
    finite = np.isfinite(w).all(2) & ~(most > 6 * 3.3895313892515355e38)
    with np.errstate(invalid="ignore"):
        s = bf16_up(np.where(finite, most, 0) / 6)
        s = np.where(6 * s < np.where(finite, most, 0), np.nan, s)                       # the quotient's own rounding
    assert not np.isnan(s).any()
    lower = np.maximum(s.astype(np.float32).view(np.uint32).astype(np.int64) - 0x10000, 0).astype(np.uint32).view(np.float32)
    s = np.where((6 * lower.astype(np.float64) >= np.where(finite, most, 0)), lower.astype(np.float64), s)
    with np.errstate(all="ignore"):
        r = np.where(finite[..., None] & (s[..., None] > 0), a / np.where(s > 0, s, 1)[..., None], 0)
    # exact comparisons: a and s * border are float64 with room to spare
    t = s[..., None]
    live = finite[..., None] & (t > 0)
    idx = np.zeros(r.shape, dtype=np.uint8)
    for border, closed in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        with np.errstate(invalid="ignore"):
            idx += (live & ((a >= border * t) if closed else (a > border * t))).astype(np.uint8)
    code = (idx + 8 * ((w < 0) & (idx > 0))).astype(np.uint8).reshape(Kp, P)
    return code, np.where(finite, s, np.nan)


def unpack(block):
    """Codes (Kp x P) and scales (Kp x groups) of a block, by the addresses of the documented layout."""
    p, K, group = block.p, block.K, block.group
    packed, scales = block.packed.cpu().numpy().reshape(-1), block.scales.float().cpu().numpy().reshape(-1)
    nq, tiles = -(-p // 128), -(-K // 16)
    c, f = np.meshgrid(np.arange(tiles * 16), np.arange(nq * 128), indexing="ij")
    t, o, q, r = c // 16, c % 16, f // 128, f % 128
    j, g, b = r // 32, r % 32 // 8, r % 8 // 2
    byte = packed[((t * nq + q) * 64 + 16 * g + o) * 16 + 4 * j + b]
    code = np.where(f % 2, byte >> 4, byte & 15).astype(np.uint8)
    c, i = np.meshgrid(np.arange(tiles * 16), np.arange(nq * 128 // group), indexing="ij")
    per = 128 // group
    return code, scales[((c // 16 * nq + i // per) * 16 + c % 16) * per + i % per].astype(np.float64)


def values(block):
    """The p x K weights that a block stands for, float64."""
    code, s = unpack(block)
    v = np.where(code & 8, -1.0, 1.0) * SIZES[code & 7]
    return (v.reshape(len(code), -1, block.group) * s[..., None]).reshape(len(code), -1)[:block.K, :block.p].T


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("p,K", [(1, 1), (7, 3), (128, 16), (129, 17), (300, 33), (31, 100), (1000, 40)])
@pytest.mark.parametrize("dtype", list(F))
def test_quantize_by_the_rule(dtype, p, K, group):
    rng = np.random.default_rng(p * 7 + K)
    W = rng.standard_normal((p, K)) * np.exp(rng.uniform(-6, 3, (1, K)))
    if dtype in ("f32", "f64"):                          # ties and borders: multiples of a quarter of a power of two
        W[:, ::3] = rng.integers(-24, 25, W[:, ::3].shape) / 4.0
    W[:, K // 2] = 0
    Wt = torch.from_numpy(W).to(F[dtype])
    code, s = rule(Wt.double().numpy(), group)
    ld = torch.full((p, K + 3), float("nan"), dtype=F[dtype], device="cuda")
    ld[:, :K] = Wt.cuda()
    for view in (ld[:, :K], Wt.t().contiguous().cuda().t()):         # classes contiguous, features contiguous
        got, gs = unpack(ssn_q4_quantize(view, group))
        assert np.array_equal(gs, s) and np.array_equal(got, code)


def test_quantize_extremes():
    """Tiny and huge weights, and groups that no scale reaches."""
    W = np.zeros((256, 20))
    W[:32, 0], W[32:64, 0] = 1e-40, -3e38
    W[5, 1], W[40, 1], W[70, 1] = np.nan, np.inf, -np.inf
    W[3, 2], W[35, 2], W[67, 2] = 1e300, 2.1e39, 2.0e39
    W[1, 3], W[33, 3] = 1e-46, 9.2e-41
    for dt in (torch.float64, torch.float32):
        Wt = torch.from_numpy(W).to(dt)
        code, s = rule(Wt.double().numpy(), 32)
        got, gs = unpack(ssn_q4_quantize(Wt.cuda(), 32))
        assert np.array_equal(gs, s, equal_nan=True) and np.array_equal(got, code)
        assert np.isnan(s[1, :3]).all() and np.isnan(s[2, 0]) and np.isfinite(s[0]).all()


def random_block(p, K, group, rng, scale=0.02):
    return ssn_q4_quantize(torch.from_numpy(rng.standard_normal((p, K)) * scale).float().cuda(), group)


def check_margins(block, X, Z=None):
    zt = X.dtype if Z is None else Z.dtype
    print(f"[case] n={X.shape[0]} p={block.p} K={block.K} group={block.group} {X.dtype} -> {zt}", flush=True)
    got = ssn_q4_margins(block, X, Z)
    assert got.dtype == zt
    W, x = values(block), X.double().cpu().numpy()
    want, size = x @ W, np.abs(x) @ np.abs(W)
    steps = block.group + block.p / block.group + 80
    tol = steps * 2.0 ** -23 * size + np.abs(want) * torch.finfo(zt).eps / 2 + torch.finfo(zt).smallest_normal * torch.finfo(zt).eps
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(~(err <= tol))[:4].tolist())
    return got


# rows around every border between the forms, features that end inside a block, a group and a vector, classes inside a tile;
# few classes with many features (parts joined through the workspace)
@pytest.mark.parametrize("n,p,K", [(1, 1, 1), (1, 8, 16), (2, 100, 7), (3, 128, 33), (4, 131, 16), (5, 1000, 100), (7, 4100, 30),
                                   (16, 257, 50), (17, 515, 65), (31, 640, 129), (32, 129, 40), (33, 300, 31), (64, 1024, 48),
                                   (65, 700, 200), (129, 2051, 77), (300, 384, 130), (1, 20000, 9), (9, 33000, 19), (70, 9000, 33)])
@pytest.mark.parametrize("dtype,group", [("bf16", 32), ("bf16", 64), ("f16", 128), ("f16", 32), ("f32", 64), ("f32", 128), ("f32", 32)])
def test_margins(dtype, group, n, p, K):
    rng = np.random.default_rng(n * 31 + p + K)
    block = random_block(p, K, group, rng)
    X = torch.from_numpy(rng.standard_normal((n, p))).to(F[dtype]).cuda()
    check_margins(block, X)


# as many classes as it takes for each form to serve (256 compute units); odd numbers of rows, features and classes
@pytest.mark.parametrize("dtype,group,n,p,K", [
    ("bf16", 32, 1, 300, 20500), ("f16", 64, 3, 1025, 24001), ("f32", 32, 2, 300, 14500), ("bf16", 128, 6, 300, 20500),
    ("f32", 64, 7, 300, 16500), ("f32", 32, 8, 300, 8300), ("f32", 64, 5, 300, 24700), ("f16", 32, 12, 300, 12500), ("f32", 128, 11, 300, 8300), ("f32", 32, 13, 300, 16500),
    ("f32", 32, 30, 140, 33001), ("bf16", 32, 100, 300, 5200), ("f16", 128, 40, 300, 20501), ("bf16", 64, 200, 300, 11001),
    ("f16", 32, 130, 300, 20501), ("bf16", 128, 257, 128, 20480), ("bf16", 32, 150, 127, 2000), ("f32", 32, 40, 100, 700)])
def test_margins_of_many_classes(dtype, group, n, p, K):
    rng = np.random.default_rng(n + p + K)
    block = random_block(p, K, group, rng)
    X = torch.from_numpy(rng.standard_normal((n, p))).to(F[dtype]).cuda()
    check_margins(block, X)
    if dtype != "f32":
        check_margins(block, X, torch.empty(n, K, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_margins_of_strided_and_unaligned_rows(dtype):
    """Rows at addresses aligned to one element, NaN between and behind them; results into a wider float32 buffer whose
    other columns and rows stay."""
    rng = np.random.default_rng(2)
    for n, p, K in ((3, 517, 45), (40, 517, 45), (130, 1029, 70)):
        block = random_block(p, K, 32, rng)
        flat = torch.full((1 + n * (p + 2),), float("nan"), dtype=F[dtype], device="cuda")
        X = flat[1:].view(n, p + 2)[:, :p]
        X.copy_(torch.from_numpy(rng.standard_normal((n, p))))
        buf = torch.full((n + 2, K + 3), 5.0, device="cuda")
        got = check_margins(block, X, buf[1:n + 1, 1:K + 1])
        assert torch.equal(got, buf[1:n + 1, 1:K + 1])
        got.fill_(5.0)
        assert bool((buf == 5.0).all())


def test_rows_do_not_meet():
    """NaN and infinities of one row stay in that row; an infinity is one for weights of its sign; a NaN scale is its
    class's NaN."""
    rng = np.random.default_rng(4)
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        for n in (3, 20, 100):
            block = random_block(300, 40, 64, rng)
            X = torch.from_numpy(rng.standard_normal((n, 300))).to(dt).cuda()
            want = ssn_q4_margins(block, X)
            X[1, 5], X[2, 299] = float("nan"), float("inf")
            got = ssn_q4_margins(block, X)
            assert bool(torch.isnan(got[1]).all()) and not bool(torch.isfinite(got[2]).any())
            keep = [i for i in range(n) if i not in (1, 2)]
            assert torch.equal(got[keep], want[keep])
        one = ssn_q4_quantize(torch.tensor([[6.0, -3.0, 1.5]], device="cuda"), 32)
        got = ssn_q4_margins(one, torch.tensor([[float("inf")], [-float("inf")], [3.0]], device="cuda").to(dt))
        assert got.tolist() == [[float("inf"), -float("inf"), float("inf")], [-float("inf"), float("inf"), -float("inf")],
                                [18.0, -9.0, 4.5]]
    W = torch.randn(300, 20, device="cuda")
    W[7, 3] = float("nan")
    got = ssn_q4_margins(ssn_q4_quantize(W, 32), torch.randn(5, 300, device="cuda"))
    assert bool(torch.isnan(got[:, 3]).all()) and not bool(torch.isnan(got[:, [0, 2, 4, 19]]).any())


def test_single_precision_rows_are_split_exactly():
    """One weight of 1 per class (the scale is 1: each group holds a 6, met by a feature of zero): margins are the features
    themselves, to the last bit, up to the largest number."""
    W = torch.eye(64, device="cuda")
    W[31], W[63] = 6.0, 6.0
    rng = np.random.default_rng(6)
    x = rng.integers(-2 ** 31, 2 ** 31, (8, 64)).astype(np.int32).view(np.float32)
    x = np.where(np.isfinite(x) & (np.abs(x) > 1e-30), x, np.float32(1.0000001))
    x[0, :4] = [3.4028235e38, -3.4028235e38, 1.17549435e-38 * 2 ** 30, 16777215.0]
    x[:, 31], x[:, 63] = 0.0, 0.0
    X = torch.from_numpy(x).cuda()
    Z = ssn_q4_margins(ssn_q4_quantize(W, 32), X)
    own = [c for c in range(64) if c not in (31, 63)]
    assert torch.equal(Z[:, own], X[:, own])


def test_no_rows_and_refusals():
    block = random_block(100, 20, 32, np.random.default_rng(0))
    assert ssn_q4_margins(block, torch.empty((0, 100), device="cuda")).shape == (0, 20)
    X = torch.zeros(2, 100, device="cuda")
    with pytest.raises(SsnError) as e:
        ssn_q4_margins(block, X.double())
    assert e.value.status == binding.SSN_E_UNSUPPORTED
    with pytest.raises(SsnError) as e:
        ssn_q4_margins(block, X, torch.zeros(2, 20, device="cuda", dtype=torch.float16))
    assert e.value.status == binding.SSN_E_INVALID_ARG
    with pytest.raises(SsnError) as e:                                       # rows on top of each other
        ssn_q4_margins(block, X[:1].expand(3, 100))
    assert e.value.status == binding.SSN_E_INVALID_ARG
    with pytest.raises(SsnError) as e:
        ssn_q4_quantize(X.expand(3, 2, 100)[:, 0], 32)
    assert e.value.status == binding.SSN_E_INVALID_ARG
    for bad in (X[:, :99], X.t(), X.cpu()):
        with pytest.raises(AssertionError):
            ssn_q4_margins(block, bad)
    with pytest.raises(AssertionError):
        ssn_q4_margins(block._replace(packed=block.packed[:, :, :32]), X)
    with pytest.raises(AssertionError):
        ssn_q4_margins(block._replace(group=64), X)
    with pytest.raises(AssertionError):
        ssn_q4_quantize(X, 16)
    torch.cuda.synchronize()


def test_captured_margins_replayed():
    """A product whose parts meet in a workspace, and one without, replayed on new rows with eager calls in between."""
    rng = np.random.default_rng(8)
    for n, p, K in ((2, 20000, 40), (3, 500, 3000), (200, 600, 300)):
        block = random_block(p, K, 32, rng)
        X = torch.randn(n, p, device="cuda").to(torch.bfloat16)
        Z = ssn_q4_margins(block, X)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            ssn_q4_margins(block, X, Z)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ssn_q4_margins(block, X, Z)
        for _ in range(4):
            X.normal_()
            want = ssn_q4_margins(block, X)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(Z, want)


def test_a_trained_layer_answered_in_4_bits():
    """Train with ssn_solve, lay the weights out in 4 bits, ask for margins, log probabilities and alternatives, and send a
    gradient back: at the weights that the codes stand for, mean(-logp) + lambda/2 ||W||^2 is the framework's objective, X^T dZ +
    lambda W its gradient, and the first alternative its prediction."""
    d = synth.make(1, n=1500)
    X = torch.from_numpy(d["X"]).float().cuda()
    labels = torch.from_numpy(d["labels"]).cuda()
    n, p, C = d["n"], d["p"], d["C"]
    ctx = Context(labels, C, d["lam"], X=X)
    W = torch.zeros((p, C - 1), device="cuda")
    S = torch.stack([torch.from_numpy(synth.sample_rows(n, 200, it=i)) for i in range(3)]).int().cuda()
    ctx.ssn_solve(W, S)
    block = ssn_q4_quantize(W, 32)
    Wq = torch.from_numpy(np.ascontiguousarray(values(block))).float().cuda()  # exact: three significant bits times eight
    assert float((Wq - W).norm() / W.norm()) < 0.2
    Z = ssn_q4_margins(block, X)
    out = ssn_logprobs(Z, labels, k=1, reference=True)
    f = ctx.ssn_objective(Wq)
    reg = 0.5 * d["lam"] * float((Wq.double() ** 2).sum())
    assert float(-out["logp"].double().mean()) + reg == pytest.approx(f, rel=1e-4)
    dZ = ssn_logprobs_grad(Z, labels, out, dlogp=torch.full((n,), -1.0 / n, device="cuda"), reference=True)
    G, _ = ctx.ssn_gradient(Wq)
    mine = X.double().t().contiguous() @ dZ.double() + d["lam"] * Wq.double()
    assert float((mine - G.double()).norm() / G.double().norm()) <= 1e-4
    pred, _ = ctx.ssn_predict(Wq)
    same = out["top_ids"][:, 0] == pred
    margins = torch.cat([Z, Z.new_zeros(n, 1)], 1).sort(1, descending=True).values
    assert bool((same | (margins[:, 0] - margins[:, 1] < 1e-4)).all())
    ctx.close()
