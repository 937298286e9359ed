"""ssn_logprobs and ssn_logprobs_grad against the definitions in 64 bits on the host: sizes around every border between the
kernels' forms, every type, masks and margins that leave a row empty, ties, given classes of every kind, strides, streams,
captured graphs, and buffers whose surroundings must stay as they were.

Tolerances count roundings of half a step u (2^-24 in fp32, 2^-53 in fp64) of the type in which sums are formed.  The row's
sum s has positive terms, a lane adds at most ceil(C / 64) + 16 of them one after the other, lanes and waves add a few more,
and a term carries its exponential's (|d| + 4) u with weight e^d, at most 8 u altogether: s is off by (C / 64 + 64) u relative,
L by that absolute.  logp = (z - M) - L adds two roundings of at most the size of |z - M| and |logp|.  The entropy L - t / s has
the same count on both of its terms."""
import numpy as np
import pytest
import torch

from paper_1802_09113_amd import binding
from paper_1802_09113_amd.binding import SsnError, ssn_logprobs, ssn_logprobs_grad

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f64": torch.float64}
INF = float("inf")


def u_of(dtype):
    return 2.0 ** -53 if dtype == torch.float64 else 2.0 ** -24


def bits(mask):
    """n x C truth values as int32 words on the device."""
    n, C = mask.shape
    padded = np.zeros((n, -(-C // 32) * 32), dtype=np.uint8)
    padded[:, :C] = mask
    return torch.from_numpy(np.packbits(padded, axis=1, bitorder="little").view(np.int32).copy()).cuda()


def definition(Z, labels, k, reference, mask, largest):
    """Statistics of every row, from the definitions, in float64 (Z: float64 host array).  A log probability below the
    most negative number of the statistics' type (the distance of the type's lowest margin from its largest one is twice
    that) rounds to -inf there."""
    z = np.concatenate([Z, np.zeros((len(Z), 1))], 1) if reference else Z.copy()
    if mask is not None:
        z[~mask] = -INF
    n, C = z.shape
    bad = (np.isnan(z) | (z == INF)).any(1)
    with np.errstate(all="ignore"):
        M = np.where(bad, np.nan, z.max(1))
        empty = M == -INF
        d = z - np.where(empty, 0, M)[:, None]
        e = np.exp(d)
        s = np.where(empty, 1, e.sum(1))
        L = np.log(s)
        logp = d - L[:, None]
        logp[logp < -largest] = -INF
        p = np.exp(logp)
        H = -np.where(p > 0, p * logp, 0).sum(1)
    logp[empty], H[empty], p[empty] = -INF, 0, 0
    logp[bad], H[bad], p[bad], L[bad] = np.nan, np.nan, np.nan, np.nan
    each = np.arange(n)[:, None]
    given = logp[each, np.clip(labels, 0, C - 1)]
    given = np.where(labels < 0, 0, np.where(labels >= C, np.nan, given))
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]
    val = z[each, order]
    none = (val == -INF) | bad[:, None]
    return dict(logp=given, maxpart=M, logpart=L, entropy=H, top_ids=np.where(none, -1, order),
                top_logp=np.where(bad[:, None], np.nan, np.where(none, -INF, logp[each, order]))), z, logp, p


def gradient(z, logp, p, ref, labels, g, l, h, reference):
    n, C = p.shape
    out = np.zeros((n, C))
    with np.errstate(all="ignore"):
        for t in range(labels.shape[1]):
            y = labels[:, t]
            w = np.where((y < 0) | (ref["logp"][:, t] == -INF), 0.0, np.where(y >= C, np.nan, g[:, t]))
            out -= w[:, None] * p
            out[np.arange(n), np.clip(y, 0, C - 1)] += np.where((y < 0) | (y >= C), 0, w)
        if l is not None:
            out += l[:, None] * p
        if h is not None:
            out -= h[:, None] * np.where(p > 0, p * (logp + ref["entropy"][:, None]), 0 * p)
    return out[:, :-1] if reference else out


def close(got, want, tol):
    got = got.double().cpu().numpy() if torch.is_tensor(got) else got
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= tol)
    assert ok.all(), (np.argwhere(~ok)[:4].tolist(), got[~ok][:4], want[~ok][:4])


def check(Zd, Zh, labels, k, reference, mask, allowed=None, grad=True, lse=True, entropy=True, seed=0):
    """Forward and gradient of device rows Zd (host copy Zh in float64) against the definitions; returns the outputs."""
    n, dt = len(Zh), Zd.dtype
    C, u = Zh.shape[1] + reference, u_of(dt)
    if allowed is None and mask is not None:
        allowed = bits(mask)
    lab = torch.from_numpy(labels.astype(np.int32)).cuda()
    print(f"[case] n={n} C={C} {dt} m={labels.shape[1]} k={k} reference={reference} mask={mask is not None}", flush=True)
    out = ssn_logprobs(Zd, lab, k=k, reference=reference, allowed=allowed)
    ref, z, logp, p = definition(Zh, labels, k, reference, mask, torch.finfo(out["maxpart"].dtype).max)
    count = (C / 64 + 64) * u
    with np.errstate(invalid="ignore"):
        size = np.where(np.isfinite(ref["logp"]), np.abs(ref["logp"]), 0)
    close(out["logp"], ref["logp"], count + 2 * u * (size + np.nan_to_num(ref["logpart"])[:, None]))
    close(out["maxpart"], ref["maxpart"], 0)
    close(out["logpart"], ref["logpart"], count + u * np.nan_to_num(ref["logpart"]))
    close(out["entropy"], ref["entropy"], 2 * count * (1 + np.nan_to_num(ref["entropy"])))
    if k:
        assert np.array_equal(out["top_ids"].cpu().numpy(), ref["top_ids"])
        size = np.where(np.isfinite(ref["top_logp"]), np.abs(ref["top_logp"]), 0)
        close(out["top_logp"], ref["top_logp"], count + 2 * u * (size + np.nan_to_num(ref["logpart"])[:, None]))
    if not grad:
        return out
    rng = np.random.default_rng(seed)
    stat = torch.float64 if dt == torch.float64 else torch.float32
    dev = lambda a: torch.from_numpy(a).to(stat).cuda()                                    # noqa: E731
    rounded = lambda a: a if stat == torch.float64 else a.astype(np.float32).astype(np.float64)  # noqa: E731
    g, l, h = (rounded(rng.standard_normal(s)) for s in (labels.shape, n, n))
    l, h = (l if lse else None), (h if entropy else None)
    dZ = ssn_logprobs_grad(Zd, lab, out, dlogp=dev(g) if labels.shape[1] else None, dlse=dev(l) if lse else None,
                           dentropy=dev(h) if entropy else None, reference=reference, allowed=allowed)
    want = gradient(z, logp, p, ref, labels, g, l, h, reference)
    # p is off by (|log p| + 8) u and the forward call's `count`, relative; its factor by the sum of the weights' sizes; the
    # result is rounded to the margins' type (the gradients' smallest steps: subnormal numbers)
    weight = np.abs(g).sum(1) + (np.abs(l) if lse else 0)
    if entropy:
        weight = weight + np.abs(h) * (4 + np.nan_to_num(ref["entropy"]))
    pz = p[:, :want.shape[1]]
    with np.errstate(all="ignore"):
        lp = np.where(pz > 0, -np.log(pz), 0)
        tol = pz * (1 + lp) * (weight[:, None] + 1) * ((lp + 16) * u + 2 * count) * 2
    step = torch.finfo(dt)
    tol = np.nan_to_num(tol) + np.nan_to_num(np.abs(want)) * (step.eps / 2 + 4 * u) + step.smallest_normal * step.eps
    tol = tol + u * np.abs(g).sum(1)[:, None] * (np.abs(np.nan_to_num(want)) > 0) * 2
    close(dZ, want, tol)
    return out


def rows(n, width, dt, rng, pad=0, scale=2.0):
    """Normal rows (device view of a buffer that is `pad` wider, with NaN in between; host copy in float64)."""
    h = torch.from_numpy(rng.standard_normal((n, width)) * scale).to(dt)
    buf = torch.full((n, width + pad), float("nan"), dtype=dt, device="cuda")
    buf[:, :width] = h.cuda()
    return buf[:, :width], h.double().numpy()


def some_labels(n, m, C, rng):
    y = rng.integers(0, C, (n, m))
    y[rng.random((n, m)) < 0.1] = -1
    return y


# one class; each border between the forms (512 classes; 8 and 16 wave loads of 16 bytes; vectors that end inside a row);
# rows split over workgroups (few rows) and not (many)
SIZES = [(1, 1), (3, 2), (300, 7), (65, 8), (64, 9), (5, 64), (3, 65), (9, 512), (3, 513), (2, 517), (1, 1000), (3, 2047), (5, 2049),
         (2, 4096), (2, 4100), (7, 4099), (3, 8191), (1, 16385), (70, 300), (1100, 900), (1, 32003), (600, 9001), (300, 9001), (2100, 3001), (2, 131077)]


@pytest.mark.parametrize("n,C", SIZES)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_sizes(dtype, n, C):
    rng = np.random.default_rng(n * 131 + C)
    for reference, mask, pad, m, k in [(False, False, 0, 1, min(5, C)), (True, True, 3, 3, min(C, 20)), (False, True, 0, 0, 0),
                                       (True, False, 1, 64, min(C, 64))]:
        if reference and C < 2:
            continue
        Zd, Zh = rows(n, C - reference, DTYPES[dtype], rng, pad)
        allowed = None
        if mask:
            allowed = rng.random((n, C)) < 0.5
            allowed[::3] = False                                    # rows without a class
            allowed[1::3, :C // 2] = False                          # leading classes out
        check(Zd, Zh, some_labels(n, m, C, rng), k, reference, allowed, lse=bool(m), entropy=bool(k) or not m)


@pytest.mark.parametrize("C", [6, 300, 700, 5000, 40000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_special_values(dtype, C):
    """Rows: all -inf; one finite; the type's lowest value everywhere; lowest and largest; NaN; +inf; NaN, +inf and -inf only
    where they are not allowed; all equal; ascending; descending; -inf at the given class; a mask without a bit."""
    dt, rng = DTYPES[dtype], np.random.default_rng(C)
    low, high = torch.finfo(dt).min, torch.finfo(dt).max
    h = torch.from_numpy(rng.standard_normal((12, C))).to(dt).double().numpy()
    mask = np.ones((12, C), dtype=bool)
    y = np.full((12, 4), C - 1)
    y[:, 1], y[:, 2], y[:, 3] = C // 2, -1, 0
    h[0] = -INF
    h[1, :] = -INF
    h[1, C // 2] = 3.0
    h[2] = low
    h[3] = low
    h[3, C - 2] = high
    h[4, C // 3] = np.nan
    h[5, C - 2] = INF
    h[6, 1], h[6, 2], h[6, 3] = np.nan, INF, -INF
    mask[6, 1:4] = False
    h[7] = 0.5
    h[8] = np.round(np.linspace(-4, 4, C) * 64) / 64
    h[9] = np.round(np.linspace(4, -4, C) * 64) / 64
    h[10, C // 2], h[10, C - 1] = -INF, -INF
    h[11] = np.nan
    mask[11] = False
    h = torch.from_numpy(h).to(dt).double().numpy()
    Zd = torch.from_numpy(h).to(dt).cuda()
    for k in (1, min(C, 33)):
        check(Zd, h, y, k, False, mask)
        check(Zd, h, y, k, False, None)
    # the same rows with the reference class behind them (class C)
    check(Zd, h, y, min(C, 17), True, np.concatenate([mask, rng.random((12, 1)) < 0.5], 1))


@pytest.mark.parametrize("C", [9, 700, 5000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f64"])
def test_margins_far_from_zero(dtype, C):
    """Rows around values whose product with log2 e is rounded by more than one, up to the edge of the type; rows filled with
    -1e9 or -1e30 but for a few classes, or for one half; neighbours two steps apart out there."""
    dt, rng = DTYPES[dtype], np.random.default_rng(C)
    sizes = [4e6, 6e6, 1.1e7, 1e8, 3e9, 1e12, 1e20, 1e30, 3e37]
    h = np.zeros((4 * len(sizes) + 4, C))
    for i, v in enumerate(sizes):
        h[4 * i], h[4 * i + 1] = v, -v
        h[4 * i + 2], h[4 * i + 3] = v * (1 + rng.integers(-2, 1, C) * 2.0 ** -7), -v * (1 + rng.integers(0, 3, C) * 2.0 ** -7)
    h[-4:] = [[-1e9], [-1e30], [-1e9], [-9.9e6]]
    h[-4, 3::61], h[-3, C // 2:] = rng.standard_normal(len(h[0, 3::61])), rng.standard_normal(C - C // 2)
    h[-2, -1] = -1e9 + 128
    h[-1, C // 2:] = -1.0001e7
    h = torch.from_numpy(h).to(dt).double().numpy()
    y = np.stack([np.full(len(h), C - 1), rng.integers(0, C, len(h))], 1)
    for reference in (False, True):
        check(torch.from_numpy(h).to(dt).cuda(), h, y, 5, reference, None)


def test_nothing_at_classes_that_are_not_allowed():
    """Also where the row has no distribution, or a given class is not allowed or none."""
    for C in (40, 3000):
        Z = torch.randn(4, C, device="cuda")
        Z[1, 7], Z[2, 8] = float("nan"), float("inf")
        mask = np.ones((4, C), dtype=bool)
        mask[:, 20:30] = False
        lab = torch.tensor([[25, 1], [25, 1], [21, 22], [25, C]], dtype=torch.int32, device="cuda")
        out = ssn_logprobs(Z, lab, allowed=bits(mask))
        dZ = ssn_logprobs_grad(Z, lab, out, dlogp=torch.ones(4, 2, device="cuda"), allowed=bits(mask))
        assert bool((dZ[:, 20:30] == 0).all())
        keep = torch.ones(C, dtype=torch.bool)
        keep[20:30] = False
        assert bool(torch.isnan(dZ[1:, keep]).all()) and bool(torch.isfinite(dZ[0]).all())


def test_given_classes_of_every_kind():
    """The same class given several times, padding, an index that is no class: values and gradients."""
    rng = np.random.default_rng(3)
    for C in (5, 50, 3000):
        Zd, Zh = rows(4, C, torch.float32, rng)
        y = np.array([[1, 1, 1, -1], [-1, -5, -100, -2 ** 31], [0, C - 1, 0, C - 1], [C, 0, 1, 2 ** 31 - 1]])
        check(Zd, Zh, y, 2, False, None)


@pytest.mark.parametrize("C", [100, 3000])
def test_one_mask_for_all_rows_and_wider_mask_rows(C):
    rng = np.random.default_rng(C)
    Zd, Zh = rows(5, C, torch.bfloat16, rng)
    one = rng.random(C) < 0.3
    check(Zd, Zh, some_labels(5, 2, C, rng), 7, False, np.tile(one, (5, 1)), allowed=bits(one[None])[0])
    many = rng.random((5, C)) < 0.3
    wide = torch.full((5, -(-C // 32) + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, :-3] = bits(many)
    check(Zd, Zh, some_labels(5, 2, C, rng), 7, False, many, allowed=wide[:, :-3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_alternatives_of_rows_full_of_ties(dtype):
    """Few distinct values: hundreds of equal margins at every place of the order, also across waves and workgroups."""
    rng = np.random.default_rng(11)
    for n, C in ((3, 400), (3, 5000), (2, 70001), (300, 9000)):
        h = rng.integers(-3, 3, (n, C)).astype(np.float64)
        check(torch.from_numpy(h).to(DTYPES[dtype]).cuda(), h, some_labels(n, 1, C, rng), min(64, C), False, None, grad=False)


@pytest.mark.parametrize("C,reference", [(9, False), (9, True), (1500, False), (1500, True)])
def test_gradient_against_differences(C, reference):
    """Central differences of the weighted sum of the outputs, in fp64: step 1e-5, error of the order 1e-10 of the third
    derivative, whose entries are below 10 here, plus 1e-16 * |sum| / 1e-5."""
    rng = np.random.default_rng(C)
    n, width = 3, C - reference
    Zd, Zh = rows(n, width, torch.float64, rng, scale=1.0)
    lab = torch.from_numpy(rng.integers(0, C, (n, 2)).astype(np.int32)).cuda()
    g, l, h = (torch.from_numpy(rng.standard_normal(s)).cuda() for s in ((n, 2), n, n))
    out = ssn_logprobs(Zd, lab, reference=reference)
    dZ = ssn_logprobs_grad(Zd, lab, out, dlogp=g, dlse=l, dentropy=h, reference=reference)

    def value(Z):
        o = ssn_logprobs(Z, lab, reference=reference)
        return float((g * o["logp"]).sum() + (l * (o["maxpart"] + o["logpart"])).sum() + (h * o["entropy"]).sum())

    picks = {0, 1, width - 1} | {int(v) for v in lab.flatten().cpu() if v < width}
    for i in range(n):
        for c in picks:
            up, down = Zd.clone(), Zd.clone()
            up[i, c] += 1e-5
            down[i, c] -= 1e-5
            assert abs((value(up) - value(down)) / 2e-5 - float(dZ[i, c])) <= 1e-8


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("C", [7, 90, 777, 9001])
def test_gradient_in_place_and_into_wider_rows(dtype, C):
    rng = np.random.default_rng(C)
    dt = DTYPES[dtype]
    Zd, _ = rows(6, C, dt, rng, pad=5)
    lab = torch.from_numpy(rng.integers(0, C, 6).astype(np.int32)).cuda()
    out = ssn_logprobs(Zd, lab)
    assert out["logp"].shape == (6,)
    g = torch.ones(6, dtype=out["logp"].dtype, device="cuda")
    want = ssn_logprobs_grad(Zd, lab, out, dlogp=g)
    buf = torch.full((8, C + 4), 7.0, dtype=dt, device="cuda")
    ssn_logprobs_grad(Zd, lab, out, dlogp=g, dZ=buf[1:7, :C])
    assert torch.equal(buf[1:7, :C], want)
    buf[1:7, :C] = 7.0
    assert bool((buf == 7.0).all()), "columns or rows beside the gradient were written"
    ssn_logprobs_grad(Zd, lab, out, dlogp=g, dZ=Zd)
    assert torch.equal(Zd, want)
    assert bool(torch.isnan(Zd._base[:, C:]).all())


def test_outputs_stop_at_their_last_row():
    """Rows behind the last one keep what they hold, and a call computes only what it is asked for."""
    Z = torch.randn(5, 6000, device="cuda")
    lab = torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    big = dict(logp=torch.full((7, 3), 9.0, device="cuda"), top_ids=torch.full((7, 4), 9, dtype=torch.int32, device="cuda"),
               top_logp=torch.full((7, 4), 9.0, device="cuda"), entropy=torch.full((7,), 9.0, device="cuda"))
    out = {name: t[:5] for name, t in big.items()}
    got = ssn_logprobs(Z, lab, k=4, out=out)
    full = ssn_logprobs(Z, lab, k=4)
    assert got is out and "maxpart" not in got
    for name, t in big.items():
        assert torch.equal(t[:5], full[name]) and bool((t[5:] == 9).all())


def test_no_rows_no_labels():
    out = ssn_logprobs(torch.empty((0, 50), device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda"), k=3)
    assert out["logp"].shape == (0, 2) and out["top_ids"].shape == (0, 3)
    ssn_logprobs_grad(torch.empty((0, 50), device="cuda"), None, out, dlse=torch.empty(0, device="cuda"))
    out = ssn_logprobs(torch.zeros((4, 1000), device="cuda"))
    assert "logp" not in out and float(out["entropy"][0]) == pytest.approx(np.log(1000.0), abs=1e-5)


def test_rows_beyond_two_to_the_31_elements():
    """Rows a gigabyte apart: element offsets pass 2^32."""
    ld = 3 * (1 << 29) + 1
    buf = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(5)
    for C in (40, 5000):
        Zd = torch.as_strided(buf, (3, C), (ld, 1))
        h = torch.from_numpy(rng.standard_normal((3, C))).to(torch.bfloat16)
        Zd.copy_(h.cuda())
        check(Zd, h.double().numpy(), some_labels(3, 2, C, rng), 5, False, None)


@pytest.mark.parametrize("n,C,k", [(40, 11, 3), (3, 40000, 9), (300, 5000, 0)])
def test_captured_and_replayed_on_another_stream(n, C, k):
    """Forward and gradient in one graph, replayed on new margins with eager calls in between: bit for bit the eager results
    (the kernels add in a fixed order)."""
    rng = np.random.default_rng(C)
    Z = torch.empty(n, C, device="cuda")
    lab = torch.from_numpy(some_labels(n, 1, C, rng).astype(np.int32)).cuda()
    g, h = torch.randn(n, 1, device="cuda"), torch.randn(n, device="cuda")

    def both(Z, out=None, dZ=None):
        out = ssn_logprobs(Z, lab, k=k, out=out)
        return out, ssn_logprobs_grad(Z, lab, out, dlogp=g, dentropy=h, dZ=dZ)

    Z.normal_()
    out, dZ = both(Z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(Z, out, dZ)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(Z, out, dZ)
    for i in range(4):
        Z.normal_()
        want, wantg = both(Z)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dZ, wantg)
        for name in want:
            assert torch.equal(out[name], want[name]), name


def test_two_streams_at_once():
    """Calls that need a workspace, on two streams at once, do not disturb each other."""
    Z = [torch.randn(2, 60000, device="cuda") for _ in range(2)]
    want = [ssn_logprobs(z, k=8) for z in Z]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(ssn_logprobs(Z[i], k=8))
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i]:
            assert all(torch.equal(o[name], want[i][name]) for name in want[i])


def test_refusals():
    Z = torch.zeros(4, 100, device="cuda")
    lab = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    for kw, status in ((dict(k=65), binding.SSN_E_UNSUPPORTED), (dict(k=-1), binding.SSN_E_INVALID_ARG)):
        with pytest.raises((SsnError, RuntimeError)) as e:
            ssn_logprobs(Z, lab, **kw)
        assert not isinstance(e.value, SsnError) or e.value.status == status
    with pytest.raises(SsnError) as e:
        ssn_logprobs(Z[:, :3], lab, k=4)
    assert e.value.status == binding.SSN_E_INVALID_ARG
    with pytest.raises(SsnError) as e:
        ssn_logprobs(Z, torch.zeros(4, 65, dtype=torch.int32, device="cuda"))
    assert e.value.status == binding.SSN_E_UNSUPPORTED
    with pytest.raises(SsnError) as e:                                       # rows on top of each other
        ssn_logprobs(torch.zeros(1, 100, device="cuda").expand(4, 100), lab)
    assert e.value.status == binding.SSN_E_INVALID_ARG
    for bad in (dict(labels=lab.long()), dict(labels=lab[:2]), dict(labels=lab, allowed=torch.zeros(4, 3, dtype=torch.int32, device="cuda")),
                dict(labels=lab, allowed=torch.zeros(4, 4, device="cuda")), dict(labels=lab.cpu()),
                dict(labels=lab, out=dict(logp=torch.zeros(4, 1, device="cuda", dtype=torch.float64)))):
        with pytest.raises(AssertionError):
            ssn_logprobs(Z, **bad)
    with pytest.raises(AssertionError):
        ssn_logprobs(Z.t(), None)
    out = ssn_logprobs(Z, lab)
    g = torch.ones(4, 1, device="cuda")
    with pytest.raises(SsnError):                                            # labels without their gradients
        ssn_logprobs_grad(Z, lab, out)
    with pytest.raises(AssertionError):
        ssn_logprobs_grad(Z, lab, out, dlogp=g, dZ=torch.zeros(4, 99, device="cuda"))
    with pytest.raises(AssertionError):
        ssn_logprobs_grad(Z, lab, out, dlogp=g.double())
    torch.cuda.synchronize()
