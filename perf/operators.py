"""What a softmax layer answers with and learns from, as cases that can be timed and compared: log probabilities of given
classes with entropy and top alternatives, their gradient, and margins of rows with a weight block held in 4 bits.

  logprobs   rows of margins (logits) -> log probabilities of given classes, entropy, the largest alternatives
  grad       the gradient of those log probabilities, of the log-sum-exp and of the entropy with respect to the margins
  margins    rows of features times a p-by-K weight block in 4 bits with a scale for each group of features

`run` computes them in plain torch operations, or, where `own` is true, by the calls of paper_1802_09113_amd.binding.

Weights in 4 bits: a code is a sign bit and a magnitude index into MAGNITUDES; a value is its code's number times the
scale (bfloat16) of its (group of features, class).  Classes go in tiles of 16, features in blocks of 128, both padded:
byte b of word j of the 16 bytes at ((tile * blocks + block) * 64 + 16 g + o) * 16 holds features
128 block + 32 j + 8 g + 2 b (low nibble) and the next one (high nibble) of class 16 tile + o; scales are laid out as
[tile][block][o][128 / group].
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f64": torch.float64, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f64": 8, "f16": 2, "bf16": 2}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# The largest matrix of margins that is drawn, and the largest from which alternatives are taken.
MAX_MARGINS = 8192 * 65536
MAX_RANKED = 64 * 131072


def listed():
    return [
        # the next token of one sequence, with its five best alternatives: one short launch after another
        dict(name="logprobs_decode_f32", kind="logprobs", n=1, C=32000, dtype="f32", reference=False, m=1, k=5,
             allowed=False, pad=0),
        # a batch of sequences answered under a grammar: a mask of allowed tokens for each, twenty alternatives
        dict(name="logprobs_serve_bf16", kind="logprobs", n=64, C=131072, dtype="bf16", reference=False, m=1, k=20,
             allowed=True, pad=0),
        # odd sizes: sixteen candidate answers per row rescored, rows of a wider buffer
        dict(name="logprobs_rescore_f16", kind="logprobs", n=509, C=50021, dtype="f16", reference=False, m=16, k=0,
             allowed=False, pad=3),
        # the loss of a training batch: one label per row, a gigabyte of margins
        dict(name="logprobs_train_bf16", kind="logprobs", n=8192, C=65536, dtype="bf16", reference=False, m=1, k=0,
             allowed=False, pad=0),
        # the framework's tall problem: seven classes with the reference class, evaluated over all its rows
        dict(name="logprobs_classes_f64", kind="logprobs", n=581012, C=7, dtype="f64", reference=True, m=1, k=3,
             allowed=False, pad=0),
        # ten classes of the image-like problem: the gradient's first factor
        dict(name="grad_classes_f64", kind="grad", n=60000, C=10, dtype="f64", reference=True, m=1, lse=False,
             entropy=False, allowed=False, pad=0),
        # a policy's update: log probability and entropy under masks of allowed actions, odd sizes
        dict(name="grad_policy_f32", kind="grad", n=1021, C=32003, dtype="f32", reference=False, m=1, lse=False,
             entropy=True, allowed=True, pad=0),
        # the backward pass of the training batch, with a penalty on the log-sum-exp
        dict(name="grad_train_bf16", kind="grad", n=8192, C=65536, dtype="bf16", reference=False, m=1, lse=True,
             entropy=False, allowed=False, pad=0),
        # a small classifier asked about one row
        dict(name="margins_small_bf16", kind="margins", n=1, p=1024, K=1000, dtype="bf16", group=32, pad=0),
        # a large output layer for one token: the weights' stream is everything
        dict(name="margins_decode_bf16", kind="margins", n=1, p=8192, K=65536, dtype="bf16", group=32, pad=0),
        # a few single-precision rows, odd everything
        dict(name="margins_few_f32", kind="margins", n=5, p=5003, K=10007, dtype="f32", group=64, pad=0),
        # a prompt's rows at once: the products begin to count
        dict(name="margins_prompt_f16", kind="margins", n=256, p=4096, K=32768, dtype="f16", group=128, pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["logprobs", "grad", "margins"])
    pad = rng.choice([0, 0, 1, 8])
    if kind == "margins":
        p, K = _log_int(rng, 300, 8192), _log_int(rng, 500, 65536)
        n = _log_int(rng, 1, max(1, min(256, 256 * 4096 * 32768 // (p * K))))
        return dict(kind=kind, n=n, p=p, K=K, dtype=rng.choice(["bf16", "f16", "f32"] if n <= 64 else ["bf16", "f16"]),
                    group=rng.choice([32, 64, 128]), pad=pad)
    dtype = rng.choice(["f32", "f16", "bf16", "bf16", "f64"])
    k = _log_int(rng, 1, 32) if kind == "logprobs" and rng.random() < 0.5 else 0
    most = MAX_RANKED if k else MAX_MARGINS if BYTES[dtype] == 2 else MAX_MARGINS // 4
    if rng.random() < 0.3:
        C = _log_int(rng, 2, 1000)                      # classes of a small problem, many rows
        n = _log_int(rng, 1000, min(600000, most // C))
    else:
        C = _log_int(rng, 5000, 131072)
        n = _log_int(rng, 1, min(8192, most // C))
    case = dict(kind=kind, n=n, C=C, dtype=dtype, reference=rng.random() < 0.3, m=rng.choice([1, 1, 1, 4, 16]))
    if kind == "logprobs":
        case["k"] = min(k, C)
    else:
        case["lse"], case["entropy"] = rng.random() < 0.5, rng.random() < 0.5
    return dict(case, allowed=rng.random() < 0.3, pad=pad)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _rows(n, width, pad, dtype, g, scale=1.0, shift=0.0):
    """Normal rows in storage that is `pad` elements wider."""
    buf = torch.empty(n, width + pad, device="cuda", dtype=dtype)
    step = max(1, (1 << 26) // (width + pad))
    for lo in range(0, n, step):
        part = buf[lo:lo + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda", dtype=torch.float32) * scale + shift)
    return buf[:, :width]


def _margins(case, g):
    """Margins as an output layer gives them: normal with a spread of two, a few classes of each row well above."""
    width = case["C"] - case["reference"]
    Z = _rows(case["n"], width, case["pad"], DTYPES[case["dtype"]], g, 2.0)
    if width > 64:
        at = torch.randint(width, (case["n"], 8), generator=g, device="cuda")
        Z.scatter_(1, at, (6 + 2 * torch.randn(at.shape, generator=g, device="cuda")).to(Z.dtype))
    return Z


def _labels(case, g, Z):
    """Given classes: the row's best for half of them, any class for the others, one in fifty a row's padding (-1)."""
    any_one = torch.randint(case["C"], (case["n"], case["m"]), generator=g, device="cuda")
    best = Z[:, :4096].argmax(1, keepdim=True) if Z.shape[1] else any_one[:, :1]
    u = torch.rand(any_one.shape, generator=g, device="cuda")
    return torch.where(u < 0.02, -1, torch.where(u < 0.5, best, any_one)).to(torch.int32)


def _allowed(case, g):
    """Bits of allowed classes: about half of them, none at all in one row of sixteen."""
    words = torch.randint(-2 ** 31, 2 ** 31, (case["n"], (case["C"] + 31) // 32), generator=g, device="cuda", dtype=torch.int64)
    return torch.where((torch.rand(case["n"], 1, generator=g, device="cuda") < 1 / 16), 0, words).to(torch.int32)


def _code_of(ratio):
    """The code of a ratio weight / scale: nearest magnitude, a tie to the even index, no negative zero."""
    a = ratio.abs()
    index = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return index + ((ratio < 0) & (index > 0)).to(torch.uint8) * 8


def _weights(case, g):
    """A trained layer in 4 bits: normal weights, every group's scale the smallest that clips none of them."""
    p, K, group = case["p"], case["K"], case["group"]
    tiles, blocks = -(-K // 16), -(-p // 128)
    packed, scales = [], []
    step = max(1, (1 << 26) // (blocks * 128 * 16))
    for lo in range(0, tiles, step):
        t = min(step, tiles - lo)
        w = 0.02 * torch.randn(t * 16, blocks * 128, generator=g, device="cuda", dtype=torch.float32)
        w[max(0, K - lo * 16):] = 0
        w[:, p:] = 0
        w = w.view(t * 16, -1, group)
        most = w.abs().amax(2)
        s = (most / 6).to(torch.bfloat16)
        s = torch.where(6 * s.float() < most, (s.view(torch.int16) + 1).view(torch.bfloat16), s)
        codes = _code_of(w / torch.where(s > 0, s, 1).float()[..., None])
        codes = codes.view(t, 16, blocks, 4, 4, 4, 2).permute(0, 2, 4, 1, 3, 5, 6)
        packed.append((codes[..., 0] | (codes[..., 1] << 4)).reshape(t, blocks, 64, 16))
        scales.append(s.view(t, 16, blocks, 128 // group).permute(0, 2, 1, 3).contiguous())
    return torch.cat(packed), torch.cat(scales)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, dt = case["n"], DTYPES[case["dtype"]]
    state = dict(case)
    if case["kind"] == "margins":
        state["packed"], state["scales"] = _weights(case, g)
        state["X"] = _rows(n, case["p"], case["pad"], dt, g)
        state["Z"] = torch.empty(n, case["K"], device="cuda", dtype=dt)
        return state
    stat = torch.float64 if dt == torch.float64 else torch.float32
    Z = state["Z"] = _margins(case, g)
    state["labels"] = _labels(case, g, Z)
    state["allowed"] = _allowed(case, g) if case["allowed"] else None
    if case["kind"] == "logprobs":
        out = dict(logp=torch.empty(n, case["m"], device="cuda", dtype=stat))
        for name in ("maxpart", "logpart", "entropy"):
            out[name] = torch.empty(n, device="cuda", dtype=stat)
        if case["k"]:
            out["top_ids"] = torch.empty(n, case["k"], device="cuda", dtype=torch.int32)
            out["top_logp"] = torch.empty(n, case["k"], device="cuda", dtype=stat)
        state["out"] = out
        return state
    # what the forward pass left behind, and the gradients that come back from the loss
    state["forward"] = _plain_logprobs(Z, state["labels"], 0, case["reference"], state["allowed"])
    state["dlogp"] = (torch.randn(n, case["m"], generator=g, device="cuda", dtype=torch.float32) / n).to(stat)
    state["dlse"] = (torch.rand(n, generator=g, device="cuda", dtype=torch.float32) / n).to(stat) if case["lse"] else None
    state["dentropy"] = (torch.rand(n, generator=g, device="cuda", dtype=torch.float32) / n).to(stat) if case["entropy"] else None
    state["dZ"] = torch.empty_like(Z.contiguous())
    return state


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _plain_mask(allowed, C):
    """The bits of int32 words as truth values, C for each row."""
    bits = (allowed[:, :, None] >> torch.arange(32, device=allowed.device, dtype=torch.int32)) & 1
    return bits.flatten(1)[:, :C].bool()


def _plain_all(Z, reference, allowed):
    """The margins of all classes: the reference class's zero appended, -inf where a class is not allowed."""
    z = Z if Z.dtype == torch.float64 else Z.float()
    if reference:
        z = torch.cat([z, z.new_zeros(z.shape[0], 1)], 1)
    if allowed is not None:
        z = torch.where(_plain_mask(allowed, z.shape[1]), z, -math.inf)
    return z


def _plain_logprobs(Z, labels, k, reference, allowed):
    z = _plain_all(Z, reference, allowed)
    top = z.amax(1)
    empty = top == -math.inf
    d = z - torch.where(empty, 0, top)[:, None]
    e = torch.exp(d)
    s = torch.where(empty, 1, e.sum(1))
    logpart = torch.log(s)
    entropy = logpart - torch.where(e > 0, e * d, 0).sum(1) / s
    given = torch.where(labels >= 0, d.gather(1, labels.clamp(min=0).long()) - logpart[:, None], 0)
    out = dict(logp=given, maxpart=top, logpart=logpart, entropy=entropy)
    if k:
        best, ids = torch.sort(d, dim=1, descending=True, stable=True)
        best, ids = best[:, :k], ids[:, :k].to(torch.int32)
        out["top_ids"] = torch.where(best == -math.inf, -1, ids)
        out["top_logp"] = best - logpart[:, None]
    return out


def _plain_grad(Z, labels, forward, dlogp, dlse, dentropy, reference, allowed):
    z = _plain_all(Z, reference, allowed)
    empty = (forward["maxpart"] == -math.inf)[:, None]
    logp = torch.where(empty, -math.inf, z - torch.where(empty, 0, forward["maxpart"][:, None]) - forward["logpart"][:, None])
    p = torch.exp(logp)
    there = (labels >= 0) & (forward["logp"] > -math.inf)
    given = torch.where(there, dlogp, 0)
    weight = given.sum(1, keepdim=True)
    if dlse is not None:
        weight = weight - dlse[:, None]
    if dentropy is not None:
        weight = weight + dentropy[:, None] * (torch.where(p > 0, logp, 0) + forward["entropy"][:, None])
    grad = (-p * weight).scatter_add_(1, labels.clamp(min=0).long(), given)
    return (grad[:, :-1] if reference else grad).to(Z.dtype)


def _plain_weights(packed, scales, p, K, group):
    """The weight block in 32 bits, K rows of p."""
    tiles, blocks = packed.shape[:2]
    codes = torch.stack([packed & 15, packed >> 4], -1).view(tiles, blocks, 4, 16, 4, 4, 2)
    codes = codes.permute(0, 3, 1, 4, 2, 5, 6).reshape(tiles * 16, -1)
    numbers = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), device=packed.device)[codes.int()]
    s = scales.float().permute(0, 2, 1, 3).reshape(tiles * 16, -1)
    return (numbers.view(tiles * 16, -1, group) * s[..., None]).view(tiles * 16, -1)[:K, :p]


def run(state):
    if own:
        from paper_1802_09113_amd import binding
        if state["kind"] == "logprobs":
            return binding.ssn_logprobs(state["Z"], state["labels"], k=state["k"], reference=state["reference"],
                                        allowed=state["allowed"], out=state["out"])
        if state["kind"] == "grad":
            return binding.ssn_logprobs_grad(state["Z"], state["labels"], state["forward"], dlogp=state["dlogp"],
                                             dlse=state["dlse"], dentropy=state["dentropy"], reference=state["reference"],
                                             allowed=state["allowed"], dZ=state["dZ"])
        block = binding.Q4Block(state["packed"], state["scales"], state["p"], state["K"], state["group"])
        return binding.ssn_q4_margins(block, state["X"], state["Z"])
    if state["kind"] == "logprobs":
        return _plain_logprobs(state["Z"], state["labels"], state["k"], state["reference"], state["allowed"])
    if state["kind"] == "grad":
        return _plain_grad(state["Z"], state["labels"], state["forward"], state["dlogp"], state["dlse"], state["dentropy"],
                           state["reference"], state["allowed"])
    W = _plain_weights(state["packed"], state["scales"], state["p"], state["K"], state["group"])
    return (state["X"].float() @ W.t()).to(state["X"].dtype)


# ---- the same results in 64 bits, from the definitions ---------------------------------------------------------------

def _exact_mask(case, state, lo, hi):
    words = state["allowed"][lo:hi].to(torch.int64) & 0xFFFFFFFF
    c = torch.arange(case["C"], device="cuda")
    return (words[:, c // 32] >> (c % 32)) % 2 == 1


def _exact_rows(case, state, lo, hi):
    """Log probabilities of all classes of some rows: z - log sum exp z over the allowed classes, -inf for the others."""
    z = torch.zeros(hi - lo, case["C"], device="cuda", dtype=torch.float64)
    z[:, :state["Z"].shape[1]] = state["Z"][lo:hi]
    if case["allowed"]:
        z[~_exact_mask(case, state, lo, hi)] = -math.inf
    logp = torch.log_softmax(z, 1)
    return z, torch.where(torch.isnan(logp), -math.inf, logp)


def _exact_logprobs(case, state, lo, hi):
    z, logp = _exact_rows(case, state, lo, hi)
    top, first = z.max(1)
    each = torch.arange(hi - lo, device="cuda")
    labels = state["labels"][lo:hi].long()
    given = logp[each[:, None], labels.clamp(min=0)]
    given[labels < 0] = 0
    logpart = torch.where(top > -math.inf, -logp[each, first], 0)
    out = dict(logp=given, maxpart=top, logpart=logpart, entropy=torch.special.entr(torch.exp(logp)).sum(1))
    if case["k"]:
        ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["k"]]
        out["top_logp"] = logp[each[:, None], ids]
        out["top_ids"] = torch.where(out["top_logp"] > -math.inf, ids, -1).to(torch.int32)
    return out


def _exact_grad(case, state, lo, hi):
    _, logp = _exact_rows(case, state, lo, hi)
    p = torch.exp(logp)
    grad = torch.zeros_like(p)
    labels, dlogp = state["labels"][lo:hi].long(), state["dlogp"][lo:hi].double()
    each = torch.arange(hi - lo, device="cuda")
    for t in range(case["m"]):                       # d logp_y = (one at y) - p
        c = labels[:, t].clamp(min=0)
        w = torch.where((labels[:, t] >= 0) & (logp[each, c] > -math.inf), dlogp[:, t], 0)
        grad -= w[:, None] * p
        grad[each, c] += w
    if case["lse"]:                                  # d lse = p
        grad += state["dlse"][lo:hi].double()[:, None] * p
    if case["entropy"]:                              # d H = -p (logp + H)
        h = torch.special.entr(p).sum(1, keepdim=True)
        grad -= state["dentropy"][lo:hi].double()[:, None] * torch.where(p > 0, p * (logp + h), 0)
    return grad[:, :state["Z"].shape[1]]


def _exact_margins(case, state, lo, hi):
    """Margins of the classes of tiles lo to hi, feature by feature out of the packed words."""
    j, c = torch.arange(case["p"], device="cuda"), torch.arange(lo * 16, min(hi * 16, case["K"]), device="cuda")
    b, r = j // 128, j % 128
    lane = (r % 32) // 8 * 16 + (c % 16)[:, None]
    byte = state["packed"][(c // 16)[:, None], b, lane, r // 32 * 4 + r % 8 // 2].long()
    code = torch.where(j % 2 == 1, byte // 16, byte % 16)
    size = torch.tensor(MAGNITUDES, device="cuda", dtype=torch.float64)[code % 8]
    scale = state["scales"][(c // 16)[:, None], b, (c % 16)[:, None], r // case["group"]].double()
    return state["X"].double() @ torch.where(code < 8, size, -size).mul_(scale).t().contiguous()


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "margins":
        tiles = -(-case["K"] // 16)
        step = max(1, (1 << 26) // (16 * case["p"]))
        return torch.cat([_exact_margins(case, state, lo, min(tiles, lo + step)) for lo in range(0, tiles, step)], 1)
    one = _exact_logprobs if case["kind"] == "logprobs" else _exact_grad
    step = max(1, (1 << 26) // case["C"])
    parts = [one(case, state, lo, min(case["n"], lo + step)) for lo in range(0, case["n"], step)]
    if case["kind"] == "grad":
        return torch.cat(parts)
    return {name: torch.cat([q[name] for q in parts]) for name in parts[0]}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    """The margins (or weights, codes and scales) once, the other inputs once, every output once.  A class costs a
    subtraction, an exponential and two sums; its gradient a subtraction, an exponential and a product."""
    n, e = case["n"], BYTES[case["dtype"]]
    if case["kind"] == "margins":
        p, K = case["p"], case["K"]
        return dict(bytes=K * p // 2 + 2 * K * -(-p // case["group"]) + n * (p + K) * e, flops=2 * n * p * K)
    C, m, stat = case["C"] - case["reference"], case["m"], 8 if case["dtype"] == "f64" else 4
    mask = n * 4 * -(-case["C"] // 32) if case["allowed"] else 0
    if case["kind"] == "logprobs":
        return dict(bytes=n * (C * e + m * (4 + stat) + 3 * stat + case["k"] * (4 + stat)) + mask, flops=5 * n * C)
    extra = 2 * stat + (case["lse"] + 2 * case["entropy"]) * stat
    return dict(bytes=n * (2 * C * e + m * (4 + 2 * stat) + extra) + mask, flops=(3 + 3 * case["entropy"]) * n * C)
