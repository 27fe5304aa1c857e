"""Cases that four more operators around the layers are measured on.

A case is one pass through one of them, as a program that trains a network over a large
vocabulary, or answers with it, makes it:

  norm      root-mean-square norm of hidden rows with the residual's addition, forward and
            backward; `coded` is its form for answering, which leaves 8-bit codes with scales
  four      outputs of a layer whose weights are held in 4 bits, with one power-of-two scale for
            each 32 columns, O = H W^T; `quantize4` is its other half, weights into 4 bits
  logprobs  log probabilities of given tokens, the entropy and the likeliest alternatives;
            `logtrain` adds the backward pass
  clip      the norm over all gradients of a step, and the gradients scaled to a largest norm

Sizes are those of the named workloads in synth/ (D from 2000 to 1 000 000, d from 32 to 1024,
m up to 512), of the paper's vocabulary (793 471 words, d = 300) and of the header's limits.
"""
import math

import numpy as np
import torch

own = False  # False: the operators in elementary torch operations; True: the library's calls

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def listed():
    return [
        # one token's hidden row for each of 64 sequences, on the way to outputs in 8 bits
        dict(name="coded_tokens", op="coded", rows=64, cols=500, type="bf16", residual=True),
        # a training batch of sentences at the benchmarked width
        dict(name="norm_batch", op="norm", rows=8_191, cols=500, type="f32", residual=True),
        # every hidden row of a long packed batch
        dict(name="norm_rows", op="norm", rows=65_536, cols=1024, type="bf16", residual=True),
        # the paper's vocabulary after more training: weights into 4 bits again
        dict(name="quantize4_words", op="quantize4", D=793_471, d=300, type="f32"),
        # outputs of a single example over the benchmarked vocabulary
        dict(name="four_one", op="four", D=200_000, d=500, m=1, type="f32", out="f32"),
        # the benchmarked minibatch
        dict(name="four_batch", op="four", D=200_000, d=500, m=128, type="f32", out="f32"),
        # the widest workload: D = 500 000, d = 1024, m = 512
        dict(name="four_wide", op="four", D=500_000, d=1024, m=512, type="bf16", out="bf16"),
        # one example's chosen word and the twenty likeliest
        dict(name="logprobs_one", op="logprobs", m=1, D=200_000, K=1, top=20, type="f32",
             spread=3.0, temperature=True),
        # the paper's vocabulary in 16 bits: 64 rows scored, with five alternatives
        dict(name="logprobs_words", op="logprobs", m=64, D=793_471, K=1, top=5, type="bf16",
             spread=2.0, temperature=False),
        # the benchmarked minibatch's ten targets a row, with an entropy bonus, both directions
        dict(name="logtrain_batch", op="logtrain", m=128, D=200_000, K=10, top=0, type="f32",
             spread=2.0, temperature=False),
        # the gradients of a small network: latency counts
        dict(name="clip_small", op="clip", tensors=40, values=400_000, type="mixed", above=True),
        # those of a network with an explicit table of the paper's vocabulary
        dict(name="clip_words", op="clip", tensors=24, values=260_000_000, type="f32",
             above=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "coded", "quantize4", "four", "four", "four", "logprobs",
                     "logprobs", "logtrain", "logtrain", "clip", "clip"])
    kind = rng.choice(["f32", "bf16", "f16"])
    d = _log_int(rng, 16, 1024)
    if rng.random() < 0.5:
        d = max(16, d // 4 * 4)  # half of the widths in use are multiples of four
    if op in ("norm", "coded"):
        return dict(op=op, rows=_log_int(rng, 1, 65_536), cols=d, type=kind,
                    residual=rng.random() < 0.6)
    if op == "quantize4":
        return dict(op=op, D=min(_log_int(rng, 1_000, 1_000_000), 256_000_000 // d), d=d,
                    type=kind)
    if op == "clip":
        return dict(op=op, tensors=_log_int(rng, 1, 60), values=_log_int(rng, 10_000, 200_000_000),
                    type=rng.choice(["f32", "bf16", "f16", "mixed"]), above=rng.random() < 0.7)
    D = _log_int(rng, 1_000, 1_000_000)
    if op == "four":
        D, m = min(D, 512_000_000 // d), _log_int(rng, 1, 512)
        return dict(op=op, D=D, d=d, m=min(m, 256_000_000 // D), type=kind,
                    out=rng.choice(["f32", "bf16", "f16"]))
    return dict(op=op, m=min(_log_int(rng, 1, 512), max(1, 51_000_000 // D)), D=D,
                K=_log_int(rng, 1, 16), top=0 if op == "logtrain" else rng.choice([0, 1, 5, 20, 32]),
                type=kind, spread=round(rng.uniform(0.3, 4.0), 2),
                temperature=rng.random() < 0.5)


# ------------------------------------------------------------------------------ inputs
def _normal(g, *shape, scale=1.0):
    return torch.empty(shape, device=DEVICE).normal_(0.0, scale, generator=g)


def _shapes(c):
    """Shapes and types of the gradients, by the case alone: many small vectors, square and wide
    matrices, and as columns of a wider one every fifth."""
    rng = np.random.default_rng(1000 * c["tensors"] + c["values"] % 1000)
    share = rng.exponential(size=c["tensors"]) ** 2
    count = np.maximum(1, share / share.sum() * c["values"]).astype(np.int64)
    shapes = []
    for i, n in enumerate(count.tolist()):
        kind = ("f32", "bf16", "f16")[i % 3] if c["type"] == "mixed" else c["type"]
        cols = int(rng.integers(16, 1025))
        if n < 4 * cols:
            shapes.append((kind, 1, n, n))
        else:
            shapes.append((kind, n // cols, cols, 2 * cols if i % 5 == 4 else cols))
    return shapes


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"case": c}
    if c["op"] == "clip":
        s["grads"], s["out"] = [], []
        for kind, rows, cols, ld in _shapes(c):
            t = _normal(g, rows, ld, scale=float(rng.uniform(0.001, 0.1))).to(DTYPES[kind])
            s["grads"].append(t[:, :cols])
            # gradients that stay as they are are left in place, others go where the step reads
            s["out"].append(torch.empty_like(t)[:, :cols] if c["above"] else t[:, :cols])
        total = sum(float(t.double().square().sum()) for t in s["grads"])
        s["max_norm"] = float(np.float32(math.sqrt(total) * (0.3 if c["above"] else 3.0)))
        if own:  # the gradients' buffers stay from step to step, and so does their list
            import paper_1412_7091_amd as lst

            s["clip"] = lst.GradientClip(s["grads"], out=s["out"])
        return s
    dt = DTYPES[c["type"]]
    if c["op"] in ("norm", "coded"):
        n = (c["rows"], c["cols"])
        s["x"] = _normal(g, *n).to(dt)
        s["residual"] = _normal(g, *n, scale=2.0).to(dt) if c["residual"] else None
        s["weight"] = 1.0 + _normal(g, c["cols"], scale=0.2)
        if c["op"] == "norm":
            s["grad_y"] = _normal(g, *n).to(dt)
            s["grad_sum"] = _normal(g, *n).to(dt) if c["residual"] else None
    elif c["op"] in ("four", "quantize4"):
        b = 1.0 / math.sqrt(c["d"])
        W = torch.empty((c["D"], c["d"]), device=DEVICE).uniform_(-b, b, generator=g)
        if c["op"] == "quantize4":
            s["W"] = W.to(dt)
        else:
            s["codes"], s["scales"] = _quantize4(W)
            s["H"] = _normal(g, c["m"], c["d"], scale=b).to(dt)
    else:
        m, D, K = c["m"], c["D"], c["K"]
        # words sorted by frequency: the common ones are likelier, a few may not be said
        logits = _normal(g, m, D, scale=c["spread"])
        logits -= 0.5 * torch.log(torch.arange(1, D + 1, device=DEVICE, dtype=torch.float32))
        logits[torch.rand((m, D), device=DEVICE, generator=g) < 0.01] = -math.inf
        s["logits"] = logits.to(dt)
        tokens = np.minimum(D - 1, np.exp(rng.uniform(0, math.log(D), (m, K))).astype(np.int64))
        tokens[rng.random((m, K)) < 0.05] = -1  # unused places of a shorter list
        s["tokens"] = torch.from_numpy(tokens.astype(np.int32)).to(DEVICE)
        s["temperature"] = None
        if c["temperature"]:
            s["temperature"] = torch.from_numpy(rng.uniform(0.5, 1.5, m).astype(np.float32)).to(DEVICE)
        if c["op"] == "logtrain":
            s["grad_logp"] = _normal(g, m, K)
            s["grad_entropy"] = _normal(g, m, scale=0.1)
    if own and c["op"] in ("norm", "coded"):  # a layer that the program keeps
        import paper_1412_7091_amd as lst

        s["layer"] = lst.RMSNorm(s["weight"], eps=EPS)
    return s


# ---------------------------------------------------------------------- the plain forms
def _norm(x, residual, weight):
    """(y in 32 bits, the sum as it is stored, the factor of each row)."""
    total = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h = total.float()
    rstd = 1 / torch.sqrt((h * h).mean(dim=1) + EPS)
    return h * rstd[:, None] * weight, total, rstd


def _norm_backward(total, rstd, weight, grad_y, grad_sum):
    hat = total.float() * rstd[:, None]
    dy = grad_y.float()
    a = dy * weight
    dx = rstd[:, None] * (a - hat * (a * hat).mean(dim=1, keepdim=True))
    if grad_sum is not None:
        dx = dx + grad_sum.float()
    return dx.to(total.dtype), (dy * hat).sum(dim=0)


def _blocks(X, size):
    n, d = X.shape
    blocks = (d + size - 1) // size
    return torch.nn.functional.pad(X.float(), (0, blocks * size - d)).view(n, blocks, size)


def _quantize8(X):
    """e4m3 codes as bytes, one biased exponent for each 128 columns: the smallest power of two
    that no value passes 448 of."""
    x = _blocks(X, 128)
    mant, e = torch.frexp(x.abs().amax(dim=2))
    e = torch.where(mant <= 0.875, e - 9, e - 8).clamp(min=-127)
    e = torch.where(mant == 0, -127, e)
    codes = (x * torch.exp2(-e.double()).float()[:, :, None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8).view(x.shape[0], -1), (e + 127).to(torch.uint8)


def _quantize4(X):
    """e2m1 codes, two a byte with the lower column in the lower half, and one biased exponent for
    each 32 columns: the smallest power of two that no value passes 6 of."""
    x = _blocks(X, 32)
    mant, e = torch.frexp(x.abs().amax(dim=2))
    e = torch.where(mant <= 0.75, e - 3, e - 2).clamp(min=-127)
    e = torch.where(mant == 0, -127, e)
    v = x * torch.exp2(-e.double()).float()[:, :, None]
    a = v.abs()
    # values 0, 1/2, 1, 3/2, 2, 3, 4, 6; halfway between two of them the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) +
            (a >= 3.5) + (a > 5)) + 8 * torch.signbit(v).to(torch.uint8)
    code = code.view(x.shape[0], -1, 2)
    return code[:, :, 0] + 16 * code[:, :, 1], (e + 127).to(torch.uint8)


def _values4(codes, scales):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6],
                         device=codes.device)
    q = table[torch.stack((codes & 15, codes >> 4), dim=2).int()]
    n, blocks = scales.shape
    scale = torch.exp2(scales.double() - 127).float()
    return (q.view(n, blocks, 32) * scale[:, :, None]).view(n, -1)


def _probabilities(logits, temperature):
    """z = (x - max) / T with -inf where there is no probability, sums of exp(z), and exp(z)."""
    x = logits.float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    z = x - x.amax(dim=1, keepdim=True)
    if temperature is not None:
        z = z / temperature[:, None]
    e = torch.exp(z)
    return z, e.sum(dim=1, keepdim=True), e


def _logprobs(s, c):
    z, total, e = _probabilities(s["logits"], s["temperature"])
    log_total = torch.log(total)
    entropy = log_total[:, 0] - torch.where(e > 0, e * z, 0.0).sum(dim=1) / total[:, 0]
    t = s["tokens"].long()
    logp = z.gather(1, t.clamp(min=0)) - log_total
    out = [torch.where(t >= 0, logp, 0.0), entropy]
    if c["top"]:
        # by value, equal ones by index
        x = torch.where(torch.isnan(s["logits"]), -math.inf, s["logits"])
        ids = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :c["top"]]
        out += [ids.int(), z.gather(1, ids) - log_total]
    if c["op"] == "logprobs":
        return out
    p = e / total
    used = (t >= 0) & torch.isfinite(logp)
    g = torch.where(used, s["grad_logp"], 0.0)
    ge = s["grad_entropy"][:, None]
    logs = torch.where(e > 0, z - log_total, 0.0)
    grad = -p * (g.sum(dim=1, keepdim=True) + ge * (logs + entropy[:, None]))
    grad.scatter_add_(1, t.clamp(min=0), g)
    if s["temperature"] is not None:
        grad = grad / s["temperature"][:, None]
    return out + [grad.to(s["logits"].dtype)]


def _clip(s):
    # squares of many small values: the sums in 64 bits
    total = torch.stack([t.double().square().sum() for t in s["grads"]]).sum()
    norm = torch.sqrt(total).float()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    done = [o.copy_(t.float() * factor) for t, o in zip(s["grads"], s["out"])]
    return norm, done


# ---------------------------------------------------------------------------- the pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "norm":
        y, total, rstd = _norm(s["x"], s["residual"], s["weight"])
        dx, dw = _norm_backward(total, rstd, s["weight"], s["grad_y"], s["grad_sum"])
        return y.to(s["x"].dtype), total, rstd, dx, dw
    if c["op"] == "coded":
        y, total, _ = _norm(s["x"], s["residual"], s["weight"])
        codes, scales = _quantize8(y)
        return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), total
    if c["op"] == "quantize4":
        # two values a byte: compared as they are held
        return _quantize4(s["W"])
    if c["op"] == "four":
        H = _values4(*_quantize4(s["H"]))
        return (H @ _values4(s["codes"], s["scales"]).T).to(DTYPES[c["out"]])
    if c["op"] == "clip":
        return _clip(s)
    return _logprobs(s, c)


def _run_own(s, c):
    import paper_1412_7091_amd as lst

    if c["op"] == "norm":
        y, total, rstd = s["layer"].forward(s["x"], s["residual"], save=True)
        dx, dw = s["layer"].backward(total, rstd, s["grad_y"], s["grad_sum"])
        return y, total, rstd, dx, dw
    if c["op"] == "coded":
        codes, scales, total = s["layer"].forward_coded(s["x"], s["residual"])
        return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), total
    if c["op"] == "quantize4":
        return lst.lst_quantize_four(s["W"])
    if c["op"] == "four":
        return lst.lst_scores_four(s["H"], s["codes"], s["scales"], dtype=DTYPES[c["out"]])
    if c["op"] == "clip":
        return s["clip"].clip(s["max_norm"]), s["out"]
    logp, entropy, ids, best, saved = lst.lst_logprobs(
        s["logits"], s["tokens"], top=c["top"], temperature=s["temperature"],
        save=c["op"] == "logtrain")
    out = [logp, entropy] + ([ids, best] if c["top"] else [])
    if c["op"] == "logprobs":
        return out
    return out + [lst.lst_logprobs_backward(s["logits"], s["tokens"], saved, s["grad_logp"],
                                            s["grad_entropy"], temperature=s["temperature"])]


# ------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    if c["op"] == "clip":
        n = [(SIZE[kind], rows * cols) for kind, rows, cols, _ in _shapes(c)]
        return {"bytes": sum(e * k for e, k in n) * (2 if c["above"] else 1),
                "flops": 3 * sum(k for _, k in n)}
    e = SIZE[c["type"]]
    if c["op"] in ("norm", "coded"):
        n = c["rows"] * c["cols"]
        # in: x, grad_y (residual, grad_sum); out: y, grad_x (sum)
        if c["op"] == "norm":
            return {"bytes": n * e * (7 if c["residual"] else 4) + 4 * c["rows"] + 8 * c["cols"],
                    "flops": 15 * n}
        held = c["rows"] * ((c["cols"] + 127) // 128) * 129
        return {"bytes": n * e * (3 if c["residual"] else 1) + held + 4 * c["cols"],
                "flops": 6 * n}
    if c["op"] in ("four", "quantize4"):
        held = c["D"] * ((c["d"] + 31) // 32) * 17  # codes and scales, whole blocks
        if c["op"] == "quantize4":
            return {"bytes": c["D"] * c["d"] * e + held, "flops": 3 * c["D"] * c["d"]}
        return {"bytes": held + c["m"] * (c["d"] * e + c["D"] * SIZE[c["out"]]),
                "flops": 2 * c["m"] * c["D"] * c["d"]}
    n = c["m"] * c["D"]
    small = c["m"] * (8 * c["K"] + 4 + 8 * c["top"])
    if c["op"] == "logprobs":
        return {"bytes": n * e + small, "flops": 6 * n}
    return {"bytes": 2 * n * e + small + 8 * c["m"] * c["K"], "flops": 12 * n}


# --------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    with torch.no_grad():
        if c["op"] in ("norm", "coded"):
            return _exact_norm(c, s)
        if c["op"] == "quantize4":
            parts = [_exact_codes4(w.double()) for w in s["W"].split(65_536)]
            return (torch.cat([_exact_pack(q, neg) for q, neg, _ in parts]),
                    torch.cat([(e + 127).to(torch.uint8) for _, _, e in parts]))
        if c["op"] == "four":
            q, neg, e = _exact_codes4(s["H"].double())
            H = _exact_rows(torch.where(neg, -q, q), e, 32)
            W = [_exact_rows(_exact_decode4(k), v.double() - 127, 32)
                 for k, v in zip(s["codes"].split(65_536), s["scales"].split(65_536))]
            return torch.cat([H @ w.T for w in W], dim=1)
        if c["op"] == "clip":
            norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.double())) ** 2
                                       for t in s["grads"]))
            factor = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
            return (torch.tensor(norm, dtype=torch.float64),
                    [t.double() * factor for t in s["grads"]])
        return _exact_logprobs(c, s)


def _exact_norm(c, s):
    dt = s["x"].dtype
    h = s["x"].double()
    total = s["x"]
    if s["residual"] is not None:
        # the stored sum, which the norm is of, is rounded to the rows' type
        total = s["x"].add(s["residual"]) if dt == torch.float32 else (
            h + s["residual"].double()).float().to(dt)
        h = total.double()
    w = s["weight"].double()
    rms = torch.sqrt(h.square().sum(dim=1, keepdim=True) / c["cols"] + EPS)
    y = h / rms * w
    if c["op"] == "coded":
        # a sixteenth of a step of a code at most: as values of the types they are held in
        q, e = _exact_codes8(y)
        return q.to(torch.float64), torch.exp2(e), total.double()
    dy = s["grad_y"].double()
    inner = (dy * w * h).sum(dim=1, keepdim=True) / c["cols"]
    dx = dy * w / rms - h * inner / rms ** 3
    if s["grad_sum"] is not None:
        dx = dx + s["grad_sum"].double()
    return y, total.double(), 1 / rms[:, 0], dx, (dy * h / rms).sum(dim=0)


def _exact_scale(x, most):
    """Exponent of the smallest power of two that no value of the last axis passes `most` of."""
    big = x.abs().amax(dim=2)
    e = torch.ceil(torch.log2(big / most))
    # the logarithm may round across a whole number
    e = torch.where(most * torch.exp2(e - 1) >= big, e - 1, e)
    e = torch.where(most * torch.exp2(e) < big, e + 1, e)
    return torch.where(big > 0, e, -127.0).clamp(min=-127)


def _exact_split(X, size):
    n, d = X.shape
    blocks = -(-d // size)
    x = torch.zeros((n, blocks * size), dtype=torch.float64, device=X.device)
    x[:, :d] = X
    return x.view(n, blocks, size)


def _exact_codes8(X):
    x = _exact_split(X, 128)
    e = _exact_scale(x, 448.0)
    v = x / torch.exp2(e)[:, :, None]
    # three bits behind the leading one, and steps of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).view(x.shape[0], -1), e


def _exact_codes4(X):
    """(magnitudes of the codes' values, their signs, exponents of the scales)."""
    x = _exact_split(X, 32)
    e = _exact_scale(x, 6.0)
    v = x / torch.exp2(e)[:, :, None]
    # one bit behind the leading one, and steps of 1/2 below 1
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=1.0))) - 1)
    return ((torch.round(v.abs() / step) * step).view(x.shape[0], -1),
            torch.signbit(v).view(x.shape[0], -1), e)


def _exact_pack(q, negative):
    code = torch.where(q < 2, 2 * q, torch.where(q < 4, q + 2, q / 2 + 4)).to(torch.int32)
    code = torch.where(negative, code + 8, code).view(q.shape[0], -1, 2)
    return (code[:, :, 0] + 16 * code[:, :, 1]).to(torch.uint8)


def _exact_decode4(codes):
    c = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1).int()
    e, m = (c >> 1) & 3, (c & 1).double()
    size = torch.where(e > 0, (2 + m) * torch.exp2(e.double() - 2), m / 2)
    return torch.where(c > 7, -size, size)


def _exact_rows(q, e, size):
    return q * torch.exp2(e).repeat_interleave(size, dim=1)


def _exact_logprobs(c, s):
    """Row after row."""
    outs = []
    for i in range(c["m"]):
        z = s["logits"][i].double()
        if s["temperature"] is not None:
            z = z / s["temperature"][i].double()
        log = z - torch.logsumexp(z, dim=0)  # -inf where masked
        p = log.exp()
        safe = torch.where(p > 0, log, 0.0)
        entropy = -(p * safe).sum()
        t = s["tokens"][i].long()
        logp = torch.where(t >= 0, log[t.clamp(min=0)], 0.0)
        row = [logp, entropy]
        if c["top"]:
            order = torch.argsort(s["logits"][i].float(), descending=True, stable=True)[:c["top"]]
            row += [order.int(), log[order]]
        if c["op"] == "logtrain":
            g = torch.where((t >= 0) & torch.isfinite(logp), s["grad_logp"][i].double(), 0.0)
            ge = s["grad_entropy"][i].double()
            grad = -p * (g.sum() + ge * (safe + entropy))
            grad.index_add_(0, t.clamp(min=0), g)
            if s["temperature"] is not None:
                grad = grad / s["temperature"][i].double()
            row.append(grad)
        outs.append(row)
    return [torch.stack(x) for x in zip(*outs)]
