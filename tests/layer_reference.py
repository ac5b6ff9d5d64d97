"""Plain 64-bit forms of the router's choice, of 4-bit matrices and of orthogonal updates, and bounds of what roundings can do to them."""
import torch

MANTISSA = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}        # half a step, relative
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def rounded(exact, dtype):
    """What one rounding to dtype may add."""
    return MANTISSA[dtype] * exact.abs() + LEAST[dtype]


# ---- choice ----------------------------------------------------------------------------------------

def choose(scores, topk, live=None, normalize=True):
    """Loops over the tokens: (ids, weights, p, counts, counted)."""
    tokens, experts = scores.shape
    ids = torch.full((tokens, topk), -1, dtype=torch.int64)
    w = torch.zeros((tokens, topk), dtype=torch.float64)
    p = torch.zeros((tokens, experts), dtype=torch.float64)
    counted = 0
    for t in range(tokens):
        row = scores[t].double().tolist()
        if live is not None and not live[t]:
            continue
        able = [e for e in range(experts) if row[e] != float("-inf")]
        if not able:
            continue
        counted += 1
        best = sorted(able, key=lambda e: (0, 0.0, e) if row[e] != row[e] else (1, -row[e], e))[:topk]
        x = torch.tensor(row, dtype=torch.float64)
        ex = (x - x[best[0]]).exp()
        ex[[e for e in range(experts) if e not in able]] = 0.0
        p[t] = ex / ex.sum()
        ids[t, :len(best)] = torch.tensor(best)
        w[t, :len(best)] = ex[best] / (ex[best].sum() if normalize else ex.sum())
    counts = torch.bincount(ids[ids >= 0], minlength=experts)
    return ids, w, p, counts, counted


def balance(p, counts, counted):
    """(shares, loss, f)."""
    experts = len(counts)
    f = counts.double() / max(1, int(counts.sum()))
    shares = p.sum(0) / max(1, counted)
    return shares, experts * (f * shares).sum(), f


def choose_grad(ids, w, p, f, counted, dw, dloss, normalize):
    """(gradient, sum of the magnitudes that make it)."""
    experts = p.shape[1]
    at, some = ids.clamp(min=0), (ids >= 0).double()
    dw = dw * some
    dot, big = (w * dw).sum(1, keepdim=True), (w * dw.abs()).sum(1, keepdim=True)
    if normalize:
        d = torch.zeros_like(p).scatter_add_(1, at, w * (dw - dot) * some)
        size = torch.zeros_like(p).scatter_add_(1, at, w * (dw.abs() + big) * some)
    else:
        d = p * (torch.zeros_like(p).scatter_add_(1, at, dw) - dot)
        size = p * (torch.zeros_like(p).scatter_add_(1, at, dw.abs()) + big)
    if dloss is not None:
        scale = dloss * experts / max(1, counted)
        fp = (f * p).sum(1, keepdim=True)
        d = d + scale * p * (f - fp)
        size = size + abs(scale) * p * (f + fp)
    return d, size


# ---- 4 bits ----------------------------------------------------------------------------------------

def quantize(w, group, zeros, scale_dtype):
    """Codes (rows x cols, int64), scales and zero points (groups x rows, float64), by the definition with its roundings: float32 quotients."""
    rows, cols = w.shape
    w = w.float()
    n = -(-cols // group)
    codes, scales, points = torch.zeros((rows, cols), dtype=torch.int64), torch.zeros((n, rows), dtype=torch.float64), torch.zeros((n, rows), dtype=torch.float64)
    for g in range(n):
        x = w[:, g * group:(g + 1) * group]
        if zeros:
            lo, hi = x.amin(1).clamp(max=0), x.amax(1).clamp(min=0)
            s = ((hi - lo) / torch.full_like(hi, 15.0)).to(scale_dtype).float()
        else:
            s = (x.abs().amax(1) / torch.full_like(x[:, 0], 7.0)).to(scale_dtype).float()
        fine = s.isfinite() & x.isfinite().all(1)
        s = torch.where(fine, s, float("nan"))
        some = fine & (s > 0)
        z = torch.where(some, (-lo / s).round().clamp(max=15.0), torch.where(fine, 0.0, 8.0)) if zeros else torch.full_like(s, 8.0)
        q = ((x / s[:, None]).round() + z[:, None]).clamp(0, 15)
        codes[:, g * group:(g + 1) * group] = torch.where(some[:, None], q, z[:, None]).long()
        scales[g], points[g] = s.double(), z.double()
    return codes, scales, points


def codes_of(data, cols):
    return torch.stack((data & 15, data >> 4), dim=-1).flatten(-2)[..., :cols].long()


def values(codes, scale, zero, group):
    at = torch.arange(codes.shape[1], device=codes.device) // group
    return (codes.double() - (8.0 if zero is None else zero.double().T[:, at])) * scale.double().T[:, at]


def product(x, codes, scale, zero, group):
    """(x W^T, the sum of magnitudes of what is added: of code - 8, and of 8 - zero, apart)."""
    at = torch.arange(codes.shape[1], device=codes.device) // group
    s, x = scale.double().T[:, at], x.double()
    z = torch.zeros_like(s) if zero is None else 8.0 - zero.double().T[:, at]
    q = codes.double() - 8.0
    return x @ ((q + z) * s).T, x.abs() @ ((q.abs() + z.abs()) * s.abs()).T


# ---- orthogonal updates --------------------------------------------------------------------------------

def orthogonalize(x, steps, coefficients, eps):
    a, b, c = coefficients
    z = x.double()
    z = z / (z.square().sum().sqrt() + eps)
    z = z.T if z.shape[0] > z.shape[1] else z
    for _ in range(steps):
        gram = z @ z.T
        z = a * z + (b * gram + c * (gram @ gram)) @ z
    return z.T if x.shape[0] > x.shape[1] else z


def parts(v, scale, n):
    """v as the sum of n float16 numbers at a scale."""
    left, out = v * scale, torch.zeros_like(v)
    for _ in range(n):
        h = left.to(torch.float16).double()
        out, left = out + h, left - h
    return out / scale


def orthogonalize_in_parts(x, steps, coefficients, eps, n):
    """The same with operands of n parts, diagonals apart in 32 bits: what the method itself loses."""
    a, b, c = coefficients
    z = x.double()
    z = (z / (z.square().sum().sqrt() + eps)).float().double()
    z = z.T if z.shape[0] > z.shape[1] else z
    for _ in range(steps):
        zh = parts(z, 4096.0, n)
        gram = (zh @ zh.T).float().double()
        d = gram.diagonal()
        off = gram - torch.diag(d)
        oh = parts(off, 16384.0, n)
        p = b * off + c * ((d[:, None] + d[None, :]) * off + oh @ oh) + torch.diag(a + b * d + c * d * d)
        p = p.float().double()
        e = p.diagonal()
        z = (e[:, None] * z + parts(p - torch.diag(e), 4096.0, n) @ zh).float().double()
    return z.T if x.shape[0] > x.shape[1] else z


def orthogonalize_bound(x, coefficients, eps, n):
    """One step: its exact result, and entry by entry what operands rounded to n parts, 32-bit sums and 32-bit roundings can change it by."""
    a, b, c = (abs(v) for v in coefficients)
    u, f = (2.0 ** -11 if n == 1 else 2.0 ** -21), 2.0 ** -24
    z = x.double()
    z = (z / (z.square().sum().sqrt() + eps)).abs()
    z = z.T if z.shape[0] > z.shape[1] else z
    m, k = z.shape
    tiny = 2.0 ** -24                                   # half the least step of float16, at the operands' scales of 2^12 and more: 2^-25 / 2^12
    dz = f * z
    dzh = dz + u * z + tiny / 4096
    gram = z @ z.T
    dg = dzh @ z.T + z @ dzh.T + (k + 8) * 2 * f * gram
    off = gram - torch.diag(gram.diagonal())
    doh = dg + u * off + tiny / 16384
    square = off @ off
    d, dd = gram.diagonal(), dg.diagonal()
    dp = (b * dg + c * ((d[:, None] + d[None, :]) * dg + (dd[:, None] + dd[None, :]) * gram + doh @ off + off @ doh + (m + 8) * 2 * f * square)
          + 8 * f * (a + b * gram + c * (2 * (d[:, None] + d[None, :]) * gram + square)))
    p = a * torch.eye(m, dtype=torch.float64, device=z.device) + b * gram + c * gram @ gram
    dph = dp + u * p + tiny / 4096
    bound = dph @ z + p @ dzh + (m + 8) * 2 * f * (p @ z)
    return orthogonalize(x, 1, coefficients, eps), (bound.T if x.shape[0] > x.shape[1] else bound)


def orthogonalize_as_run(x, steps, coefficients, eps, rounded):
    """Steps on bfloat16 as they are made, in 64 bits but for the roundings: X in two parts, operands of one, and, if `rounded`, the off-diagonals of A in the linear
    terms of b A + c A^2 the rounded ones that the product takes."""
    a, b, c = coefficients
    z = x.double()
    z = (z / (z.square().sum().sqrt() + eps)).float().double()
    z = z.T if z.shape[0] > z.shape[1] else z
    for _ in range(steps):
        z, zh = parts(z, 4096.0, 2), parts(z, 4096.0, 1)
        gram = zh @ zh.T
        d = gram.diagonal()
        off = gram - torch.diag(d)
        oh = parts(off, 16384.0, 1)
        square = oh @ oh
        p = (b + c * (d[:, None] + d[None, :])) * (oh if rounded else off) + c * square
        e = a + b * d + c * (d * d + square.diagonal())
        z = e[:, None] * z + parts(p - torch.diag(p.diagonal()), 4096.0, 1) @ zh
    return z.T if x.shape[0] > x.shape[1] else z
