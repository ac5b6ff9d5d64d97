"""Performance cases of what stands around a layer's matrix products: the router's choice of experts with its balance loss, weights in 4 bits, and
a weight update made orthogonal.  Kinds of cases:

  choose      a token's scores -> its topk experts and their weights (softmax over the experts, the chosen ones' share of it or their
              probabilities as they are); balance: choices and mean probability of each expert and the loss sum_e f_e P_e * experts;
              grad: the scores' gradient from the weights' and the loss's
  pack        a weight matrix in 4 bits with a scale, or a scale and a zero point, per group along its rows, and the values that they stand for
  packed      y = x W^T with such a weight matrix
  packed_experts  the same for rows sorted by expert, each expert with its own matrix
  ortho       a batch of matrices made orthogonal by five Newton-Schulz steps X <- aX + (bA + cA^2)X, A = X X^T, from X = G / |G|

Ties between scores go to the lowest expert.  Rows of padding (not live) have no experts, and nothing of them counts; what stands there may be
anything.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LARGEST = 20 * 4096 ** 3               # operations of the largest listed case
MOST_SCORES = 65000 * 256


def listed():
    return [
        # a few tokens in flight, served: no gradient, no loss; latency
        {"name": "choose_decode", "kind": "choose", "tokens": 24, "experts": 32, "topk": 4, "scores": "f32", "normalize": True, "balance": False, "grad": False, "padded": False},
        # a training batch: choice, loss, and the scores' gradient
        {"name": "choose_train", "kind": "choose", "tokens": 16384, "experts": 64, "topk": 4, "scores": "f32", "normalize": True, "balance": True, "grad": True, "padded": False},
        # many small experts, a padded batch of 16-bit scores (with ties), weights as probabilities
        {"name": "choose_many", "kind": "choose", "tokens": 65000, "experts": 256, "topk": 8, "scores": "bf16", "normalize": False, "balance": True, "grad": True, "padded": True},
        # a weight matrix, ragged, laid out for serving
        {"name": "pack_ragged", "kind": "pack", "batch": 1, "rows": 1300, "cols": 777, "w": "f32", "group": 32, "zeros": True, "scale": "f32"},
        # the experts of a layer laid out for serving
        {"name": "pack_experts", "kind": "pack", "batch": 16, "rows": 2048, "cols": 2048, "w": "bf16", "group": 128, "zeros": False, "scale": "f16"},
        # one token through a projection: latency and the read of the weight
        {"name": "packed_token", "kind": "packed", "rows": 1, "n": 4096, "k": 4096, "x": "bf16", "out": "bf16", "group": 128, "zeros": False, "scale": "f16"},
        # a dozen tokens in flight through a large matrix, small groups with zero points
        {"name": "packed_rows", "kind": "packed", "rows": 12, "n": 8192, "k": 8192, "x": "f16", "out": "f16", "group": 64, "zeros": True, "scale": "f16"},
        # ragged sizes, all of it in 32 bits
        {"name": "packed_ragged", "kind": "packed", "rows": 33, "n": 1300, "k": 777, "x": "f32", "out": "f32", "group": 32, "zeros": True, "scale": "f32"},
        # a few tokens in flight, four of 32 experts each
        {"name": "packed_experts", "kind": "packed_experts", "tokens": 24, "topk": 4, "experts": 32, "n": 2048, "k": 2048, "x": "bf16", "out": "bf16", "group": 128, "zeros": False, "scale": "f16"},
        # a few small matrices in 32 bits
        {"name": "ortho_small", "kind": "ortho", "batch": 4, "rows": 200, "cols": 300, "x": "f32"},
        # the update of a layer's experts
        {"name": "ortho_experts", "kind": "ortho", "batch": 16, "rows": 1024, "cols": 2048, "x": "bf16"},
        # the update of a large square weight
        {"name": "ortho_square", "kind": "ortho", "batch": 1, "rows": 4096, "cols": 4096, "x": "bf16"},
    ]


def _size(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, most of them no multiples of anything."""
    kind = rng.choice(["choose", "choose", "pack", "packed", "packed", "packed_experts", "ortho", "ortho"])
    even = (lambda v: v) if rng.random() < 0.6 else (lambda v: max(64, v // 64 * 64))
    if kind == "choose":
        experts = rng.choice([8, 16, 32, 60, 64, 128, 160, 256, 384])
        case = {"kind": kind, "tokens": _size(rng, 1, 65000), "experts": experts, "topk": rng.choice([1, 2, 4, 6, 8]),
                "scores": rng.choice(["f32", "f32", "bf16", "f16"]), "normalize": rng.random() < 0.6, "balance": rng.random() < 0.7, "grad": rng.random() < 0.7,
                "padded": rng.random() < 0.3}
        while case["tokens"] * experts > MOST_SCORES:
            case["tokens"] -= case["tokens"] // 4
        return case
    group, zeros, scale = rng.choice([32, 64, 128]), rng.random() < 0.5, rng.choice(["f16", "f16", "bf16", "f32"])
    if kind == "pack":
        return {"kind": kind, "batch": rng.choice([1, 1, 2, 8]), "rows": _size(rng, 16, 2600), "cols": even(_size(rng, 64, 8192)), "w": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "group": group, "zeros": zeros, "scale": scale}
    x = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "packed":
        return {"kind": kind, "rows": _size(rng, 1, 128), "n": even(_size(rng, 64, 10240)), "k": even(_size(rng, 64, 10240)), "x": x,
                "out": rng.choice([x, x, "f32"]), "group": group, "zeros": zeros, "scale": scale}
    if kind == "packed_experts":
        experts = rng.choice([4, 8, 16, 32])
        return {"kind": kind, "tokens": _size(rng, 1, 256), "topk": rng.choice([1, 2, 4]), "experts": experts, "n": even(_size(rng, 128, 4096)),
                "k": even(_size(rng, 128, 2048)), "x": x, "out": rng.choice([x, x, "f32"]), "group": group, "zeros": zeros, "scale": scale}
    case = {"kind": kind, "batch": rng.choice([1, 1, 2, 4, 16]), "rows": even(_size(rng, 32, 4096)), "cols": even(_size(rng, 32, 4096)), "x": rng.choice(["bf16", "bf16", "f16", "f32"])}
    while work(case)["flops"] > LARGEST:
        case["batch"] = max(1, case["batch"] // 2)
        case["cols"] -= case["cols"] // 4
    return case


# ---- inputs ------------------------------------------------------------------------------------

def _rand(r, *shape, dtype=torch.bfloat16):
    """Activations: normal, with a spread per column (a few channels are much larger), as a trained model has them."""
    x = torch.randn(shape, generator=r, device="cuda")
    return x.mul_(torch.randn((shape[-1],), generator=r, device="cuda").mul_(0.7).exp_()).to(dtype)


def _packed(r, case, batch=None):
    """Codes of two elements to a byte, the even column in the low half, rows padded to 16 bytes; scales (and zero points) groups x rows, as
    a checkpoint holds them."""
    lead = () if batch is None else (batch,)
    n, k, st = case["n"], case["k"], TYPES[case["scale"]]
    groups = -(-k // case["group"])
    data = torch.randint(0, 256, lead + (n, -(-k // 32) * 16), generator=r, device="cuda", dtype=torch.uint8)
    scale = torch.randn(lead + (groups, n), generator=r, device="cuda").mul_(0.3).exp_().mul_(0.1 * k ** -0.5).to(st)
    zero = torch.randint(5, 11, lead + (groups, n), generator=r, device="cuda").to(st) if case["zeros"] else None
    return {"data": data, "scale": scale, "zero": zero}


_handle = None


def prepare(case, seed):
    """Inputs, and where the framework's kernels run its handle and the 4-bit weights as its calls take them (the same memory)."""
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind == "choose":
        tokens, experts = case["tokens"], case["experts"]
        # uneven: some experts are chosen far more often than others
        scores = torch.randn((tokens, experts), generator=r, device="cuda") * 1.5 + torch.randn((experts,), generator=r, device="cuda") * 0.8
        s["live"] = None
        if case["padded"]:
            s["live"] = torch.rand((tokens,), generator=r, device="cuda") < 0.9
            scores = torch.where(s["live"][:, None], scores, float("nan"))
        s["scores"] = scores.to(TYPES[case["scores"]])
        if case["grad"]:
            # gradients of a loss that is a mean over the tokens, scaled where 16 bits need it
            up = 1024.0 if case["scores"] == "f16" else 1.0
            s["dweights"] = torch.randn((tokens, min(case["topk"], experts)), generator=r, device="cuda") * (up / tokens)
            s["dloss"] = 0.01 * up
    elif kind == "pack":
        w = torch.randn((case["batch"], case["rows"], case["cols"]), generator=r, device="cuda") * case["cols"] ** -0.5
        s["w"] = w.mul_(torch.randn((case["cols"],), generator=r, device="cuda").mul_(0.3).exp_()).to(TYPES[case["w"]])
    elif kind == "packed":
        s["x"], s["w"] = _rand(r, case["rows"], case["k"], dtype=TYPES[case["x"]]), _packed(r, case)
    elif kind == "packed_experts":
        score = torch.randn((case["tokens"], case["experts"]), generator=r, device="cuda")
        ids = torch.sort(score, dim=1, descending=True).indices[:, :case["topk"]].reshape(-1)
        counts = (ids[:, None] == torch.arange(case["experts"], device="cuda")).sum(0)
        s["offsets"] = torch.cat((counts.new_zeros(1), counts.cumsum(0))).to(torch.int32)
        s["counts"] = counts.tolist()                  # the plain form's loop over the experts
        s["x"] = _rand(r, ids.numel(), case["k"], dtype=TYPES[case["x"]])
        s["w"] = _packed(r, case, case["experts"])
    else:
        # a gradient: a few directions that many tokens share, and noise
        b, m, n = case["batch"], case["rows"], case["cols"]
        rank = max(1, min(m, n) // 8)
        u = torch.randn((b, m, rank), generator=r, device="cuda") * torch.linspace(0, -2, rank, device="cuda").exp()
        g = torch.bmm(u, torch.randn((b, rank, n), generator=r, device="cuda")) * rank ** -0.5
        s["x"] = ((g + torch.randn((b, m, n), generator=r, device="cuda") * 0.3) * 1e-3).to(TYPES[case["x"]])
    if own:
        _bind(s)
    return s


def _bind(s):
    global _handle
    from paper_2511_13778_amd import ozdgemm, packed
    if _handle is None:
        _handle = ozdgemm.Handle(0)
    case = s["case"]
    if isinstance(s.get("w"), dict):
        s["w"] = packed.Packed(s["w"]["data"], s["w"]["scale"], s["w"]["zero"], cols=case["k"], group=case["group"])


def run(state):
    return (_own if own else _plain)(state)


# ---- the framework's operators -----------------------------------------------------------------

def _own(s):
    from paper_2511_13778_amd import experts, orthogonal, packed
    case, h = s["case"], _handle
    kind = case["kind"]
    if kind == "choose":
        c = experts.choose(h, s["scores"], min(case["topk"], case["experts"]), live=s["live"], normalize=case["normalize"], balance=case["balance"])
        out = {"ids": c.ids, "weights": c.weights}
        if case["balance"]:
            out["counts"], out["shares"], out["loss"] = c.counts, c.shares, c.loss
        if case["grad"]:
            out["dscores"] = experts.choose_backward(h, s["scores"], c, s["dweights"], s["dloss"] if case["balance"] else None)
        return out
    if kind == "pack":
        w = packed.quantize(h, s["w"], group=case["group"], zeros=case["zeros"], scale_dtype=TYPES[case["scale"]])
        out = {"values": packed.unpack(h, w, dtype=s["w"].dtype), "scale": w.scale}
        if case["zeros"]:
            out["zero"] = w.zero
        return out
    if kind == "packed":
        return packed.gemm(h, s["x"], s["w"], dtype=TYPES[case["out"]])
    if kind == "packed_experts":
        return packed.gemm_grouped(h, s["x"], s["w"], s["offsets"], dtype=TYPES[case["out"]])
    return orthogonal.orthogonalize(h, s["x"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)


# ---- the plain form: elementary operations in 32 bits --------------------------------------------

def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "choose":
        return _plain_choose(s)
    if kind == "pack":
        return _plain_pack(s)
    if kind == "packed":
        return (s["x"].float() @ _plain_values(s["w"], case).T).to(TYPES[case["out"]])
    if kind == "packed_experts":
        y = torch.zeros((s["x"].shape[0], case["n"]), device="cuda", dtype=TYPES[case["out"]])
        at = 0
        for e, count in enumerate(s["counts"]):
            if count:
                w = {name: None if t is None else t[e] for name, t in s["w"].items()}
                y[at:at + count] = (s["x"][at:at + count].float() @ _plain_values(w, case).T).to(y.dtype)
            at += count
        return y
    # Five steps of a steep polynomial multiply an error in X by hundreds: where the result has 32 bits, 32 bits on the way are too few.
    x = s["x"].to(torch.float64 if case["x"] == "f32" else torch.float32)
    turn = case["rows"] > case["cols"]
    x = x.transpose(1, 2).contiguous() if turn else x
    x = x / (s["x"].double().square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS).to(x.dtype)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return (x.transpose(1, 2) if turn else x).to(s["x"].dtype).contiguous()


def _plain_choose(s):
    case = s["case"]
    experts, topk = case["experts"], min(case["topk"], case["experts"])
    score = s["scores"].float()
    live = torch.ones(score.shape[0], dtype=torch.bool, device=score.device) if s["live"] is None else s["live"]
    score = torch.where(live[:, None], score, 0.0)
    p = (score - score.max(dim=1, keepdim=True).values).exp()
    p = p / p.sum(dim=1, keepdim=True)
    ids = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :topk]       # stable: ties to the lowest expert
    w = p.gather(1, ids)
    total = w.sum(dim=1, keepdim=True)
    if case["normalize"]:
        w = w / total
    chosen = torch.zeros_like(p).scatter_(1, ids, 1.0) * live[:, None]
    out = {"ids": torch.where(live[:, None], ids, -1).to(torch.int32), "weights": torch.where(live[:, None], w, 0.0)}
    many = live.sum().clamp(min=1)
    if case["balance"]:
        counts = chosen.double().sum(0)
        f = counts / counts.sum().clamp(min=1)
        share = torch.where(live[:, None], p, 0.0).double().sum(0) / many
        out["counts"], out["shares"], out["loss"] = counts.to(torch.int32), share.float(), ((f * share).sum() * experts).float()
    if case["grad"]:
        dw = s["dweights"]
        if case["normalize"]:
            d = torch.zeros_like(p).scatter_(1, ids, w * (dw - (w * dw).sum(dim=1, keepdim=True)))
        else:
            d = torch.zeros_like(p).scatter_(1, ids, dw)
            d = p * (d - (w * dw).sum(dim=1, keepdim=True))
        if case["balance"]:
            d = d + (s["dloss"] * experts / many.float()) * p * (f.float() - (p * f.float()).sum(dim=1, keepdim=True))
        out["dscores"] = torch.where(live[:, None], d, 0.0).to(s["scores"].dtype)
    return out


def _by_group(w, group, fill=0.0):
    """... x cols -> ... x groups x group, filled up behind the last column."""
    cols = w.shape[-1]
    groups = -(-cols // group)
    full = w.new_full(w.shape[:-1] + (groups * group,), fill)
    full[..., :cols] = w
    return full.view(w.shape[:-1] + (groups, group))


def _plain_pack(s):
    case = s["case"]
    st, cols = TYPES[case["scale"]], case["cols"]
    w = _by_group(s["w"].float(), case["group"])
    if case["zeros"]:
        lo, hi = w.amin(-1).clamp(max=0.0), w.amax(-1).clamp(min=0.0)
        scale = ((hi - lo) / torch.full_like(hi, 15.0)).to(st)        # by a tensor: by a number it is a product with the inverse
        some = scale != 0
        zero = torch.where(some, (-lo / scale.float()).round().clamp(0, 15), 0.0)
        code = ((w / scale.float()[..., None]).round() + zero[..., None]).clamp(0, 15)
    else:
        top = w.abs().amax(-1)
        scale = (top / torch.full_like(top, 7.0)).to(st)
        some = scale != 0
        zero = torch.full_like(scale, 8.0, dtype=torch.float32)
        code = (w / scale.float()[..., None]).round().clamp(-8, 7) + 8
    values = torch.where(some[..., None], (code - zero[..., None]) * scale.float()[..., None], 0.0)
    out = {"values": values.flatten(-2)[..., :cols].to(s["w"].dtype).contiguous(), "scale": scale.transpose(-1, -2).contiguous()}
    if case["zeros"]:
        out["zero"] = zero.to(st).transpose(-1, -2).contiguous()
    return out


def _plain_values(w, case):
    """The matrix in float32."""
    k = case["k"]
    code = torch.stack((w["data"] & 15, w["data"] >> 4), dim=-1).flatten(-2)[..., :k].float()
    group = torch.arange(k, device=code.device) // case["group"]
    zero = 8.0 if w["zero"] is None else w["zero"].float().T[:, group]
    return (code - zero) * w["scale"].float().T[:, group]


# ---- what the operators are, in 64 bits ------------------------------------------------------------

def exact(case, seed):
    """run()'s outputs from their definitions in float64; whole numbers have none."""
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    kind = case["kind"]
    if kind == "choose":
        return _exact_choose(s)
    if kind == "pack":
        return _exact_pack(s)
    if kind == "packed":
        return _exact_product(s["x"], s["w"], case)
    if kind == "packed_experts":
        parts = torch.split(s["x"], s["counts"])
        return torch.cat([_exact_product(x, {n: None if t is None else t[e] for n, t in s["w"].items()}, case) for e, x in enumerate(parts)])
    out = []
    for g in s["x"].double():
        x = (g.T if g.shape[0] > g.shape[1] else g).contiguous()
        x = x / (torch.linalg.vector_norm(x) + EPS)
        for _ in range(STEPS):
            ax = (x @ x.T) @ x
            x = COEFFICIENTS[0] * x + COEFFICIENTS[1] * ax + COEFFICIENTS[2] * ((x @ x.T) @ ax)
        out.append(x.T if g.shape[0] > g.shape[1] else x)
    return torch.stack(out)


def _exact_product(x, w, case):
    n, k, group = case["n"], case["k"], case["group"]
    y = torch.zeros((x.shape[0], n), dtype=torch.float64, device=x.device)
    for g in range(-(-k // group)):
        cols = torch.arange(g * group, min(k, (g + 1) * group), device=x.device)
        byte = w["data"][:, cols // 2].to(torch.int64)
        code = torch.where(cols % 2 == 1, byte // 16, byte % 16).double()
        zero = 8.0 if w["zero"] is None else w["zero"][g].double()[:, None]
        y += (x[:, cols].double() @ (code - zero).T) * w["scale"][g].double()
    return y


def _exact_pack(s):
    """The definition's own roundings (scale to its type, quotient to 32 bits and then to a whole number) are part of it."""
    case, w = s["case"], s["w"].double()
    cols, group, st = case["cols"], case["group"], TYPES[case["scale"]]
    values, scales, zeros = torch.zeros_like(w), [], []
    for at in range(0, cols, group):
        x = w[..., at:at + group]
        if case["zeros"]:
            lo, hi = x.min(-1).values.clamp(max=0), x.max(-1).values.clamp(min=0)
            sc = ((hi - lo).float().double() / 15).float().to(st).double()
            z = torch.where(sc > 0, (-lo / sc).float().round(), 0).clamp(0, 15).double()
            q = ((x / sc[..., None]).float().round().double() + z[..., None]).clamp(0, 15)
        else:
            sc = (x.abs().max(-1).values / 7).float().to(st).double()
            z = torch.full_like(sc, 8)
            q = ((x / sc[..., None]).float().round().double() + 8).clamp(0, 15)
        values[..., at:at + group] = torch.where(sc[..., None] > 0, (q - z[..., None]) * sc[..., None], 0)
        scales.append(sc)
        zeros.append(z)
    out = {"values": values, "scale": torch.stack(scales, -2)}
    if case["zeros"]:
        out["zero"] = torch.stack(zeros, -2)
    return out


def _exact_choose(s):
    case = s["case"]
    topk = min(case["topk"], case["experts"])
    rows = torch.arange(case["tokens"], device="cuda") if s["live"] is None else s["live"].nonzero()[:, 0]
    score = s["scores"][rows].double()
    p = torch.softmax(score, 1)
    ids = torch.argsort(score, dim=1, descending=True, stable=True)[:, :topk]
    w = p.gather(1, ids)
    if case["normalize"]:
        w = w / w.sum(1, keepdim=True)

    def whole(x):
        return torch.zeros((case["tokens"], x.shape[1]), dtype=torch.float64, device="cuda").index_copy_(0, rows, x)

    out = {"ids": None, "weights": whole(w)}
    f = (torch.bincount(ids.reshape(-1), minlength=case["experts"]).double() / max(1, ids.numel()))
    if case["balance"]:
        share = p.sum(0) / max(1, len(rows))
        out["counts"], out["shares"], out["loss"] = None, share, case["experts"] * (f * share).sum()
    if case["grad"]:
        dw = s["dweights"][rows].double()
        # by the chain rule: gradient with respect to the probabilities, then through the softmax
        if case["normalize"]:
            total = p.gather(1, ids).sum(1, keepdim=True)
            at = (dw - (dw * w).sum(1, keepdim=True)) / total
        else:
            at = dw
        dp = torch.zeros_like(p).scatter_(1, ids, at)
        if case["balance"]:
            dp = dp + s["dloss"] * case["experts"] / max(1, len(rows)) * f
        out["dscores"] = whole(p * (dp - (p * dp).sum(1, keepdim=True)))
    return out


# ---- what a case cannot do without --------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if kind == "choose":
        tokens, experts, topk, e = case["tokens"], case["experts"], min(case["topk"], case["experts"]), size[case["scores"]]
        n = tokens * experts * e + tokens * topk * 8 + (8 * experts if case["balance"] else 0) + (tokens if case["padded"] else 0)
        if case["grad"]:
            n += tokens * topk * 4 + tokens * experts * e
        return {"bytes": n, "flops": tokens * experts * (12 if case["grad"] else 4)}
    groups = lambda cols: -(-cols // case["group"]) * size[case["scale"]] * (2 if case["zeros"] else 1)  # noqa: E731
    if kind == "pack":
        rows, cols = case["batch"] * case["rows"], case["cols"]
        return {"bytes": rows * (cols * (2 * size[case["w"]]) + groups(cols)), "flops": 4 * rows * cols}
    if kind in ("packed", "packed_experts"):
        n, k = case["n"], case["k"]
        rows = case["rows"] if kind == "packed" else case["tokens"] * case["topk"]
        # experts that get a token: as many as there are, if the choices go that far
        matrices = 1 if kind == "packed" else min(case["experts"], rows)
        return {"bytes": matrices * n * (k // 2 + groups(k)) + rows * (k * size[case["x"]] + n * size[case["out"]]), "flops": 2 * rows * n * k}
    b, m, n = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # A and A^2 are symmetric: half of each
    return {"bytes": 2 * b * m * n * size[case["x"]], "flops": STEPS * b * (m * m * n + m * m * m + 2 * m * m * n)}
