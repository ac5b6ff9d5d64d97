"""Performance cases of the 8-bit block-scaled operators: quantiser, matrix product, experts' products, tokens sorted by expert and back.

A matrix in 8-bit floats (e4m3 or e5m2) has a scale for each block of 128 along its rows ("rows"), or for each
128 x 128 block ("blocks"), as E8M0 (a biased exponent in a byte) or in float32.  Kinds of cases:

  quantize  x -> 8-bit floats and scales: by "rows", "both" (rows of x, and rows of its transpose), "blocks" (x and its
            transpose share the scales of their 128 x 128 blocks: a weight laid out for both directions)
  gemm      C = A B^T of two such matrices; B scaled by "blocks" (a weight) or by "rows" (activations, gradients)
  linear    a training step of a linear layer: x, w, dy in bfloat16 -> y, dx, dw, all quantised on the way
  experts   rows sorted by expert times each expert's weight
  experts_grad   the gradients of that product: of its rows, and of the weights (contraction over each expert's rows)
  dispatch  tokens sorted by expert and gathered; grad: the gradient that flows back to the tokens too
  combine   experts' rows back to their tokens, weighted and summed; grad: gradients of rows and weights too
  layer     a serving step: sorted, gathered and quantised, experts' products, back to the tokens

Routing comes from random scores with a bias per expert, so loads are uneven and some experts get nothing; a few
choices are dropped (-1).
"""
import math

import torch

own = False

BLOCK = 128
LARGEST = 2 * 8192 ** 3                 # operations of the largest listed case
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}  # largest finite value: 1.75 * 2^8, 1.75 * 2^15


def listed():
    return [
        # activations of a few tokens in front of a product: latency
        {"name": "quantize_tokens", "kind": "quantize", "rows": 16, "cols": 4096, "x": "bf16", "q": "e4m3", "scale": "e8m0", "form": "rows"},
        # activations of a training step, ragged, for the forward product and for the weight gradient
        {"name": "quantize_both", "kind": "quantize", "rows": 4100, "cols": 8192, "x": "bf16", "q": "e4m3", "scale": "f32", "form": "both"},
        # one token through a projection: the weight is read once
        {"name": "gemm_token", "kind": "gemm", "m": 1, "n": 4096, "k": 4096, "qa": "e4m3", "scale": "e8m0", "form": "blocks", "out": "bf16"},
        # the ragged sizes of the FP64 benchmark, scales of any value as checkpoints hold them, result in 32 bits
        {"name": "gemm_ragged", "kind": "gemm", "m": 1000, "n": 1300, "k": 777, "qa": "e4m3", "scale": "f32", "form": "blocks", "out": "f32"},
        # a prompt or training product at the headline benchmark's size
        {"name": "gemm_8192", "kind": "gemm", "m": 8192, "n": 8192, "k": 8192, "qa": "e4m3", "scale": "e8m0", "form": "blocks", "out": "bf16"},
        # training step of a linear layer, 4096 tokens, e5m2 gradients
        {"name": "linear_train", "kind": "linear", "m": 4096, "n": 2048, "k": 4096, "scale": "e8m0"},
        # a few tokens in flight through 32 experts: sort, gather, quantise, products, back
        {"name": "layer_decode", "kind": "layer", "tokens": 24, "topk": 4, "experts": 32, "n": 2048, "k": 2048, "scale": "e8m0"},
        # a prompt through 16 experts, scales in float32
        {"name": "experts_prompt", "kind": "experts", "tokens": 8192, "topk": 2, "experts": 16, "n": 4096, "k": 2048, "scale": "f32", "out": "bf16"},
        # gradients of an expert layer's product
        {"name": "experts_train", "kind": "experts_grad", "tokens": 4096, "topk": 2, "experts": 8, "n": 2048, "k": 2048, "scale": "e8m0"},
        # a few tokens sorted and gathered: latency
        {"name": "dispatch_decode", "kind": "dispatch", "tokens": 33, "topk": 8, "experts": 128, "cols": 2048, "x": "bf16", "grad": False},
        # a training batch sorted and gathered, and its gradient back
        {"name": "dispatch_train", "kind": "dispatch", "tokens": 16384, "topk": 4, "experts": 64, "cols": 2048, "x": "bf16", "grad": True},
        # the same batch back to its tokens, with the gradients of the experts' rows and of the weights
        {"name": "combine_train", "kind": "combine", "tokens": 16384, "topk": 4, "experts": 64, "cols": 2048, "x": "bf16", "grad": True},
    ]


def _size(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, most of them no multiples of a tile."""
    kind = rng.choice(["quantize", "gemm", "gemm", "gemm", "linear", "layer", "experts", "experts_grad", "dispatch", "combine"])
    even = (lambda v: v) if rng.random() < 0.7 else (lambda v: max(128, v // 128 * 128))
    scale = rng.choice(["e8m0", "f32"])
    if kind == "quantize":
        return {"kind": kind, "rows": _size(rng, 1, 16384), "cols": even(_size(rng, 100, 16384)), "x": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "q": rng.choice(["e4m3", "e5m2"]), "scale": scale, "form": rng.choice(["rows", "both", "blocks"])}
    if kind == "gemm":
        case = {"kind": kind, "m": _size(rng, 1, 8192), "n": even(_size(rng, 64, 8192)), "k": even(_size(rng, 64, 16384)),
                "qa": rng.choice(["e4m3", "e4m3", "e5m2"]), "scale": scale, "form": rng.choice(["blocks", "blocks", "rows"]),
                "out": rng.choice(["bf16", "bf16", "f16", "f32"])}
        while 2 * case["m"] * case["n"] * case["k"] > LARGEST:
            case["k"] -= case["k"] // 4
        return case
    if kind == "linear":
        return {"kind": kind, "m": _size(rng, 200, 8192), "n": even(_size(rng, 200, 4096)), "k": even(_size(rng, 200, 4096)), "scale": scale}
    experts = rng.choice([4, 8, 16, 32, 60, 64])
    topk = rng.choice([1, 2, 4, min(8, experts)])
    if kind == "layer":
        return {"kind": kind, "tokens": _size(rng, 1, 256), "topk": topk, "experts": experts, "n": even(_size(rng, 256, 4096)),
                "k": even(_size(rng, 256, 4096)), "scale": scale}
    if kind == "experts":
        case = {"kind": kind, "tokens": _size(rng, 1, 8192), "topk": topk, "experts": experts, "n": even(_size(rng, 256, 4096)),
                "k": even(_size(rng, 256, 4096)), "scale": scale, "out": rng.choice(["bf16", "bf16", "f16", "f32"])}
        while 2 * case["tokens"] * topk * case["n"] * case["k"] > LARGEST:
            case["tokens"] -= case["tokens"] // 4
        return case
    if kind == "experts_grad":
        return {"kind": kind, "tokens": _size(rng, 64, 8192), "topk": min(topk, 4), "experts": min(experts, 16), "n": even(_size(rng, 256, 2048)),
                "k": even(_size(rng, 256, 2048)), "scale": scale}
    case = {"kind": kind, "tokens": _size(rng, 1, 32768), "topk": topk, "experts": rng.choice([experts, 2 * experts, 256]), "cols": even(_size(rng, 100, 4096)),
            "x": rng.choice(["bf16", "bf16", "f16", "f32"]), "grad": rng.random() < 0.6}
    while case["tokens"] * topk * case["cols"] > 16384 * 4 * 2048:
        case["tokens"] -= case["tokens"] // 4
    return case


# ---- inputs ------------------------------------------------------------------------------------

def _rand(r, *shape, dtype=torch.bfloat16):
    """Activations: normal, with a spread per column (a few channels are much larger), as a trained model has them."""
    x = torch.randn(shape, generator=r, device="cuda")
    return x.mul_(torch.randn((shape[-1],), generator=r, device="cuda").mul_(0.7).exp_()).to(dtype)


def _route(r, tokens, topk, experts):
    """Chosen experts (tokens x topk, -1: dropped), int64 as a top-k gives them, and their weights."""
    score = torch.randn((tokens, experts), generator=r, device="cuda") + torch.randn((experts,), generator=r, device="cuda") * 0.8
    top, ids = score.topk(topk, dim=1)
    w = top.softmax(dim=1)
    return ids.masked_fill(torch.rand((tokens, topk), generator=r, device="cuda") < 0.01, -1), w


def _quantized(r, rows, cols, q, scale, form, batch=None):
    """A matrix in 8-bit floats as a program holds it: rows padded to 16 bytes, scales' rows to four.  Scales in float32 get any value."""
    nb, rb = -(-cols // BLOCK), rows if form == "rows" else -(-rows // BLOCK)
    lead = () if batch is None else (batch,)
    data = torch.zeros(lead + (rows, -(-cols // 16) * 16), device="cuda", dtype=TYPES[q])
    for part in (data.unbind(0) if lead else (data,)):
        part[:, :cols] = (torch.randn((rows, cols), generator=r, device="cuda") * (TOP[q] / 6)).clamp_(-TOP[q], TOP[q]).to(TYPES[q])
    s = torch.zeros(lead + (rb, -(-nb // 4) * 4), device="cuda")
    s[..., :nb] = torch.randn(lead + (rb, nb), generator=r, device="cuda") * 0.8 - 10.0
    return {"data": data, "cols": cols, "rows_per_scale": 1 if form == "rows" else BLOCK,
            "scale": (s.round() + 127).to(torch.uint8) if scale == "e8m0" else torch.exp2(s)}


_handle = None


def prepare(case, seed):
    """Inputs, and where the framework's kernels run its handle and the 8-bit matrices as its calls take them (the same memory)."""
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind == "quantize":
        s["x"] = _rand(r, case["rows"], case["cols"], dtype=TYPES[case["x"]])
    elif kind == "gemm":
        s["a"] = _quantized(r, case["m"], case["k"], case["qa"], case["scale"], "rows")
        s["b"] = _quantized(r, case["n"], case["k"], "e4m3", case["scale"], case["form"])
    elif kind == "linear":
        s["x"] = _rand(r, case["m"], case["k"])
        s["w"] = (torch.randn((case["n"], case["k"]), generator=r, device="cuda") * case["k"] ** -0.5).to(torch.bfloat16)
        s["dy"] = _rand(r, case["m"], case["n"]) * 1e-3
    else:
        ids, s["weights"] = _route(r, case["tokens"], case["topk"], case["experts"])
        slots = ids.numel()
        if kind == "layer":
            s["ids"], s["x"] = ids, _rand(r, case["tokens"], case["k"])
            s["w"] = _quantized(r, case["n"], case["k"], "e4m3", case["scale"], "blocks", case["experts"])
        elif kind == "dispatch":
            s["ids"], s["x"] = ids, _rand(r, case["tokens"], case["cols"], dtype=TYPES[case["x"]])
            if case["grad"]:
                s["dxs"] = _rand(r, slots, case["cols"], dtype=TYPES[case["x"]])
        else:
            s["offsets"], s["order"], s["place"] = _sort(ids, case["experts"])
            s["counts"] = (s["offsets"][1:] - s["offsets"][:-1]).tolist()      # the plain form's loop over the experts
            if kind == "combine":
                s["ys"] = _rand(r, slots, case["cols"], dtype=TYPES[case["x"]])
                if case["grad"]:
                    s["dy"] = _rand(r, case["tokens"], case["cols"], dtype=TYPES[case["x"]])
            elif kind == "experts":
                s["a"] = _quantized(r, slots, case["k"], "e4m3", case["scale"], "rows")
                s["w"] = _quantized(r, case["n"], case["k"], "e4m3", case["scale"], "blocks", case["experts"])
            else:
                s["xs"] = _rand(r, slots, case["k"])
                s["dys"] = _rand(r, slots, case["n"]) * 1e-3
                s["wt"] = _quantized(r, case["k"], case["n"], "e4m3", case["scale"], "blocks", case["experts"])
    if own:
        _bind(s)
    return s


def _bind(s):
    global _handle
    from paper_2511_13778_amd import experts, ozdgemm, scaled
    if _handle is None:
        _handle = ozdgemm.Handle(0)
    for key in ("a", "b", "w", "wt"):
        if isinstance(s.get(key), dict):
            m = s[key]
            s[key] = scaled.Scaled(m["data"], m["scale"], cols=m["cols"], block_rows=m["rows_per_scale"])
    if "order" in s:
        s["routing"] = experts.Routing(s["offsets"], s["order"], s["place"], s["case"]["topk"])


def run(state):
    return (_own if own else _plain)(state)


# ---- the framework's operators -----------------------------------------------------------------

def _own(s):
    from paper_2511_13778_amd import experts, scaled
    case, h = s["case"], _handle
    kind = case["kind"]
    if kind == "quantize":
        q, sc = TYPES[case["q"]], _scale_type(case)
        form = case["form"]
        got = scaled.quantize(h, s["x"], dtype=q, scale_dtype=sc, block_rows=BLOCK if form == "blocks" else 1,
                              which="rows" if form == "rows" else "both")
        return {k: v for m, name in zip((got,) if form == "rows" else got, ("", "t_"))
                for k, v in ((name + "q", m.values()), (name + "scale", m.scales()))}
    if kind == "gemm":
        return scaled.gemm(h, s["a"], s["b"], dtype=TYPES[case["out"]])
    if kind == "linear":
        sc = _scale_type(case)
        x, xt = scaled.quantize(h, s["x"], scale_dtype=sc, which="both")
        w, wt = scaled.quantize(h, s["w"], scale_dtype=sc, block_rows=BLOCK, which="both")
        d, dt = scaled.quantize(h, s["dy"], dtype=torch.float8_e5m2, scale_dtype=sc, which="both")
        return {"y": scaled.gemm(h, x, w), "dx": scaled.gemm(h, d, wt), "dw": scaled.gemm(h, dt, xt, dtype=torch.float32)}
    if kind == "experts":
        return scaled.gemm_grouped(h, s["a"], s["w"], s["offsets"], dtype=TYPES[case["out"]])
    if kind == "experts_grad":
        sc = _scale_type(case)
        d, dt = scaled.quantize(h, s["dys"], dtype=torch.float8_e5m2, scale_dtype=sc, which="both", offsets=s["offsets"])
        xt = scaled.quantize(h, s["xs"], scale_dtype=sc, which="columns", offsets=s["offsets"])
        return {"dx": scaled.gemm_grouped(h, d, s["wt"], s["offsets"]),
                "dw": scaled.gemm_grouped_k(h, dt, xt, s["offsets"], dtype=torch.float32)}
    if kind == "layer":
        routing = experts.sort_tokens(h, s["ids"], case["experts"])
        a = scaled.quantize(h, s["x"], scale_dtype=_scale_type(case), routing=routing)
        ys = scaled.gemm_grouped(h, a, s["w"], routing.offsets)
        return experts.combine(h, ys, routing, s["weights"])
    if kind == "dispatch":
        routing = experts.sort_tokens(h, s["ids"], case["experts"])
        out = {"offsets": routing.offsets, "order": routing.order, "place": routing.place, "xs": experts.gather(h, s["x"], routing)}
        if case["grad"]:
            out["dx"] = experts.combine(h, s["dxs"], routing)
        return out
    out = {"y": experts.combine(h, s["ys"], s["routing"], s["weights"])}
    if case["grad"]:
        out["dys"], out["dw"] = experts.combine_backward(h, s["dy"], s["ys"], s["routing"], s["weights"])
    return out


def _scale_type(case):
    return torch.uint8 if case["scale"] == "e8m0" else torch.float32


# ---- the plain form: elementary operations in 32 bits --------------------------------------------

def _sort(ids, experts):
    """offsets (experts + 1), order (slot -> choice, -1 behind the last), place (choice -> slot or -1); choices of an expert in their own order."""
    flat = ids.reshape(-1).to(torch.int64)
    key = torch.where(flat < 0, experts, flat)
    by = torch.sort(key, stable=True).indices
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device).index_add_(0, key, torch.ones_like(key))
    ends = counts[:experts].cumsum(0)
    offsets = torch.cat((ends.new_zeros(1), ends)).to(torch.int32)
    slots = torch.arange(flat.numel(), device=ids.device)
    live = slots < ends[-1]
    order = torch.where(live, by, -1).to(torch.int32)
    place = torch.empty_like(by).index_copy_(0, by, torch.where(live, slots, -1)).to(torch.int32)
    return offsets, order, place.view(ids.shape)


def _quantize(x, q, form="rows"):
    """(8-bit floats, exponents of the scales) of a matrix: scales are the least powers of two that keep a block in range."""
    rows, cols = x.shape
    x = x.float()
    high = 1 if form == "rows" else BLOCK
    nr, nc = -(-rows // high), -(-cols // BLOCK)
    full = x.new_zeros((nr * high, nc * BLOCK))
    full[:rows, :cols] = x
    tiles = full.view(nr, high, nc, BLOCK)
    top = tiles.abs().amax(dim=(1, 3))
    frac, e = torch.frexp(top / TOP[q])
    e = torch.where(frac == 0.5, e - 1, e)
    e = torch.where(top == 0, 0, e).clamp(-126, 126)
    out = (tiles * _power(-e).view(nr, 1, nc, 1)).view(nr * high, nc * BLOCK)[:rows, :cols].to(TYPES[q])
    return out, e


def _power(e):
    """2^e in 32 bits for whole e in [-126, 127]: the exponent field itself, no library power in between."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scales(e, kind):
    return (e + 127).to(torch.uint8) if kind == "e8m0" else _power(e)


def _values(m):
    """What an 8-bit matrix stands for, in 32 bits."""
    cols = m["cols"]
    s = _power(m["scale"].int() - 127) if m["scale"].dtype == torch.uint8 else m["scale"]
    x = m["data"][..., :cols].float()
    s = s.repeat_interleave(BLOCK, dim=-1)[..., :cols]
    return x * (s if m["rows_per_scale"] == 1 else s.repeat_interleave(BLOCK, dim=-2)[..., :x.shape[-2], :])


def _rounded(x, q, form="rows"):
    """x after quantisation, in 32 bits."""
    v, e = _quantize(x, q, form)
    s = _power(e).repeat_interleave(BLOCK, dim=1)[:, :x.shape[1]]
    return v.float() * (s if form == "rows" else s.repeat_interleave(BLOCK, dim=0)[:x.shape[0]])


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        form = "blocks" if case["form"] == "blocks" else "rows"
        v, e = _quantize(s["x"], case["q"], form)
        out = {"q": v, "scale": _scales(e, case["scale"])}
        if case["form"] != "rows":
            v, e = _quantize(s["x"].t(), case["q"], form)
            out |= {"t_q": v, "t_scale": _scales(e, case["scale"])}
        return out
    if kind == "gemm":
        return (_values(s["a"]) @ _values(s["b"]).t()).to(TYPES[case["out"]])
    if kind == "linear":
        w = _rounded(s["w"], "e4m3", "blocks")
        return {"y": (_rounded(s["x"], "e4m3") @ w.t()).bfloat16(), "dx": (_rounded(s["dy"], "e5m2") @ w).bfloat16(),
                "dw": _rounded(s["dy"].t(), "e5m2") @ _rounded(s["x"].t(), "e4m3").t()}
    if kind == "experts":
        a, w = _values(s["a"]), _values(s["w"])
        parts = [x @ y.t() for x, y in zip(a[:sum(s["counts"])].split(s["counts"]), w)]
        return torch.cat(parts + [a.new_zeros((a.shape[0] - sum(s["counts"]), case["n"]))]).to(TYPES[case["out"]])
    if kind == "experts_grad":
        wt, live = _values(s["wt"]), sum(s["counts"])
        d = _rounded(s["dys"][:live], "e5m2")
        dx = [x @ y.t() for x, y in zip(d.split(s["counts"]), wt)]
        dw = [_rounded(y.t(), "e5m2") @ _rounded(x.t(), "e4m3").t() if x.shape[0] else d.new_zeros((case["n"], case["k"]))
              for y, x in zip(s["dys"][:live].split(s["counts"]), s["xs"][:live].split(s["counts"]))]
        return {"dx": torch.cat(dx + [d.new_zeros((s["xs"].shape[0] - live, case["k"]))]).bfloat16(), "dw": torch.stack(dw)}
    if kind == "layer":                    # every token through every expert: a few tokens, each weight is read once anyway
        w = _values(s["w"])
        every = (_rounded(s["x"], "e4m3") @ w.view(-1, case["k"]).t()).view(case["tokens"], case["experts"], case["n"])
        chosen = every.gather(1, s["ids"].clamp(min=0).unsqueeze(2).expand(-1, -1, case["n"]))
        return (chosen * (s["weights"] * (s["ids"] >= 0)).unsqueeze(2)).sum(1).bfloat16()
    if kind == "dispatch":
        offsets, order, place = _sort(s["ids"], case["experts"])
        xs = s["x"][order.clamp(min=0) // case["topk"]] * (order >= 0).unsqueeze(1)
        out = {"offsets": offsets, "order": order, "place": place, "xs": xs}
        if case["grad"]:
            out["dx"] = (s["dxs"][place.clamp(min=0)].float() * (place >= 0).unsqueeze(2)).sum(1).to(s["x"].dtype)
        return out
    place, dtype = s["place"], s["ys"].dtype
    at, live = place.clamp(min=0), place >= 0
    chosen = s["ys"][at].float() * live.unsqueeze(2)
    out = {"y": (chosen * s["weights"].unsqueeze(2)).sum(1).to(dtype)}
    if case["grad"]:
        order = s["order"]
        by = order.clamp(min=0)
        dy = s["dy"].float()
        out["dys"] = (dy[by // case["topk"]] * (s["weights"].reshape(-1)[by] * (order >= 0)).unsqueeze(1)).to(dtype)
        out["dw"] = (chosen * dy.unsqueeze(1)).sum(2)
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    sc = 1 if case.get("scale") == "e8m0" else 4
    blocks = lambda n: -(-n // BLOCK)  # noqa: E731
    rows_of = lambda r, c: r * (c + sc * blocks(c))  # noqa: E731   8-bit matrix with a scale per row and block
    tile_of = lambda r, c: r * c + sc * blocks(r) * blocks(c)  # noqa: E731
    if kind == "quantize":
        r, c = case["rows"], case["cols"]
        each = tile_of if case["form"] == "blocks" else rows_of
        return {"bytes": r * c * size[case["x"]] + each(r, c) + (each(c, r) if case["form"] != "rows" else 0), "flops": 2 * r * c}
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": rows_of(m, k) + (rows_of if case["form"] == "rows" else tile_of)(n, k) + m * n * size[case["out"]], "flops": 2 * m * n * k}
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * (2 * m * k + 2 * m * n + n * k) + 4 * n * k, "flops": 6 * m * n * k}
    slots = case["tokens"] * case["topk"]
    used = min(case["experts"], slots)              # experts whose weights are read, at most
    if kind == "experts":
        n, k = case["n"], case["k"]
        return {"bytes": rows_of(slots, k) + used * tile_of(n, k) + slots * n * size[case["out"]], "flops": 2 * slots * n * k}
    if kind == "experts_grad":
        n, k = case["n"], case["k"]
        return {"bytes": slots * (2 * n + 2 * k + 2 * k) + used * tile_of(k, n) + case["experts"] * n * k * 4, "flops": 4 * slots * n * k}
    if kind == "layer":
        n, k = case["n"], case["k"]
        return {"bytes": slots * (8 + 4) + case["tokens"] * 2 * (n + k) + used * tile_of(n, k), "flops": 2 * slots * n * k}
    row = case["cols"] * size[case["x"]]
    if kind == "dispatch":
        b = slots * (8 + 4 + 4) + (case["tokens"] + slots) * row
        return {"bytes": b + ((slots + case["tokens"]) * row if case["grad"] else 0), "flops": slots * case["cols"] if case["grad"] else 0}
    b = slots * (4 + 4) + (slots + case["tokens"]) * row
    return {"bytes": b + ((case["tokens"] + slots) * row + slots * 4 if case["grad"] else 0), "flops": (2 + 3 * case["grad"]) * slots * case["cols"]}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _two(e):
    """2^e in 64 bits for whole e."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_blocks(x, q, high):
    """(values on the 8-bit grid times their scale, exponents) by the definition, in 64 bits: `high`: rows of a block."""
    x = x.double()
    rows, cols = x.shape
    out, exps = torch.zeros_like(x), torch.zeros((-(-rows // high), -(-cols // BLOCK)), dtype=torch.float64, device=x.device)
    mant, low = (3, -6) if q == "e4m3" else (2, -14)
    for c in range(0, cols, BLOCK):
        part = x[:, c:c + BLOCK].abs().amax(1)
        if high > 1:
            part = torch.nn.functional.pad(part, (0, -rows % high)).view(-1, high).amax(1)
        e = torch.where(part > 0, torch.ceil(torch.log2(torch.where(part > 0, part, TOP[q]) / TOP[q])), 0.0)
        e = torch.where(part > TOP[q] * _two(e), e + 1, torch.where((part > 0) & (part <= TOP[q] * _two(e - 1)), e - 1, e)).clamp(-126, 127)
        exps[:, c // BLOCK] = e
        e = e.repeat_interleave(high)[:rows].unsqueeze(1)
        v = x[:, c:c + BLOCK] * _two(-e)
        step = _two((torch.frexp(v).exponent - 1).clamp(min=low).double() - mant)
        out[:, c:c + BLOCK] = torch.round(v / step) * step
    return out, exps


def _exact_rounded(x, q, high=1):
    v, e = _exact_blocks(x, q, high)
    return v * _two(e).repeat_interleave(BLOCK, 1)[:, :x.shape[1]].repeat_interleave(high, 0)[:x.shape[0]]


def _exact_values(m):
    data = m["data"][..., :m["cols"]].double()
    s = m["scale"].double()
    if m["scale"].dtype == torch.uint8:
        s = _two(s - 127)
    cols = torch.arange(m["cols"], device=data.device) // BLOCK
    rows = torch.arange(data.shape[-2], device=data.device) // m["rows_per_scale"]
    return data * s[..., rows, :][..., cols]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        high = BLOCK if case["form"] == "blocks" else 1
        v, e = _exact_blocks(s["x"], case["q"], high)
        out = {"q": v, "scale": None if case["scale"] == "e8m0" else _two(e)}
        if case["form"] != "rows":
            v, e = _exact_blocks(s["x"].t(), case["q"], high)
            out |= {"t_q": v, "t_scale": None if case["scale"] == "e8m0" else _two(e)}
        return out
    if kind == "gemm":
        return _exact_values(s["a"]) @ _exact_values(s["b"]).t()
    if kind == "linear":
        w = _exact_rounded(s["w"], "e4m3", BLOCK)
        return {"y": _exact_rounded(s["x"], "e4m3") @ w.t(), "dx": _exact_rounded(s["dy"], "e5m2") @ w,
                "dw": _exact_rounded(s["dy"].t(), "e5m2") @ _exact_rounded(s["x"].t(), "e4m3").t()}
    if kind in ("experts", "experts_grad"):
        w = _exact_values(s["w"] if kind == "experts" else s["wt"])
        a = _exact_values(s["a"]) if kind == "experts" else _exact_rounded(s["dys"], "e5m2")
        y = a.new_zeros((a.shape[0], w.shape[1]))
        dw = None if kind == "experts" else a.new_zeros((case["experts"], case["n"], case["k"]))
        at = 0
        for e, count in enumerate(s["counts"]):
            rows = slice(at, at + count)
            at += count
            if not count:
                continue
            y[rows] = a[rows] @ w[e].t()
            if dw is not None:
                dw[e] = _exact_rounded(s["dys"][rows].t(), "e5m2") @ _exact_rounded(s["xs"][rows].t(), "e4m3").t()
        return y if dw is None else {"dx": y, "dw": dw}
    if kind == "layer":
        x, w = _exact_rounded(s["x"], "e4m3"), _exact_values(s["w"])
        y = x.new_zeros((case["tokens"], case["n"]))
        for t in range(case["tokens"]):
            for p, e in zip(s["weights"][t].tolist(), s["ids"][t].tolist()):
                if e >= 0:
                    y[t] += p * (w[e] @ x[t])
        return y
    rows = s["ids" if kind == "dispatch" else "place"].shape[0]
    token = torch.arange(rows, device="cuda")
    if kind == "dispatch":
        _, order, place = _sort(s["ids"], case["experts"])
        out = {"offsets": None, "order": None, "place": None, "xs": s["x"].double()[order.clamp(min=0) // case["topk"]] * (order >= 0).unsqueeze(1)}
        if case["grad"]:
            dx = torch.zeros((rows, case["cols"]), dtype=torch.float64, device="cuda")
            for j in range(case["topk"]):
                ok = place[:, j] >= 0
                dx.index_add_(0, token[ok], s["dxs"].double()[place[ok, j]])
            out["dx"] = dx
        return out
    y, ys = torch.zeros((rows, case["cols"]), dtype=torch.float64, device="cuda"), s["ys"].double()
    dys, dw = torch.zeros_like(ys), torch.zeros(s["place"].shape, dtype=torch.float64, device="cuda")
    for j in range(case["topk"]):
        ok = s["place"][:, j] >= 0
        at, w = s["place"][ok, j].long(), s["weights"][ok, j].double().unsqueeze(1)
        y[ok] += w * ys[at]
        if case["grad"]:
            dys[at] = w * s["dy"][ok].double()
            dw[ok, j] = (ys[at] * s["dy"][ok].double()).sum(1)
    return {"y": y} | ({"dys": dys, "dw": dw} if case["grad"] else {})
