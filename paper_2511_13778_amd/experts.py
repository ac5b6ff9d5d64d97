"""The router's choice, rows sorted by expert and back, on torch tensors: what stands before and behind the experts' products
(scaled.gemm_grouped, packed.gemm_grouped).

A layer whose tokens go to their chosen experts:

    choice = choose(h, scores, topk)                          # scores: tokens x experts; its balance loss is choice.loss
    routing = sort_tokens(h, choice.ids, experts)             # ids: tokens x topk, -1 where a choice is dropped
    a = scaled.quantize(h, x, routing=routing)                # each choice's row, sorted by expert, in 8-bit floats
    ys = scaled.gemm_grouped(h, a, w, routing.offsets)
    y = combine(h, ys, routing, choice.weights)

Gradients are calls too (combine without weights is gather's, combine_backward is combine's, choose_backward is choose's): results carry no history for torch's autograd.
Everything is enqueued on the current stream of the handle's GPU, where all tensors are; nothing is read back, so no call waits for the GPU.
"""
from __future__ import annotations

import torch

from . import orthogonal
from . import ozdgemm as g
from . import packed
from . import scaled
from .scaled import check_device, check_ints, check_matrix, float_type, stream_of


class Routing:
    """Where each choice went: offsets (experts + 1: an expert's slots), order (slot -> choice, -1 behind the last), place (choice -> slot, -1
    if dropped), all int32; choice t * topk + j is token t's j-th."""

    __slots__ = ("offsets", "order", "place", "topk", "tokens")

    def __init__(self, offsets, order, place, topk):
        check_ints(offsets, "offsets")
        check_ints(order, "order")
        check_ints(place, "place", order.numel())
        if offsets.device != order.device or place.device != order.device:
            raise ValueError("offsets, order and place on one GPU, not %s, %s and %s" % (offsets.device, order.device, place.device))
        if topk < 1 or order.numel() % topk:
            raise ValueError("%d choices are not %s per token" % (order.numel(), topk))
        self.offsets, self.order, self.place, self.topk, self.tokens = offsets, order, place, topk, order.numel() // topk


def sort_tokens(h: g.Handle, ids, experts: int) -> Routing:
    """Sorts the choices ids (tokens x topk, int64 or int32) by expert, each expert's in their own order."""
    if not ids.is_cuda or ids.dim() != 2 or ids.shape[1] < 1 or ids.dtype not in (torch.int64, torch.int32) or not ids.is_contiguous():
        raise ValueError("ids: contiguous tokens x topk, int64 or int32, on the GPU")
    check_device(h, ids)
    tokens, topk = ids.shape
    n = tokens * topk
    need = h.sort_tokens_workspace_bytes(tokens, topk, experts)
    # one allocation for the three tables and the workspace
    at = [0, experts + 1, experts + 1 + n]
    ws_at = -(-(at[2] + n) // 64) * 64
    all_ = torch.empty(ws_at + (need + 3) // 4, dtype=torch.int32, device=ids.device)
    base = all_.data_ptr()
    h.call("oz_sort_tokens", stream_of(ids), tokens, topk, experts, ids.data_ptr(), ids.element_size(), base, base + 4 * at[1], base + 4 * at[2],
           base + 4 * ws_at if need else None, need)
    r = Routing.__new__(Routing)            # right by construction
    r.offsets, r.order, place, _ = torch.split_with_sizes(all_, (experts + 1, n, n, all_.numel() - at[2] - n))
    r.place, r.topk, r.tokens = place.view(tokens, topk), topk, tokens
    return r


def gather(h: g.Handle, x, routing: Routing, out=None):
    """Each choice's row of x (tokens x cols), sorted by expert; zeros behind the last."""
    ldx = check_matrix(x, "x")
    check_device(h, x, routing.order, out)
    if x.shape[0] != routing.tokens:
        raise ValueError("x has %d rows, the routing %d tokens" % (x.shape[0], routing.tokens))
    slots = routing.order.numel()
    y = torch.empty((slots, x.shape[1]), dtype=x.dtype, device=x.device) if out is None else out
    ldy = check_matrix(y, "out")
    if tuple(y.shape) != (slots, x.shape[1]) or y.dtype != x.dtype:
        raise ValueError("out: %d x %d of %s" % (slots, x.shape[1], x.dtype))
    h.call("oz_gather_rows", stream_of(x), routing.tokens, routing.topk, x.shape[1], float_type(x.dtype), x.data_ptr(), ldx,
           routing.order.data_ptr(), routing.place.data_ptr(), y.data_ptr(), ldy)
    return y


def _weights(weights, routing):
    if weights is None:
        return None
    if not weights.is_cuda or weights.dtype != torch.float32 or not weights.is_contiguous() or weights.numel() != routing.order.numel():
        raise ValueError("weights: contiguous float32, one per choice, on the GPU")
    return weights.data_ptr()


def combine(h: g.Handle, xs, routing: Routing, weights=None, out=None):
    """Sum over each token's choices of weight * the choice's row of xs, in 32 bits, rounded once.  Without weights: the gradient of gather."""
    ldx = check_matrix(xs, "xs")
    check_device(h, xs, routing.order, weights, out)
    if xs.shape[0] != routing.order.numel():
        raise ValueError("xs has %d rows, the routing %d slots" % (xs.shape[0], routing.order.numel()))
    y = torch.empty((routing.tokens, xs.shape[1]), dtype=xs.dtype, device=xs.device) if out is None else out
    ldy = check_matrix(y, "out")
    if tuple(y.shape) != (routing.tokens, xs.shape[1]) or y.dtype != xs.dtype:
        raise ValueError("out: %d x %d of %s" % (routing.tokens, xs.shape[1], xs.dtype))
    h.call("oz_combine_rows", stream_of(xs), routing.tokens, routing.topk, xs.shape[1], float_type(xs.dtype), xs.data_ptr(), ldx, xs.shape[0],
           routing.place.data_ptr(), _weights(weights, routing), y.data_ptr(), ldy)
    return y


def combine_backward(h: g.Handle, dy, xs, routing: Routing, weights=None):
    """Gradients of combine for dy (tokens x cols): (of xs, of the weights or None where there are none)."""
    lddy, ldx = check_matrix(dy, "dy"), check_matrix(xs, "xs")
    check_device(h, dy, xs, routing.order, weights)
    if xs.shape != (routing.order.numel(), dy.shape[1]) or dy.shape[0] != routing.tokens or dy.dtype != xs.dtype:
        raise ValueError("dy %s %s and xs %s %s do not belong to this routing" % (tuple(dy.shape), dy.dtype, tuple(xs.shape), xs.dtype))
    dxs = torch.empty(xs.shape, dtype=xs.dtype, device=xs.device)
    dw = None if weights is None else torch.empty(weights.shape, dtype=torch.float32, device=xs.device)
    h.call("oz_combine_rows_grad", stream_of(dy), routing.tokens, routing.topk, dy.shape[1], float_type(dy.dtype), dy.data_ptr(), lddy,
           xs.data_ptr(), ldx, xs.shape[0], routing.order.data_ptr(), routing.place.data_ptr(), _weights(weights, routing), dxs.data_ptr(),
           max(dxs.shape[1], 1), None if dw is None else dw.data_ptr())
    return dxs, dw


class Choice:
    """What choose found: ids (tokens x topk, int32, -1 where there is none), weights (float32), and, if asked for, counts (how often each
    expert was chosen, int32), counted (one int32: tokens that have an expert), shares (their mean probability of each expert, float32) and
    loss (float32, one value).  counts may be added up over several GPUs before choose_backward, in place or set to others."""

    # _made: ids and weights as choose made them, which need no second look
    __slots__ = ("ids", "weights", "live", "normalize", "_parts", "_table", "_made", "_set")

    def __init__(self, ids, weights, counts=None, counted=None, shares=None, loss=None, live=None, normalize=True):
        self.ids, self.weights, self.live, self.normalize = ids, weights, live, normalize
        self._parts, self._table, self._made, self._set = [counts, counted, shares, loss], None, None, False

    # choose leaves the four results of the whole batch in one table of float32, (2 experts + 2 values): cut out when they are asked for
    def _part(at, cut):
        def get(self):
            have = self._parts[at]
            if have is None and self._table is not None:
                have = self._parts[at] = cut(*self._table)
            return have

        def put(self, value):
            self._parts[at], self._set = value, True
        return property(get, put)

    counts = _part(0, lambda table, n: table.narrow(0, 0, n).view(torch.int32))
    counted = _part(1, lambda table, n: table.narrow(0, n, 1).view(torch.int32))
    shares = _part(2, lambda table, n: table.narrow(0, n + 1, n))
    loss = _part(3, lambda table, n: table.select(0, 2 * n + 1))
    del _part


def _live(live, tokens):
    if live is None:
        return None
    if not live.is_cuda or live.dtype not in (torch.bool, torch.uint8) or not live.is_contiguous() or live.numel() != tokens:
        raise ValueError("live: contiguous bool, one per token, on the GPU")
    return live.data_ptr()


def choose(h: g.Handle, scores, topk: int, live=None, normalize=True, balance=True) -> Choice:
    """Each token's topk experts by falling score (ties: the lowest), scores tokens x experts (-inf: not to be had), with their weights: the softmax
    over all experts, of which the chosen ones' share of their sum is taken if normalize.  Tokens where live is False are padding.
    balance: also counts, shares and the loss experts * sum_e f_e P_e (f_e an expert's share of the choices, P_e its mean probability)."""
    ld = check_matrix(scores, "scores")
    check_device(h, scores, live)
    tokens, experts = scores.shape
    if not 1 <= topk <= min(experts, 64):
        raise ValueError("topk 1 .. 64 of %d experts, not %s" % (experts, topk))
    c = Choice(scores.new_empty((tokens, topk), dtype=torch.int32), scores.new_empty((tokens, topk), dtype=torch.float32), live=live, normalize=bool(normalize))
    c._made = c.ids, c.weights
    more = (None, None, None, None, None, 0)
    if balance:
        # one allocation for the four results of the batch, which a kept loss holds on to, and another for the workspace, which goes back after the call
        need = h.choose_experts_workspace_bytes(tokens, experts)
        table, ws = scores.new_empty(2 * experts + 2, dtype=torch.float32), scores.new_empty(need, dtype=torch.uint8)
        c._table = table, experts
        at = table.data_ptr()
        more = (at, at + 4 * experts, at + 4 * experts + 4, at + 8 * experts + 4, ws.data_ptr(), need)
    h.call("oz_choose_experts", stream_of(scores), tokens, experts, topk, scores.data_ptr(), ld, float_type(scores.dtype), _live(live, tokens),
           int(c.normalize), c.ids.data_ptr(), c.weights.data_ptr(), *more)
    return c


def choose_backward(h: g.Handle, scores, choice: Choice, dweights=None, dloss=None):
    """The gradient of choose's scores, for dweights (tokens x topk, float32) and dloss (a number, or one float32 on the GPU); either may be None."""
    ld = check_matrix(scores, "scores")
    ids, weights, live = choice.ids, choice.weights, choice.live
    check_device(h, scores, ids, live, dweights)
    tokens, experts = scores.shape
    made = choice._made
    if made is None or made[0] is not ids or made[1] is not weights:
        check_device(h, weights)
        check_ints(ids, "ids")
        if ids.dim() != 2 or weights.shape != ids.shape or weights.dtype != torch.float32 or not weights.is_contiguous():
            raise ValueError("ids and weights: int32 and float32 of the same tokens x topk, not %s and %s" % (tuple(ids.shape), tuple(weights.shape)))
    if ids.shape[0] != tokens:
        raise ValueError("scores %s do not belong to this choice of %s" % (tuple(scores.shape), tuple(ids.shape)))
    if dweights is not None and (dweights.dtype != torch.float32 or dweights.shape != ids.shape or not dweights.is_contiguous()):
        raise ValueError("dweights: contiguous float32 of %s" % (tuple(ids.shape),))
    counts = counted = scalar = None
    factor = 1.0
    if dloss is not None:
        if choice._table is not None and not choice._set:
            table, of = choice._table
            if of != experts or table.device != scores.device:
                raise ValueError("scores of %d experts do not belong to this choice of %d" % (experts, of))
            counts = table.data_ptr()
            counted = counts + 4 * experts
        else:
            counts, counted = choice.counts, choice.counted
            if counts is None or counted is None:
                raise ValueError("a gradient of the loss needs the choice's counts: choose(balance=True)")
            check_device(h, counts, counted)
            counts, counted = check_ints(counts, "counts", experts).data_ptr(), check_ints(counted, "counted", 1).data_ptr()
        if torch.is_tensor(dloss):
            check_device(h, dloss)
            if not dloss.is_cuda or dloss.dtype != torch.float32 or dloss.numel() != 1:
                raise ValueError("dloss: a number, or one float32 on the GPU")
            scalar = dloss.data_ptr()
        else:
            factor = float(dloss)
    d = scores.new_empty((tokens, experts))
    h.call("oz_choose_experts_grad", stream_of(scores), tokens, experts, ids.shape[1], scores.data_ptr(), ld, float_type(scores.dtype),
           _live(live, tokens), int(choice.normalize), ids.data_ptr(), weights.data_ptr(), None if dweights is None else dweights.data_ptr(),
           counts, counted, scalar, factor, d.data_ptr(), max(experts, 1))
    return d


class ExpertLayer:
    """Experts of two linear layers with silu between them, y = sum_j w_j W2_e silu(W1_e x) over a token's choices e: an example of the calls
    above as a training step and a serving step make them.

    w1 (experts x inner x width) and w2 (experts x width x inner) are the caller's, in any float type; prepare_weights() makes their 8-bit
    copies, for the forward products and, transposed, for the input gradients, and is called again when they have changed; pack_weights()
    their 4-bit ones, for serve_packed().  update() moves them.  Only silu and its derivative are torch's.

    The experts' rows between the second product and combine have x's type, as the activations between the products have before they are
    quantised: half the bytes of float32 at the price of one more rounding of each (with bfloat16 2^-9, against the 2^-4 of an element in
    8 bits).  The products alone can be asked for float32 rows, which combine then adds as they are."""

    def __init__(self, h: g.Handle, w1, w2, scale_dtype=torch.uint8):
        if w1.dim() != 3 or w2.shape != (w1.shape[0], w1.shape[2], w1.shape[1]):
            raise ValueError("w1 experts x inner x width and w2 experts x width x inner, not %s and %s" % (tuple(w1.shape), tuple(w2.shape)))
        self.h, self.w1, self.w2, self.scale_dtype, self.experts = h, w1, w2, scale_dtype, w1.shape[0]
        self.p1 = self.p2 = None
        self.prepare_weights()

    def prepare_weights(self):
        self.q1, self.q1t = scaled.quantize(self.h, self.w1.detach(), scale_dtype=self.scale_dtype, block_rows=128, which="both")
        self.q2, self.q2t = scaled.quantize(self.h, self.w2.detach(), scale_dtype=self.scale_dtype, block_rows=128, which="both")

    def serve(self, x, ids, weights):
        """y for tokens x (tokens x width) without anything kept for gradients."""
        h = self.h
        routing = sort_tokens(h, ids, self.experts)
        a = scaled.quantize(h, x, scale_dtype=self.scale_dtype, routing=routing)
        inner = torch.nn.functional.silu(scaled.gemm_grouped(h, a, self.q1, routing.offsets, dtype=x.dtype))
        out = scaled.gemm_grouped(h, scaled.quantize(h, inner, scale_dtype=self.scale_dtype), self.q2, routing.offsets, dtype=x.dtype)
        return combine(h, out, routing, weights)

    def pack_weights(self, group=64, scale_dtype=torch.float16):
        """The 4-bit copies that serve_packed reads, made anew when the weights have changed: a quarter of bfloat16's bytes, for a value that is off by at
        most a fourteenth of its group's largest."""
        self.p1, self.p2 = (packed.quantize(self.h, w.detach(), group=group, scale_dtype=scale_dtype) for w in (self.w1, self.w2))

    def serve_packed(self, x, ids, weights):
        """serve on the 4-bit copies, activations as they are: for few tokens in flight, where the time is the weights'."""
        if self.p1 is None:
            raise ValueError("pack_weights() first")
        h = self.h
        routing = sort_tokens(h, ids, self.experts)
        inner = torch.nn.functional.silu(packed.gemm_grouped(h, gather(h, x, routing), self.p1, routing.offsets))
        return combine(h, packed.gemm_grouped(h, inner, self.p2, routing.offsets), routing, weights)

    @torch.no_grad()
    def update(self, dw1, dw2, rate, dtype=torch.bfloat16):
        """A step of the weights against their gradients (or running means of them) made orthogonal, then prepare_weights(): each expert's matrix moves by
        rate in every direction, by rate * sqrt(out / in) where it makes more values than it takes.  In bfloat16, whose rounding of
        the direction (0.2 %) is far below what Newton-Schulz leaves open, or, in some three times as long, dtype=torch.float32 (10^-6).  The 4-bit
        copies, which are the old weights', are dropped."""
        for w, d in ((self.w1, dw1), (self.w2, dw2)):
            w.sub_(orthogonal.orthogonalize(self.h, d.to(dtype)), alpha=rate * max(1.0, w.shape[1] / max(w.shape[2], 1)) ** 0.5)
        self.p1 = self.p2 = None
        self.prepare_weights()

    def forward(self, x, ids, weights):
        """(y, what backward needs)."""
        h, sc = self.h, self.scale_dtype
        routing = sort_tokens(h, ids, self.experts)
        xs = gather(h, x, routing)
        a, at = scaled.quantize(h, xs, scale_dtype=sc, which="both", offsets=routing.offsets)
        pre = scaled.gemm_grouped(h, a, self.q1, routing.offsets, dtype=x.dtype)
        b, bt = scaled.quantize(h, torch.nn.functional.silu(pre), scale_dtype=sc, which="both", offsets=routing.offsets)
        out = scaled.gemm_grouped(h, b, self.q2, routing.offsets, dtype=x.dtype)
        return combine(h, out, routing, weights), (routing, weights, at, pre, bt, out)

    def backward(self, dy, kept, dw1=None, dw2=None):
        """(dx, dweights, dw1, dw2) of forward; the weights' gradients in float32, added to dw1 and dw2 where they are given."""
        h, sc = self.h, self.scale_dtype
        routing, weights, at, pre, bt, out = kept
        offsets = routing.offsets
        dout, dweights = combine_backward(h, dy, out, routing, weights)
        d, dt = scaled.quantize(h, dout, dtype=torch.float8_e5m2, scale_dtype=sc, which="both", offsets=offsets)
        dw2 = scaled.gemm_grouped_k(h, dt, bt, offsets, out=dw2, accumulate=dw2 is not None)
        dinner = scaled.gemm_grouped(h, d, self.q2t, offsets, dtype=dy.dtype)
        dpre = torch.ops.aten.silu_backward(dinner, pre)
        d, dt = scaled.quantize(h, dpre, dtype=torch.float8_e5m2, scale_dtype=sc, which="both", offsets=offsets)
        dw1 = scaled.gemm_grouped_k(h, dt, at, offsets, out=dw1, accumulate=dw1 is not None)
        dx = combine(h, scaled.gemm_grouped(h, d, self.q1t, offsets, dtype=dy.dtype), routing)
        return dx, dweights, dw1, dw2
