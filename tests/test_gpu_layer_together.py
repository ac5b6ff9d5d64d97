"""The router's choice, the experts' products with 4-bit weights and orthogonal updates as a layer uses them, one after the other, on other streams, in graphs and
where offsets pass 32 bits."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
from test_gpu_orthogonal import QUINTIC, gradient, off  # noqa: E402
from test_gpu_packed import check_product, weights  # noqa: E402

F = 2.0 ** -24


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def test_routed_products_and_the_routers_gradient(h):
    """y = sum_j w_j W_e x and its gradient with that of 0.3 * loss down to the scores, in float32, against torch's in 64 bits."""
    from paper_2511_13778_amd import experts as ex, packed
    r = torch.Generator(device="cuda").manual_seed(1)
    tokens, width, out, n, topk = 150, 200, 90, 12, 3
    x, dy = (torch.randn(s, generator=r, device="cuda") for s in ((tokens, width), (tokens, out)))
    scores = torch.randn((tokens, n), generator=r, device="cuda")
    scores[:, 5] = float("-inf")                               # an expert that nobody gets
    live = torch.rand((tokens,), generator=r, device="cuda") < 0.9
    w = packed.quantize(h, torch.randn((n, out, width), generator=r, device="cuda") * width ** -0.5, group=32, zeros=True)

    c = ex.choose(h, scores, topk, live=live)
    routing = ex.sort_tokens(h, c.ids, n)
    ys = packed.gemm_grouped(h, ex.gather(h, x, routing), w, routing.offsets)
    y = ex.combine(h, ys, routing, c.weights)
    dys, dw = ex.combine_backward(h, dy, ys, routing, c.weights)
    d = ex.choose_backward(h, scores, c, dw, 0.3)

    s = scores.double().requires_grad_()
    p = s.softmax(1) * live[:, None]
    best = s.detach().topk(topk, dim=1).indices
    assert torch.equal(torch.where(live[:, None], best, -1), c.ids.long())
    chosen = p.gather(1, best)
    share = chosen / chosen.sum(1, keepdim=True).clamp(min=1e-300)
    every = torch.stack([x.double() @ packed.unpack(h, w, torch.float32)[e].double().T for e in range(n)], 1)         # tokens x experts x out
    mine = every.gather(1, best[..., None].expand(-1, -1, out))
    ey = (share[..., None] * mine).sum(1)
    f = torch.bincount(c.ids[c.ids >= 0].long(), minlength=n).double() / (topk * live.sum())
    loss = n * (f * p.sum(0)).sum() / live.sum()
    ((ey * dy.double()).sum() + 0.3 * loss).backward()

    # an element of ys is off by (width + 8) steps of what is added (and the unpacked weights by half a step); weights and their gradient as where they are
    # tested alone: here scores lie within 12 of each other
    rel = (2 * 12 + 48) * F
    size = torch.stack([x.double().abs() @ packed.unpack(h, w, torch.float32)[e].double().abs().T for e in range(n)], 1)
    size = size + torch.stack([x.double().abs() @ (w.scale[e].double().abs().T.repeat_interleave(32, 1)[:, :width] * 16).T for e in range(n)], 1)   # code and zero apart
    bad = (width + 9) * 2 * F * size.gather(1, best[..., None].expand(-1, -1, out))
    assert ((y.double() - ey.detach()).abs() <= (share[..., None] * (bad + (rel + 4 * F) * mine.abs())).sum(1).detach() + 1e-30).all()
    off_dw = (dy.double().abs()[:, None] * (bad + (out + 8) * 2 * F * mine.abs())).sum(2)
    exact_dw = (dy.double()[:, None] * mine).sum(2)
    assert ((dw.double() - exact_dw).abs() <= off_dw)[live].all()
    ids, pd, sd = c.ids.long(), p.detach(), share.detach() * live[:, None]
    _, sizes = ref.choose_grad(ids, sd, pd, f, int(live.sum()), exact_dw, 0.3, True)
    _, passed = ref.choose_grad(ids, sd, pd, f, int(live.sum()), off_dw, None, True)
    assert ((d.double() - s.grad.nan_to_num(0.0)).abs() <= (2 * rel + (topk + 16) * F) * sizes + passed + 1e-30).all()
    assert not d[:, 5].any() and not d[~live].any() and not y[~live].any()


def test_layer_serves_packed_and_moves(h):
    from paper_2511_13778_amd import experts as ex, packed
    r = torch.Generator(device="cuda").manual_seed(2)
    n, width, inner, topk = 5, 130, 260, 2
    w1, w2 = (torch.randn(s, generator=r, device="cuda") * s[-1] ** -0.5 for s in ((n, inner, width), (n, width, inner)))
    layer = ex.ExpertLayer(h, w1, w2)
    with pytest.raises(ValueError, match="pack_weights"):
        layer.serve_packed(torch.zeros((1, width), device="cuda"), torch.zeros((1, 1), dtype=torch.int32, device="cuda"), None)
    layer.pack_weights(group=32)
    for tokens in (1, 40):
        x = torch.randn((tokens, width), generator=r, device="cuda").bfloat16()
        c = ex.choose(h, torch.randn((tokens, n), generator=r, device="cuda"), topk, balance=False)
        y = layer.serve_packed(x, c.ids, c.weights)
        e = c.ids.long()
        u1, u2 = (packed.unpack(h, p).double()[e] for p in (layer.p1, layer.p2))
        hidden = torch.nn.functional.silu(u1 @ x.double()[:, None, :, None])
        exact = ((u2 @ hidden).squeeze(3) * c.weights.double()[..., None]).sum(1)
        # four roundings to bfloat16 on the way, at most 2^-8 each, the first times silu's slope of 1.1 at most
        assert off(y.double(), exact) < 4.1 * 2.0 ** -8
    dw1, dw2 = gradient(r, n, inner, width), gradient(r, n, width, inner)
    before = w1.clone(), w2.clone()
    layer.update(dw1, dw2, 0.5)
    for w, old, d, s in ((w1, before[0], dw1, 2 ** 0.5), (w2, before[1], dw2, 1.0)):
        for i in range(n):
            x = d[i].bfloat16()
            exact = ref.orthogonalize(x, 5, QUINTIC, 1e-7)
            own = off(ref.orthogonalize_in_parts(x, 5, QUINTIC, 1e-7, 1), exact)
            sums = 3 * max(x.shape) ** 0.5 * F * 3.4445 ** 2
            last = 2 * F * (old[i].double().norm() + exact.norm()) / (0.5 * s * exact.norm())       # the difference of the weights in float32
            assert off((old[i] - w[i]).double() / (0.5 * s), exact) <= 1.5 * own + sums + 2.0 ** -8 + last.item()
    # and the 8-bit copies are the moved weights'
    fresh = ex.ExpertLayer(h, w1, w2)
    x = torch.randn((20, width), generator=r, device="cuda").bfloat16()
    c = ex.choose(h, torch.randn((20, n), generator=r, device="cuda"), topk, balance=False)
    assert torch.equal(layer.serve(x, c.ids, c.weights), fresh.serve(x, c.ids, c.weights))


def step_of(h, w, topk, n):
    from paper_2511_13778_amd import experts as ex, orthogonal, packed

    def step(scores, x, dw, m):
        c = ex.choose(h, scores, topk)
        routing = ex.sort_tokens(h, c.ids, n)
        y = ex.combine(h, packed.gemm_grouped(h, ex.gather(h, x, routing), w, routing.offsets), routing, c.weights)
        return y, c.loss, ex.choose_backward(h, scores, c, dw, c.loss), orthogonal.orthogonalize(h, m), packed.unpack(h, packed.quantize(h, m))
    return step


def inputs(r, tokens, n, width, topk):
    return [torch.randn(s, generator=r, device="cuda") for s in ((tokens, n), (tokens, width), (tokens, topk), (96, 70))]


def test_two_graphs_replayed_in_turn(h):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(3)
    tokens, width, n, topk = 70, 96, 8, 2
    step = step_of(h, packed.quantize(h, torch.randn((n, 64, width), generator=r, device="cuda")), topk, n)
    given, made, graphs = [], [], []
    for _ in range(2):
        args = inputs(r, tokens, n, width, topk)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*args)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(*args)
        given.append(args)
        made.append(out)
        graphs.append(graph)
    for turn in range(4):
        for i in (0, 1):
            for a, b in zip(given[i], inputs(r, tokens, n, width, topk)):
                a.copy_(b)
        for i in (turn % 2, 1 - turn % 2):
            graphs[i].replay()
        want = [step(*a) for a in given]                        # eager work between replays
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(made[i], want[i])), (turn, i)


def test_two_streams_at_once(h):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(4)
    tokens, width, n, topk = 3000, 256, 16, 2
    step = step_of(h, packed.quantize(h, torch.randn((n, 200, width), generator=r, device="cuda")), topk, n)
    args = [inputs(r, tokens, n, width, topk) for _ in range(2)]
    want = [step(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, a in zip(streams, args):
            with torch.cuda.stream(s):
                got.append(step(*a))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_offsets_beyond_32_bits(h):
    """Rows that lie 70000 and more elements apart, so that the last begin behind 2^32: the same as the same values close together."""
    from paper_2511_13778_amd import experts as ex, orthogonal, packed
    r = torch.Generator(device="cuda").manual_seed(5)
    rows, ld = 66000, 70000
    assert (rows - 1) * ld > 2 ** 32
    big = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")
    scores = torch.randn((rows, 8), generator=r, device="cuda").bfloat16()
    big[:, 3:11] = scores
    a, b = ex.choose(h, big[:, 3:11], 2), ex.choose(h, scores, 2)
    assert torch.equal(a.ids, b.ids) and torch.equal(a.weights, b.weights) and torch.equal(a.loss, b.loss)
    dw = torch.randn((rows, 2), generator=r, device="cuda")
    assert torch.equal(ex.choose_backward(h, big[:, 3:11], a, dw, 1.0), ex.choose_backward(h, scores, b, dw, 1.0))
    x = torch.randn((rows, 64), generator=r, device="cuda").bfloat16()
    big[:, 100:164] = x
    p, q = packed.quantize(h, big[:, 100:164], group=32), packed.quantize(h, x, group=32)
    assert torch.equal(p.data, q.data) and torch.equal(p.scale, q.scale)
    packed.unpack(h, p, out=big[:, 200:264])
    assert torch.equal(big[:, 200:264], packed.unpack(h, q, torch.bfloat16))
    w = weights(r, 16, 64, 32, False, torch.float16)
    packed.gemm(h, big[:, 100:164], w, out=big[:, 300:316])
    assert torch.equal(big[:, 300:316], packed.gemm(h, x, w))
    m = torch.randn((30000, 16), generator=r, device="cuda").bfloat16()
    wide = big.view(-1)[:30000 * 150000].view(30000, 150000)
    wide[:, 40:56] = m
    orthogonal.orthogonalize(h, wide[:, 40:56], out=wide[:, 80:96])
    assert torch.equal(wide[:, 80:96], orthogonal.orthogonalize(h, m))
    # codes that lie far apart
    far = big.view(torch.uint8).view(-1)[:rows * 139984].view(rows, 139984)
    far[:, 16:48] = q.data
    y = packed.gemm(h, x[:3], packed.Packed(far[:, 16:48], q.scale, cols=64, group=32))
    assert torch.equal(y, packed.gemm(h, x[:3], q))
    packed.quantize(h, x[:1], group=32)
    check_product(y[:, -50:], x[:3], ref.codes_of(q.data[-50:], 64), q.scale[:, -50:], None, 32, "far")


def test_refusals_with_a_status(h):
    from paper_2511_13778_amd import experts as ex, orthogonal, packed
    from paper_2511_13778_amd.ozdgemm import OzError
    with pytest.raises(OzError):
        ex.choose(h, torch.zeros((2, 1025), device="cuda"), 2)
    x = torch.zeros((4, 4), device="cuda")
    for steps in (0, 65):
        with pytest.raises(OzError):
            orthogonal.orthogonalize(h, x, steps=steps)
    with pytest.raises(OzError):
        orthogonal.orthogonalize(h, x, eps=float("nan"))
    with pytest.raises(OzError):
        orthogonal.orthogonalize(h, torch.zeros((1, 32769), device="cuda"))
    assert torch.equal(orthogonal.orthogonalize(h, x), x)


def test_a_closed_handle_is_refused():
    from paper_2511_13778_amd import experts as ex, orthogonal, packed
    from paper_2511_13778_amd import ozdgemm as g
    other = g.Handle(0)
    x = torch.randn((8, 64), device="cuda")
    w = packed.quantize(other, x)
    ex.choose(other, x, 2)
    orthogonal.orthogonalize(other, x)
    torch.cuda.synchronize()
    other.close()
    for call in (lambda: ex.choose(other, x, 2), lambda: ex.choose(other, x[:4], 2), lambda: orthogonal.orthogonalize(other, x), lambda: orthogonal.orthogonalize(other, x[:4]),
                 lambda: packed.quantize(other, x), lambda: packed.gemm(other, x, w)):
        with pytest.raises(g.OzError):
            call()


def test_weights_that_moved_are_not_served_from_old_copies(h):
    from paper_2511_13778_amd import experts as ex
    r = torch.Generator(device="cuda").manual_seed(6)
    n, width, inner, topk = 4, 96, 160, 2
    w1, w2 = (torch.randn(s, generator=r, device="cuda") * s[-1] ** -0.5 for s in ((n, inner, width), (n, width, inner)))
    layer = ex.ExpertLayer(h, w1, w2)
    layer.pack_weights(group=32)
    x = torch.randn((6, width), generator=r, device="cuda").bfloat16()
    c = ex.choose(h, torch.randn((6, n), generator=r, device="cuda"), topk, balance=False)
    layer.serve_packed(x, c.ids, c.weights)
    layer.update(gradient(r, n, inner, width), gradient(r, n, width, inner), 0.5)
    with pytest.raises(ValueError, match="pack_weights"):
        layer.serve_packed(x, c.ids, c.weights)
    layer.pack_weights(group=32)
    fresh = ex.ExpertLayer(h, w1, w2)
    fresh.pack_weights(group=32)
    assert torch.equal(layer.serve_packed(x, c.ids, c.weights), fresh.serve_packed(x, c.ids, c.weights))
    layer.prepare_weights()                   # the same weights: their copies stay
    assert torch.equal(layer.serve_packed(x, c.ids, c.weights), fresh.serve_packed(x, c.ids, c.weights))


def test_update_in_all_of_the_gradients_bits(h):
    # float32 gradients as they are where that is asked for: off by the method's 22-bit operands and the difference of the weights, far below a rounding to bfloat16
    from paper_2511_13778_amd import experts as ex
    r = torch.Generator(device="cuda").manual_seed(7)
    n, width, inner = 3, 60, 100
    w1, w2 = (torch.randn(s, generator=r, device="cuda") * s[-1] ** -0.5 for s in ((n, inner, width), (n, width, inner)))
    layer, before = ex.ExpertLayer(h, w1, w2), (w1.clone(), w2.clone())
    dw1, dw2 = gradient(r, n, inner, width), gradient(r, n, width, inner)
    layer.update(dw1, dw2, 0.5, dtype=torch.float32)
    for w, old, d, s in ((w1, before[0], dw1, (inner / width) ** 0.5), (w2, before[1], dw2, 1.0)):
        for i in range(n):
            exact = ref.orthogonalize(d[i], 5, QUINTIC, 1e-7)
            own = off(ref.orthogonalize_in_parts(d[i], 5, QUINTIC, 1e-7, 2), exact)
            sums = 3 * max(d[i].shape) ** 0.5 * F * 3.4445 ** 2
            last = 3 * F * (old[i].double().norm() + exact.norm()) / (0.5 * s * exact.norm())       # the product with the rate and the difference, in float32
            assert off((old[i] - w[i]).double() / (0.5 * s), exact) <= 1.5 * own + sums + F + last.item() < 2.0 ** -12
