"""Choices sorted by expert, rows gathered and combined, and the gradients, against plain loops and 64-bit sums."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import scaled_reference as ref  # noqa: E402


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def choices(seed, tokens, topk, experts, dropped=0.05):
    r = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, experts, (tokens, topk), generator=r)
    ids[torch.rand((tokens, topk), generator=r) < 0.3] = experts // 2          # a busy expert
    ids[torch.rand((tokens, topk), generator=r) < dropped] = -1
    return ids


SIZES = [(1, 1, 1), (1, 8, 8), (3, 2, 5), (33, 8, 128), (64, 4, 60), (511, 1, 3), (1000, 4, 256), (4096, 1, 64), (1025, 4, 7), (5000, 8, 1024), (300000, 4, 33)]


@pytest.mark.parametrize("tokens,topk,experts", SIZES)
@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
def test_sort(h, tokens, topk, experts, dtype):
    from paper_2511_13778_amd import experts as ex
    ids = choices(tokens + experts, tokens, topk, experts)
    if tokens > 2:
        ids[1, 0] = experts            # no such expert: dropped as well
        ids[2, 0] = -7
    got = ex.sort_tokens(h, ids.to(dtype).cuda(), experts)
    offsets, order, place = ref.sort_choices(ids, experts)
    assert got.offsets.tolist() == offsets and got.order.tolist() == order and got.place.reshape(-1).tolist() == place


def test_sort_all_dropped_and_none(h):
    from paper_2511_13778_amd import experts as ex
    got = ex.sort_tokens(h, torch.full((9, 2), -1, device="cuda"), 4)
    assert got.offsets.tolist() == [0] * 5 and got.order.tolist() == [-1] * 18 and (got.place == -1).all()
    got = ex.sort_tokens(h, torch.empty((0, 2), dtype=torch.int64, device="cuda"), 4)
    assert got.offsets.tolist() == [0] * 5 and got.order.numel() == 0


UNIT = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def near(got, exact, size, terms, dtype):
    """One rounding to dtype, and `terms` roundings of the sum in 32 bits."""
    err = (got.double() - exact).abs()
    bound = UNIT[dtype] * exact.abs() + (terms + 2) * 2.0 ** -24 * size + 2.0 ** -25
    assert (err <= bound).all(), (err / bound).max().item()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,topk,experts,cols", [(1, 1, 1, 1), (5, 2, 4, 7), (33, 8, 128, 2048), (70, 3, 9, 513), (100, 5, 16, 1000), (40, 1, 3, 9000), (9, 64, 70, 136)])
def test_gather_and_combine(h, tokens, topk, experts, cols, dtype):
    from paper_2511_13778_amd import experts as ex
    ids = choices(tokens, tokens, topk, experts, 0.2).cuda()
    routing = ex.sort_tokens(h, ids, experts)
    r = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((tokens, cols), generator=r, device="cuda").to(dtype)
    order, place = routing.order.long(), routing.place.long()
    want = torch.where((order >= 0).unsqueeze(1), x[order.clamp(min=0) // topk], torch.zeros((), dtype=dtype, device="cuda"))
    xs = ex.gather(h, x, routing)
    assert torch.equal(xs, want)
    xs = torch.randn(xs.shape, generator=r, device="cuda").to(dtype)
    xs[order < 0] = float("nan")                     # rows of no choice are not read
    w = torch.randn((tokens, topk), generator=r, device="cuda")
    live = place >= 0
    rows = torch.where(live.unsqueeze(2), xs[place.clamp(min=0)].double(), 0.0)
    for weights, wd in ((w, w.double() * live), (None, live.double())):
        near(ex.combine(h, xs, routing, weights), (rows * wd.unsqueeze(2)).sum(1), (rows * wd.unsqueeze(2)).abs().sum(1), topk, dtype)
    dy = torch.randn((tokens, cols), generator=r, device="cuda").to(dtype)
    dxs, dw = ex.combine_backward(h, dy, xs, routing, w)
    exact = torch.where((order >= 0).unsqueeze(1), dy.double()[order.clamp(min=0) // topk] * w.double().reshape(-1)[order.clamp(min=0)].unsqueeze(1), 0.0)
    near(dxs, exact, exact.abs(), 1, dtype)
    prod = rows * dy.double().unsqueeze(1)
    near(dw, prod.sum(2), prod.abs().sum(2), cols, torch.float32)
    assert not dxs[order < 0].any() and not dw[~live].any()


def test_gradients_by_differences(h):
    # y is linear in the rows and in the weights, so differences of float32 outputs are exact up to rounding
    from paper_2511_13778_amd import experts as ex
    ids = choices(1, 12, 3, 5, 0.2).cuda()
    routing = ex.sort_tokens(h, ids, 5)
    r = torch.Generator(device="cuda").manual_seed(3)
    xs, w, dy = (torch.randn(s, generator=r, device="cuda") for s in ((36, 40), (12, 3), (12, 40)))
    x = torch.randn((12, 40), generator=r, device="cuda")
    dxs, dw = ex.combine_backward(h, dy, xs, routing, w)
    dx = ex.combine(h, dxs, routing)                       # gradient of gather
    loss = lambda xs, w: (ex.combine(h, xs, routing, w).double() * dy.double()).sum().item()  # noqa: E731
    for t, grad, f in ((xs, dxs, lambda v: loss(v, w)), (w, dw, lambda v: loss(xs, v)),
                       (x, dx, lambda v: (ex.gather(h, v, routing).double() * dxs.double()).sum().item())):
        d = torch.randn(t.shape, generator=r, device="cuda")
        want = (grad.double() * d.double()).sum().item()
        got = (f(t + d) - f(t - d)) / 2
        # every output has a few roundings of 2^-24 of terms of order ten, 480 to 1440 of them
        assert abs(got - want) < 2e-3, (got, want)


def test_views(h):
    from paper_2511_13778_amd import experts as ex
    ids = choices(2, 50, 2, 6).cuda()
    routing = ex.sort_tokens(h, ids, 6)
    for dtype, first, cols in ((torch.bfloat16, 3, 101), (torch.float32, 1, 64), (torch.float16, 8, 200)):
        whole = torch.randn((50, 300), device="cuda").to(dtype)
        x = whole[:, first:first + cols]
        xs = ex.gather(h, x, routing)
        assert torch.equal(xs, ex.gather(h, x.contiguous(), routing))
        out = torch.zeros((50, 300), dtype=dtype, device="cuda")
        ex.combine(h, xs, routing, out=out[:, first:first + cols])
        assert torch.equal(out[:, first:first + cols], ex.combine(h, xs, routing))
        out[:, first:first + cols] = 0
        assert not out.any()


def test_quantize_through_the_routing(h):
    from paper_2511_13778_amd import experts as ex, scaled
    ids = choices(2, 70, 3, 6, 0.2).cuda()
    routing = ex.sort_tokens(h, ids, 6)
    x = torch.randn((70, 300), device="cuda").bfloat16()
    xs = ex.gather(h, x, routing)
    for which in ("rows", "columns"):
        a = scaled.quantize(h, x, routing=routing, which=which)
        b = scaled.quantize(h, xs, which=which)
        assert torch.equal(a.values().view(torch.uint8), b.values().view(torch.uint8)) and torch.equal(a.scales(), b.scales())


def test_refusals(h):
    from paper_2511_13778_amd import experts as ex, ozdgemm as g
    ids = torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    for experts in (0, 1025):
        with pytest.raises(g.OzError) as e:
            ex.sort_tokens(h, ids, experts)
        assert e.value.status == 1
    for bad in (ids.cpu(), ids.float(), ids[0], ids.t()):
        with pytest.raises(ValueError):
            ex.sort_tokens(h, bad, 4)
    routing = ex.sort_tokens(h, ids, 4)
    x = torch.zeros((4, 8), device="cuda")
    with pytest.raises(ValueError):
        ex.gather(h, x[:3], routing)
    with pytest.raises(ValueError):
        ex.combine(h, x, routing)
    with pytest.raises(ValueError):
        ex.combine(h, torch.zeros((8, 8), device="cuda"), routing, torch.zeros((4, 2), device="cuda").double())
    with pytest.raises(ValueError):
        ex.gather(h, x.double(), routing)
    with pytest.raises(ValueError):
        ex.Routing(routing.offsets, routing.order.long(), routing.place, 2)
    with pytest.raises(g.OzError) as e:                    # too many choices per token
        h.call("oz_combine_rows", 0, 1, 65, 8, g.OZ_F32, x.data_ptr(), 8, 4, routing.place.data_ptr(), None, x.data_ptr(), 8)
    assert e.value.status == 1
    with pytest.raises(g.OzError) as e:                    # slots that are not the choices
        h.call("oz_combine_rows_grad", 0, 4, 2, 8, g.OZ_F32, x.data_ptr(), 8, x.data_ptr(), 8, 7, routing.order.data_ptr(),
               routing.place.data_ptr(), None, x.data_ptr(), 8, None)
    assert e.value.status == 1
    big = torch.zeros((9000, 2), dtype=torch.int64, device="cuda")
    with pytest.raises(g.OzError) as e:                    # a workspace is needed
        h.call("oz_sort_tokens", 0, 9000, 2, 4, big.data_ptr(), 8, routing.offsets.data_ptr(), big.data_ptr(), big.data_ptr(), None, 0)
    assert e.value.status == 2
    torch.cuda.synchronize()
