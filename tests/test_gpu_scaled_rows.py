"""Rows at any alignment and of any length, calls of many tiles and of many groups, through the quantiser, the products and the routing."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import scaled_reference as ref  # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
FLOATS = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def same(m, src, dtype, block_rows=1):
    """The quantiser's result is exact: one rounding, powers of two."""
    v, e = ref.quantize(src, dtype, block_rows)
    got = m.values().float().double()
    assert torch.equal(got.nan_to_num(nan=1e9), v.nan_to_num(nan=1e9))
    scales = ref.scale_values(m.scales())
    assert torch.equal(scales.isnan(), e == 128) and torch.equal(scales.nan_to_num(nan=0.0), torch.where(e == 128, 0.0, ref.power(e.clamp(max=127))))


@pytest.mark.parametrize("x_type", FLOATS)
@pytest.mark.parametrize("first", [0, 1, 3])
def test_quantize_row_ends(h, first, x_type):
    # every number of columns about one load of eight and one block, rows that start at any element; what lies around is NaN
    from paper_2511_13778_amd import scaled
    for cols in [*range(1, 18), *range(121, 138)]:
        whole = torch.full((21, 150), float("nan"), device="cuda").to(x_type)
        x = whole[:, first:first + cols]
        x.copy_(torch.randn((21, cols), generator=gen(cols), device="cuda"))
        same(scaled.quantize(h, x), x, E4M3)
        for block_rows in (1, 128):
            a, t = scaled.quantize(h, x, E5M2, torch.float32, block_rows, which="both")
            same(a, x, E5M2, block_rows)
            same(t, x.t(), E5M2, block_rows)


@pytest.mark.parametrize("x_type", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [E4M3, E5M2])
def test_quantize_infinities_nan_and_least_numbers_in_16_bits(h, dtype, x_type):
    from paper_2511_13778_amd import scaled
    x = torch.randn((200, 300), generator=gen(1), device="cuda").to(x_type)
    x[3, 5], x[4, 201], x[150, 299] = float("inf"), float("nan"), float("-inf")
    x[70:140, :] = 0
    x[70] = torch.finfo(x_type).smallest_normal / 8          # subnormal
    x[71] = torch.finfo(x_type).max
    x[72] = -torch.finfo(x_type).max
    for block_rows in (1, 128):
        same(scaled.quantize(h, x, dtype, block_rows=block_rows), x, dtype, block_rows)
        a, t = scaled.quantize(h, x, dtype, block_rows=block_rows, which="both")
        same(a, x, dtype, block_rows)
        same(t, x.t(), dtype, block_rows)


@pytest.mark.parametrize("x_type", FLOATS)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_many_tiles(h, block_rows, x_type):
    # more than a thousand tiles in one call, whose kernel has more rows per thread
    from paper_2511_13778_amd import scaled
    x = torch.randn((530, 133, 135), generator=gen(2), device="cuda").to(x_type)
    a, t = scaled.quantize(h, x, block_rows=block_rows, which="both")
    for i in (0, 1, 263, 529):
        one, turned = scaled.quantize(h, x[i], block_rows=block_rows, which="both")
        same(one, x[i], E4M3, block_rows)
        same(turned, x[i].t(), E4M3, block_rows)
        for got, want in ((a, one), (t, turned)):
            assert torch.equal(got.data[i].view(torch.uint8), want.data.view(torch.uint8)) and torch.equal(got.scales()[i], want.scales())
    tall = torch.randn((8300, 2050), generator=gen(3), device="cuda").to(x_type)      # 65 x 17 tiles
    a, t = scaled.quantize(h, tall, E5M2, torch.float32, block_rows, which="both")
    same(a, tall, E5M2, block_rows)
    same(t, tall.t(), E5M2, block_rows)


@pytest.mark.parametrize("groups", [63, 64, 65, 200])
def test_many_groups(h, groups):
    # about the number of lanes, and above; most groups empty or short, some past a tile
    from paper_2511_13778_amd import scaled
    counts = torch.randint(0, 4, (groups,), generator=torch.Generator().manual_seed(groups)).tolist()
    counts[0], counts[groups // 2], counts[groups - 1] = 0, 130, 70
    ends = [0]
    for c in counts:
        ends.append(ends[-1] + c)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    rows, k, n = ends[-1] + 3, 140, 40
    x = torch.randn((rows, k), generator=gen(5), device="cuda").bfloat16()
    w = torch.randn((groups, n, k), generator=gen(6), device="cuda").bfloat16()
    a, b = scaled.quantize(h, x), scaled.quantize(h, w, block_rows=128)
    da = ref.dequantize(a.data, a.scale, k, 1)
    db = ref.dequantize(b.data, b.scale, k, 128)
    exact, size = torch.zeros((rows, n), dtype=torch.float64, device="cuda"), torch.zeros((rows, n), dtype=torch.float64, device="cuda")
    for e in range(groups):
        s = slice(ends[e], ends[e + 1])
        exact[s], size[s] = da[s] @ db[e].t(), da[s].abs() @ db[e].abs().t()
    got = scaled.gemm_grouped(h, a, b, offsets, dtype=torch.float32)
    # sums of k terms in 32 bits, and one rounding per block's scale
    assert ((got.double() - exact).abs() <= (k + 128) * 2.0 ** -24 * size).all()
    y = torch.randn((rows, n), generator=gen(7), device="cuda").bfloat16()
    at, xt = scaled.quantize(h, y, which="columns", offsets=offsets), scaled.quantize(h, x, which="columns", offsets=offsets)
    dw = scaled.gemm_grouped_k(h, at, xt, offsets, dtype=torch.float32)
    for e in range(groups):
        s = slice(ends[e], ends[e + 1])
        if counts[e] == 0:
            assert not dw[e].any()
            continue
        (qy, ey), (qx, ex) = ref.quantize(y[s].t(), E4M3, 1), ref.quantize(x[s].t(), E4M3, 1)
        dy = qy * ref.power(ey).repeat_interleave(128, 1)[:, :counts[e]]
        dx = qx * ref.power(ex).repeat_interleave(128, 1)[:, :counts[e]]
        assert ((dw[e].double() - dy @ dx.t()).abs() <= (counts[e] + 128) * 2.0 ** -24 * (dy.abs() @ dx.abs().t())).all()


@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("m,n", [(3, 50), (70, 131), (300, 389), (1030, 1290)])
def test_products_into_rows_at_any_element(h, m, n, out):
    # the same results, to the bit, as into rows at multiples of 16 bytes; nothing beside them is written
    from paper_2511_13778_amd import scaled
    a = scaled.quantize(h, torch.randn((m, 300), generator=gen(8), device="cuda"))
    b = scaled.quantize(h, torch.randn((n, 300), generator=gen(9), device="cuda"), block_rows=128)
    want = scaled.gemm(h, a, b, dtype=out)
    for first in (1, 2, 5):
        whole = torch.full((m, n + 9), 7.0, device="cuda").to(out)
        view = whole[:, first:first + n]
        scaled.gemm(h, a, b, out=view)
        assert torch.equal(view, want)
        view.fill_(0)
        scaled.gemm(h, a, b, out=view, accumulate=True)
        assert torch.equal(view, want)
        view.fill_(7.0)
        assert (whole == 7.0).all()


@pytest.mark.parametrize("dtype", FLOATS)
def test_routed_rows_at_any_element(h, dtype):
    # rows of every length about a load of 16 bytes, and about what a wave moves, that start at any element
    from paper_2511_13778_amd import experts as ex
    ids = torch.randint(-1, 5, (23, 3), generator=gen(10), device="cuda")
    routing = ex.sort_tokens(h, ids, 5)
    order, place = routing.order.long(), routing.place.long()
    w = torch.randn((23, 3), generator=gen(11), device="cuda")
    for cols in [*range(1, 20), 511, 513, 1023, 1025, 2047, 2051]:
        for first in (0, 1, 5):
            whole = torch.full((23, cols + 8), float("nan"), device="cuda").to(dtype)
            x = whole[:, first:first + cols]
            x.copy_(torch.randn((23, cols), generator=gen(cols), device="cuda"))
            out = torch.full((69, cols + 8), 7.0, device="cuda").to(dtype)
            xs = ex.gather(h, x, routing, out=out[:, first:first + cols])
            assert torch.equal(xs, torch.where((order >= 0).unsqueeze(1), x[order.clamp(min=0) // 3], torch.zeros((), dtype=dtype, device="cuda")))
            assert (out[:, :first] == 7.0).all() and (out[:, first + cols:] == 7.0).all()
            back = torch.full((23, cols + 8), 7.0, device="cuda").to(dtype)
            y = ex.combine(h, xs, routing, w, out=back[:, first:first + cols])
            assert (back[:, :first] == 7.0).all() and (back[:, first + cols:] == 7.0).all()
            assert torch.equal(y, ex.combine(h, xs.contiguous(), routing, w))
            terms = torch.where((place >= 0).unsqueeze(2), x.double().unsqueeze(1) * w.double().unsqueeze(2), 0.0)
            unit = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}[dtype]
            assert ((y.double() - terms.sum(1)).abs() <= unit * terms.sum(1).abs() + 5 * 2.0 ** -24 * terms.abs().sum(1) + 2.0 ** -25).all()
            dxs, dw = ex.combine_backward(h, x, xs, routing, w)
            again, dw2 = ex.combine_backward(h, x.contiguous(), xs.contiguous(), routing, w)
            assert torch.equal(dxs, again) and torch.equal(dw, dw2)
