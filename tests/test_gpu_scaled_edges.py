"""Ends of the ranges of sizes and values (rows without columns, scales near the least and the largest, padding of blocks without a scale, limits), what
calls do with the matrices, routings and weights that they are given, and captured calls, through the public calls."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import scaled_reference as ref  # noqa: E402
from test_gpu_scaled import E4M3, E5M2, close, dense, gen  # noqa: E402


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_weights_gradient_of_rows_without_columns(h, dtype):
    # an empty sum for every choice, dropped or not, whatever the memory held before
    from paper_2511_13778_amd import experts as ex, ozdgemm as g
    ids = torch.tensor([[0, 2], [-1, 1], [2, 2]], device="cuda")
    routing = ex.sort_tokens(h, ids, 3)
    w = torch.rand((3, 2), device="cuda")
    xs, dy = torch.empty((6, 0), dtype=dtype, device="cuda"), torch.empty((3, 0), dtype=dtype, device="cuda")
    dw = torch.full((3, 2), float("nan"), device="cuda")
    h.call("oz_combine_rows_grad", 0, 3, 2, 0, {torch.float32: g.OZ_F32, torch.bfloat16: g.OZ_BF16, torch.float16: g.OZ_F16}[dtype], None, 1, None, 1, 6,
           routing.order.data_ptr(), routing.place.data_ptr(), w.data_ptr(), None, 1, dw.data_ptr())
    assert torch.equal(dw, torch.zeros_like(dw))
    dxs, dw = ex.combine_backward(h, dy, xs, routing, w)
    assert dxs.shape == (6, 0) and torch.equal(dw, torch.zeros_like(dw))
    assert ex.combine(h, xs, routing, w).shape == (3, 0) and ex.gather(h, dy, routing).shape == (6, 0)


# exponents of A's and of B's scales in one block of k: each at or near an end of what a byte holds, their products ordinary
PAIRS = [(-127, 127), (127, -127), (0, 0), (-127, 112), (114, -126), (-112, 111), (119, -118), (-3, 2)]


def far_apart(seed, m, n, k, a_type, down=0):
    """A (m x k) and B (n x k) whose E8M0 scales differ a little from row to row and lie far out in most blocks; down: taken off the products."""
    from paper_2511_13778_amd import scaled
    r = gen(seed)
    nb = -(-k // 128)
    parts = []
    for rows, dtype, side in ((m, a_type, 0), (n, E4M3, 1)):
        x = torch.zeros((rows, -(-k // 16) * 16), device="cuda")
        x[:, :k] = torch.randn((rows, k), generator=r, device="cuda") * (ref.TOP[dtype] / 8)
        e = torch.tensor([PAIRS[(b + seed) % len(PAIRS)][side] for b in range(nb)], device="cuda")
        e = (e + torch.randint(-1, 2, (rows, nb), generator=r, device="cuda") - (down if side else 0)).clamp(-127, 127)
        s = torch.full((rows, -(-nb // 4) * 4), 255, dtype=torch.uint8, device="cuda")
        s[:, :nb] = (e + 127).to(torch.uint8)
        parts.append(scaled.Scaled(x.clamp(-ref.TOP[dtype], ref.TOP[dtype]).to(dtype), s, k))
    return parts


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("a_type", [E4M3, E5M2])
@pytest.mark.parametrize("m,n,k", [(1, 40, 1100), (20, 70, 1060), (60, 33, 260), (70, 150, 1100), (75, 121, 2432), (1143, 2782, 640), (1094, 3794, 1410), (3867, 3169, 652)])
def test_scales_at_the_ends_of_a_byte(h, m, n, k, a_type, out):
    # each kernel, whatever the result's type: a product whose two scales make an ordinary factor is an ordinary product
    from paper_2511_13778_amd import scaled
    a, b = far_apart(m + k, m, n, k, a_type)
    da, db = dense(a), dense(b)
    exact, size = da @ db.t(), da.abs() @ db.abs().t()
    got = scaled.gemm(h, a, b, dtype=out)
    close(got, exact, size, k)
    c = torch.ones_like(got)
    scaled.gemm(h, a, b, out=c, accumulate=True)
    close(c, exact + 1, size + 1, k)


def test_scales_at_the_ends_of_a_byte_in_float16(h):
    from paper_2511_13778_amd import scaled
    for m, n, k in ((5, 70, 1100), (130, 257, 1000)):
        a, b = far_apart(m, m, n, k, E4M3, 14)
        a.scale[:, :-(-k // 128)].clamp_(max=113)               # B's are held at -127: within float16's range
        da, db = dense(a), dense(b)
        close(scaled.gemm(h, a, b, dtype=torch.float16), da @ db.t(), da.abs() @ db.abs().t(), k)


def test_one_element_and_its_scales(h):
    # 16 2^125 times 1 2^-125 is 16, in every type; NaN scales stay NaN and zeros stay zero
    from paper_2511_13778_amd import scaled
    for rows in (1, 40, 90):
        for ea, eb, x, want in ((125, -125, 16.0, 16.0), (-125, 125, 16.0, 16.0), (-127, 127, 2.0 ** -9, 2.0 ** -9), (127, -127, 448.0, 448.0), (127, 127, 0.0, 0.0),
                                (-127, -127, 1.0, 0.0), (128, -100, 1.0, float("nan")), (127, -126, 64.0, 128.0)):
            a, b = torch.zeros((rows, 128), device="cuda"), torch.zeros((rows, 128), device="cuda")
            a[:, 77], b[:, 77] = x, 1.0
            sa, sb = (torch.full((rows, 4), e + 127, dtype=torch.uint8, device="cuda") for e in (ea, eb))
            for out in (torch.float32, torch.bfloat16, torch.float16):
                got = scaled.gemm(h, scaled.Scaled(a.to(E4M3), sa), scaled.Scaled(b.to(E4M3), sb), dtype=out)
                assert torch.equal(got.float().nan_to_num(nan=-1.0), torch.full((rows, rows), want, device="cuda").nan_to_num(nan=-1.0)), (rows, ea, eb, out)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_scales_at_the_ends_of_a_byte_in_groups(h, out):
    from paper_2511_13778_amd import scaled
    counts, n, k = [3, 0, 200, 40, 1], 150, 700
    rows = sum(counts)
    offsets = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    a, b = far_apart(2, rows, n * len(counts), k, E4M3)
    da, db = dense(a), dense(b).view(len(counts), n, k)
    got = scaled.gemm_grouped(h, a, scaled.Scaled(b.data.view(len(counts), n, -1), b.scale.view(len(counts), n, -1), k), offsets, dtype=out)
    for e, c in enumerate(counts):
        s = slice(int(offsets[e]), int(offsets[e]) + c)
        if c:
            close(got[s], da[s] @ db[e].t(), da[s].abs() @ db[e].abs().t(), k)
    # contraction in groups: the quantised transposes' scales are set to what is wanted
    y, x = torch.randn((rows, 140), generator=gen(3), device="cuda"), torch.randn((rows, 260), generator=gen(4), device="cuda")
    a, b = (scaled.quantize(h, v, which="columns", offsets=offsets) for v in (y, x))
    for b_ in range(a.scale.shape[1]):
        a.scale[:, b_], b.scale[:, b_] = PAIRS[b_ % len(PAIRS)][0] + 127, PAIRS[b_ % len(PAIRS)][1] + 127
    da, db = dense(a), dense(b)
    got = scaled.gemm_grouped_k(h, a, b, offsets, dtype=out)
    at = 0
    for e, c in enumerate(counts):
        wide = -(-c // 128) * 128
        pa, pb = da[:, at:at + c], db[:, at:at + c]
        if c:
            close(got[e], pa @ pb.t(), pa.abs() @ pb.abs().t(), c)
        at += wide


def plain_scales(seed, rows, k, dtype, block_rows, exponents):
    """A matrix with float32 scales of either sign: block b's are near 2^exponents[b]."""
    from paper_2511_13778_amd import scaled
    r = gen(seed)
    x = torch.zeros((rows, -(-k // 16) * 16), device="cuda")
    x[:, :k] = torch.randn((rows, k), generator=r, device="cuda") * (ref.TOP[dtype] / 8)
    high = -(-rows // block_rows)
    s = torch.rand((high, len(exponents)), generator=r, device="cuda") + 1
    s *= torch.where(torch.rand(s.shape, generator=r, device="cuda") < 0.5, -1.0, 1.0)
    s = (s.double() * ref.power(torch.tensor(exponents, device="cuda"))).float()
    return scaled.Scaled(x.clamp(-ref.TOP[dtype], ref.TOP[dtype]).to(dtype), s, k, block_rows)


@pytest.mark.parametrize("rows_b", [1, 128])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", [(5, 70, 300), (70, 150, 300), (75, 121, 2432), (1143, 2782, 640), (2183, 1893, 1425), (899, 4368, 1543)])
def test_float32_scales_whose_product_leaves_the_range(h, m, n, k, out, rows_b):
    # each kernel: scales that together are no float32, and results that are one
    from paper_2511_13778_amd import scaled
    unit, loss = {torch.bfloat16: (2.0 ** -8, 2.0 ** -14), torch.float32: (2.0 ** -23, (k + 128) * 2.0 ** -24)}[out]
    nb = -(-k // 128)
    # 2^-146 times sums of about 2^19: as precise as any
    low = [-73] * nb
    a, b = plain_scales(m, m, k, E4M3, 1, low), plain_scales(n, n, k, E4M3, rows_b, low)
    da, db = dense(a), dense(b)
    exact, size = da @ db.t(), da.abs() @ db.abs().t()
    got = scaled.gemm(h, a, b, dtype=out)
    assert ((got.double() - exact).abs() <= unit * exact.abs() + loss * size + 2.0 ** -133).all()
    # 2^140 times zeros, and in one place times 2^-18; blocks beside them with ordinary scales
    high = [70 if i % 3 == 1 else -4 for i in range(nb)]
    a, b = plain_scales(m + 1, m, k, E5M2, 1, high), plain_scales(n + 1, n, k, E4M3, rows_b, high)
    for x in (a, b):
        for i in range(1, nb, 3):
            x.data[:, i * 128:(i + 1) * 128] = torch.zeros((), device="cuda").to(x.data.dtype)
    got = scaled.gemm(h, a, b, dtype=out)
    da, db = dense(a), dense(b)
    exact, size = da @ db.t(), da.abs() @ db.abs().t()
    assert ((got.double() - exact).abs() <= unit * exact.abs() + loss * size).all()
    a.data[m - 1, 130], b.data[n - 1, 130] = 2.0 ** -9, 2.0 ** -9
    da, db = dense(a), dense(b)
    got = scaled.gemm(h, a, b, dtype=out)[m - 1, n - 1].item()
    exact = (da[m - 1] * db[n - 1]).sum().item()
    assert 2.0 ** 120 < abs(exact) < 2.0 ** 125 and abs(got - exact) <= (unit + loss) * abs(exact)


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("x_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(200, 300), (3, 5), (129, 131), (1, 250), (1300, 1301)])
def test_padding_of_blocks_without_a_scale(h, rows, cols, x_type, scale):
    # up to the next multiple of 16, and of 128 behind a group, bytes are zero also where an infinity or NaN makes the block NaN
    from paper_2511_13778_amd import scaled
    x = torch.randn((rows, cols), generator=gen(rows), device="cuda").to(x_type)
    x[rows - 1, cols - 1] = float("inf")
    x[0, cols - 1] = float("nan")
    for dtype in (E4M3, E5M2):
        for block_rows in (1, 128):
            a, t = scaled.quantize(h, x, dtype, scale, block_rows, which="both")
            for m in (a, t, scaled.quantize(h, x, dtype, scale, block_rows), scaled.quantize(h, x, dtype, scale, block_rows, which="columns")):
                assert m.values().float().isnan().any()
                assert not m.data[:, m.cols:].view(torch.uint8).any()
    ends = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    t = scaled.quantize(h, x, scale_dtype=scale, which="columns", offsets=ends)
    data, at = t.data.view(torch.uint8), 0
    for n in (rows // 3, rows - rows // 3):
        wide = -(-n // 128) * 128
        assert not data[:, at + n:at + wide].any() and (not n or (data[cols - 1, at:at + n] & 0x7F == 0x7F).any())
        at += wide


def test_attributes_of_a_matrix_are_what_products_read(h):
    from paper_2511_13778_amd import scaled
    r = gen(1)
    x, y, w = (torch.randn(s, generator=r, device="cuda") for s in ((20, 300), (30, 300), (40, 300)))
    for scale in (torch.uint8, torch.float32):
        a, other, b = (scaled.quantize(h, t, scale_dtype=scale) for t in (x, y, w))
        first, second = scaled.gemm(h, a, b, dtype=torch.float32), scaled.gemm(h, other, b, dtype=torch.float32)
        old = a.scale
        a.scale = old + 1 if scale == torch.uint8 else old * 2
        assert torch.equal(scaled.gemm(h, a, b, dtype=torch.float32), 2 * first)
        old.fill_(0)                                             # the tensor that was there before is no longer read
        assert torch.equal(scaled.gemm(h, a, b, dtype=torch.float32), 2 * first)
        for bad in (dict(data=a.data.float()), dict(scale=a.scale[:3]), dict(scale=a.scale.cpu()), dict(data=a.data.t()), dict(cols=1000), dict(block_rows=64)):
            with pytest.raises(ValueError):
                setattr(a, *next(iter(bad.items())))
        assert torch.equal(scaled.gemm(h, a, b, dtype=torch.float32), 2 * first)      # a refusal changes nothing
        a.scale = torch.cat((a.scale, a.scale))                  # more rows than there are, then the matrix that has them
        a.data, a.scale = other.data, other.scale
        assert torch.equal(scaled.gemm(h, a, b, dtype=torch.float32), second)
        # a view with other strides, and fewer columns: what follows in a row is not read
        a.data = torch.cat((other.data, other.data), 1)
        assert torch.equal(scaled.gemm(h, a, b, dtype=torch.float32), second)
        a.cols = b.cols = 128
        part = [scaled.quantize(h, t[:, :128].contiguous(), scale_dtype=scale) for t in (y, w)]
        assert torch.equal(scaled.gemm(h, a, b, dtype=torch.float32), scaled.gemm(h, *part, dtype=torch.float32))
        made = scaled.empty(5, 128, scale_dtype=scale)
        made.data, made.scale = a.data[:5], a.scale[:5]
        made.cols = 128
        assert torch.equal(scaled.gemm(h, made, b, dtype=torch.float32), scaled.gemm(h, *part, dtype=torch.float32)[:5])


def test_routing_of_another_number_of_tokens(h):
    from paper_2511_13778_amd import experts as ex, scaled
    routing = ex.sort_tokens(h, torch.tensor([[0, 1], [1, 0], [2, 1]], device="cuda"), 3)
    x = torch.randn((4, 130), device="cuda")
    for rows in (2, 4, 0):
        for which in ("rows", "columns", "both"):
            with pytest.raises(ValueError):
                scaled.quantize(h, x[:rows], which=which, routing=routing)
    assert scaled.quantize(h, x[:3], routing=routing).rows == 6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_combine_without_weights(h, dtype):
    # the rows' gradient as with weights of one, and none of weights that there are not
    from paper_2511_13778_amd import experts as ex
    ids = torch.randint(-1, 4, (33, 3), generator=gen(2), device="cuda")
    routing = ex.sort_tokens(h, ids, 4)
    dy, xs = torch.randn((33, 70), generator=gen(3), device="cuda").to(dtype), torch.randn((99, 70), generator=gen(4), device="cuda").to(dtype)
    want, _ = ex.combine_backward(h, dy, xs, routing, torch.ones((33, 3), device="cuda"))
    for got, dw in (ex.combine_backward(h, dy, xs, routing), ex.combine_backward(h, dy, xs, routing, None)):
        assert torch.equal(got, want) and dw is None


def test_layer_of_parameters_gives_its_gradients_by_itself(h):
    import warnings
    from paper_2511_13778_amd import experts as ex
    r = gen(6)
    w1, w2 = torch.randn((3, 40, 30), generator=r, device="cuda"), torch.randn((3, 30, 40), generator=r, device="cuda")
    x, dy = (torch.randn((20, 30), generator=r, device="cuda").bfloat16() for _ in range(2))
    ids, p = torch.randint(0, 3, (20, 2), generator=r, device="cuda"), torch.rand((20, 2), generator=r, device="cuda")
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        plain, held = ex.ExpertLayer(h, w1, w2), ex.ExpertLayer(h, torch.nn.Parameter(w1), torch.nn.Parameter(w2))
        results = []
        for layer in (plain, held):
            y, kept = layer.forward(x, ids, p)
            results.append((y, *layer.backward(dy, kept)))
    for a, b in zip(*results):
        assert torch.equal(a, b) and not b.requires_grad


def test_limits_that_the_header_names(h):
    # one step past each; refused on the host, before any address is used
    from paper_2511_13778_amd import ozdgemm as g
    big, some = 1 << 24, torch.zeros(64, dtype=torch.int32, device="cuda")
    at = some.data_ptr()

    def m(ld, scale_ld=4, scale=g.OZ_E8M0):
        return g.oz_scaled_t(at, at, ld, scale_ld, 0, 0, g.OZ_E4M3, scale, 1, 0)

    def quantize(rows, cols, batch=1, ldx=None, groups=None):
        return ("oz_quantize", 0, rows, cols, at, cols if ldx is None else ldx, g.OZ_BF16, batch, 0, None, 1, 1, None if groups is None else at, groups or 0,
                m(-(-cols // 16) * 16, -(-cols // 512) * 4), None)

    def gemm(rows, cols, k=128, ldc=None, a=None):
        return ("oz_scaled_gemm", 0, rows, cols, k, a or m(128), m(128), at, cols if ldc is None else ldc, g.OZ_BF16, 0, None, 0)
    calls = [quantize(1, 1 << 22), quantize(big, 9 * 128), quantize(1, 16, 65536), quantize(1, 16, ldx=(1 << 32) + 1), quantize(1, 16, groups=1025),
             quantize(big + 1, 16), gemm(big, 4096), gemm(64, big), gemm(big + 1, 1), gemm(1, 1, ldc=(1 << 32) + 1), gemm(1, 1, a=m(1 << 23)),
             gemm(1, 1, a=m(128, 1 << 17)),
             ("oz_scaled_gemm_grouped", 0, 1025, at, 1, 1, 1, m(16), m(16), at, 1, g.OZ_BF16),
             ("oz_gather_rows", 0, 1 << 26, 1, 8, g.OZ_BF16, at, 8, at, at, at, 8), ("oz_combine_rows", 0, 1 << 26, 1, 8, g.OZ_BF16, at, 8, 1 << 26, at, None, at, 8),
             ("oz_combine_rows_grad", 0, 1 << 26, 1, 8, g.OZ_BF16, at, 8, at, 8, 1 << 26, at, at, None, at, 8, None),
             ("oz_sort_tokens", 0, 1 << 29, 2, 4, at, 4, at, at, at, None, 0)]
    for name, *args in calls:
        with pytest.raises(g.OzError) as e:
            h.call(name, *args)
        assert e.value.status == 1, (name, args)
    torch.cuda.synchronize()


def test_captured_calls_replay_like_eager_ones(h):
    # a layer served, a cut k with its planes, a sort in two launches and its gradients: replayed with other inputs, eager work in between
    from paper_2511_13778_amd import experts as ex, scaled
    r = gen(9)
    layer = ex.ExpertLayer(h, torch.randn((6, 90, 70), generator=r, device="cuda"), torch.randn((6, 70, 90), generator=r, device="cuda"))
    w = scaled.quantize(h, torch.randn((300, 9000), generator=r, device="cuda"), block_rows=128)

    def fresh():
        return (torch.randn((2500, 70), generator=r, device="cuda").bfloat16(), torch.randint(-1, 6, (2500, 2), generator=r, device="cuda"),
                torch.rand((2500, 2), generator=r, device="cuda"), torch.randn((100, 9000), generator=r, device="cuda").bfloat16())

    def work(x, ids, p, long):
        routing = ex.sort_tokens(h, ids, 6)
        xs = ex.gather(h, x, routing)
        dxs, dp = ex.combine_backward(h, x, xs, routing, p)
        return (layer.serve(x, ids, p), xs, dxs, dp, scaled.gemm(h, scaled.quantize(h, long), w), scaled.gemm(h, scaled.quantize(h, long), w, dtype=torch.float32))
    held = fresh()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        work(*held)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work(*held)
    for _ in range(5):
        now = fresh()
        want = work(*now)
        for to, new in zip(held, now):
            to.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
