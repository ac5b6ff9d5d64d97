"""Weights in 4 bits: quantised, read back, multiplied, against plain 64-bit forms."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402

FLOATS = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def same(a, b):
    assert a.shape == b.shape and torch.equal(torch.nan_to_num(a, nan=-12345.0), torch.nan_to_num(b, nan=-12345.0))


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (5, 33), (7, 100), (16, 128), (2, 511), (4, 513), (9, 1000), (130, 96)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantize(h, rows, cols, group, zeros):
    from paper_2511_13778_amd import packed
    r = torch.Generator().manual_seed(rows * cols)
    for dtype in FLOATS:
        for scale_dtype in FLOATS:
            w = (torch.randn((rows, cols), generator=r) * torch.randn((rows, 1), generator=r).exp()).to(dtype)
            w[0] = w[0].abs()
            got = packed.quantize(h, w.cuda(), group=group, zeros=zeros, scale_dtype=scale_dtype)
            codes, scale, zero = ref.quantize(w, group, zeros, scale_dtype)
            assert torch.equal(ref.codes_of(got.data.cpu(), cols), codes)
            assert not ref.codes_of(got.data.cpu(), got.data.shape[1] * 2)[:, cols:].any()
            same(got.scale.cpu().double(), scale)
            if zeros:
                same(got.zero.cpu().double(), zero)
            values = ref.values(codes, scale, zero, group)
            for out in FLOATS:
                # one product of 32 bits, and one rounding (exact where the scale has 16 bits)
                err = (packed.unpack(h, got, dtype=out).cpu().double() - values).abs()
                assert (err <= ref.rounded(values, out) + ref.rounded(values, torch.float32)).all()


@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_zeros_and_not_numbers(h, zeros):
    from paper_2511_13778_amd import packed
    w = torch.randn((6, 256))
    w[0, :128] = 0.0
    w[1, 40] = float("nan")
    w[2, 200] = float("inf")
    w[3, 7] = -float("inf")
    w[4] = 3e38
    w[5] = -w[5].abs()
    for scale_dtype in FLOATS:
        got = packed.quantize(h, w.cuda(), zeros=zeros, scale_dtype=scale_dtype)
        codes, scale, zero = ref.quantize(w, 128, zeros, scale_dtype)
        assert torch.equal(ref.codes_of(got.data.cpu(), 256), codes)
        same(got.scale.cpu().double(), scale)
        v = packed.unpack(h, got).cpu()
        assert not v[0, :128].any() and v[1, :128].isnan().all() and v[1, 128:].isfinite().all() and v[2, 128:].isnan().all() and v[3, :128].isnan().all()
        assert v[4].isnan().all() == (scale_dtype == torch.float16)


def test_quantize_batches_and_strides(h):
    from paper_2511_13778_amd import packed
    big = torch.randn((3, 20, 300), device="cuda")
    x = big[:, 3:17, 5:250]
    got = packed.quantize(h, x, group=64, zeros=True)
    for i in range(3):
        one = packed.quantize(h, x[i].contiguous(), group=64, zeros=True)
        assert torch.equal(got.data[i], one.data) and torch.equal(got.scale[i], one.scale) and torch.equal(got.zero[i], one.zero)
    out = torch.full((3, 20, 300), 7.0, device="cuda")
    packed.unpack(h, got, out=out[:, 3:17, 5:250])
    assert torch.equal(out[:, 3:17, 5:250], packed.unpack(h, got))
    out[:, 3:17, 5:250] = 7.0
    assert (out == 7.0).all()                 # nothing beside it is touched


def weights(r, n, k, group, zeros, scale_dtype, lead=()):
    from paper_2511_13778_amd import packed
    data = torch.randint(0, 256, lead + (n, max(-(-k // 32), 1) * 16), generator=r, device="cuda", dtype=torch.uint8)       # codes behind the end are anything
    blocks = -(-k // group)
    scale = torch.randn(lead + (blocks, n), generator=r, device="cuda").to(scale_dtype)
    zero = (torch.rand(lead + (blocks, n), generator=r, device="cuda") * 15).to(scale_dtype) if zeros else None
    return packed.Packed(data, scale, zero, cols=k, group=group)


def check_product(got, x, codes, scale, zero, group, what):
    exact, size = ref.product(x, codes, scale, zero, group)
    k = x.shape[1]
    # every addition of 32 bits off by a step of what is added, scales and zero points four more
    bound = (k + 8) * 2.0 ** -23 * size + ref.rounded(exact, got.dtype)
    if x.dtype == got.dtype == torch.bfloat16:
        # 128 + code is summed, at most 143 in the place of code - 8, and 136 (or 128 + zero point) times the sum of x comes off: additions of a
        # group's up to 128 products in 4 instructions and one fused subtraction, each off by a step of sums of 143 |x|
        at = torch.arange(k, device=x.device) // group
        bound = bound + 10 * 2.0 ** -24 * 143 * (x.double().abs() @ scale.double().abs().T[:, at].T)
    err = (got.double() - exact).abs()
    assert got.shape == exact.shape and (err <= bound).all(), (what, (err / bound).max().item())


SHAPES = [(1, 1, 1), (1, 16, 32), (1, 17, 33), (2, 40, 129), (16, 64, 128), (17, 33, 200), (15, 100, 1000), (33, 50, 95), (64, 31, 257), (65, 48, 640), (130, 20, 2100), (3, 5, 5000)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_gemm(h, m, n, k, group, zeros):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(m + n + k)
    for i, dtype in enumerate(FLOATS):
        w = weights(r, n, k, group, zeros, FLOATS[(i + m) % 3])
        x = torch.randn((m, k), generator=r, device="cuda").to(dtype)
        codes = ref.codes_of(w.data, k)
        for out in {dtype, torch.float32}:
            check_product(packed.gemm(h, x, w, dtype=out), x, codes, w.scale, w.zero, group, (dtype, out))


def test_float32_rows_lose_nothing(h):
    # values that need all 24 bits, and others far from 1: the parts that x is cut into hold all of it
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(5)
    w = weights(r, 16, 32, 32, False, torch.float32)
    w.data.fill_(0x88)
    w.data[:, 0] = 0x89                       # 1 in column 0, nothing elsewhere
    w.scale.fill_(1.0)
    x = torch.randn((10, 32), generator=r, device="cuda") * torch.tensor([1e-30, 1e-20, 1e-3, 1.0, 1e10, 1e20, 1e30, 3e38 / 8, 1.0, 1.0], device="cuda")[:, None]
    y = packed.gemm(h, x, w)
    assert torch.equal(y, x[:, :1].expand(10, 16))


def test_infinities_and_rows_apart(h):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(6)
    for dtype in FLOATS:
        w = weights(r, 40, 300, 64, True, torch.float16)
        x = torch.randn((20, 300), generator=r, device="cuda").to(dtype)
        y = packed.gemm(h, x, w)
        x[3, 299] = float("inf")
        x[7, 0] = float("nan")
        z = packed.gemm(h, x, w)
        rest = [i for i in range(20) if i not in (3, 7)]
        assert torch.equal(y[rest], z[rest]) and not z[3].isfinite().any() and z[7].isnan().all()


@pytest.mark.parametrize("dtype", FLOATS)
def test_strides_and_alignment(h, dtype):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(7)
    m, n, k = 9, 37, 201
    w = weights(r, n + 3, k, 32, True, torch.float16)
    part = packed.Packed(w.data[2:2 + n], w.scale[:, 2:2 + n], w.zero[:, 2:2 + n], cols=k, group=32)
    codes = ref.codes_of(part.data, k)
    for ld, start in ((201, 1), (203, 0), (256, 3)):
        big = torch.full((m * ld + start + 300,), float("nan"), device="cuda", dtype=dtype)
        x = big[start:start + m * ld].view(m, ld)[:, :k]
        x.copy_(torch.randn((m, k), generator=r, device="cuda"))
        room = torch.full((m + 2, n + 5), 7.0, device="cuda", dtype=dtype)
        got = packed.gemm(h, x, part, out=room[1:-1, 2:2 + n])
        check_product(got, x, codes, part.scale, part.zero, 32, (ld, start))
        got.fill_(7.0)
        assert (room == 7.0).all()


@pytest.mark.parametrize("counts", [[0, 5, 0, 1, 40, 17, 0], [0, 0, 0], [1], [100, 0, 33], [3] * 70])
@pytest.mark.parametrize("dtype", FLOATS)
def test_grouped(h, counts, dtype):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(len(counts))
    n, k, behind = 45, 330, 6
    w = weights(r, n, k, 64, True, torch.bfloat16, (len(counts),))
    m = sum(counts) + behind
    x = torch.randn((m, k), generator=r, device="cuda").to(dtype)
    x[sum(counts):] = float("nan")            # rows behind the last group are not read
    offsets = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    y = packed.gemm_grouped(h, x, w, offsets)
    at = 0
    for e, c in enumerate(counts):
        if c:
            check_product(y[at:at + c], x[at:at + c], ref.codes_of(w.data[e], k), w.scale[e], w.zero[e], 64, e)
        at += c
    assert not y[at:].any()


def test_nothing_to_do(h):
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(8)
    w = weights(r, 20, 64, 32, False, torch.float16)
    assert packed.gemm(h, torch.empty((0, 64), device="cuda"), w).shape == (0, 20)
    none = packed.empty(20, 0)
    assert not packed.gemm(h, torch.empty((3, 0), device="cuda"), none).any()
    assert packed.unpack(h, packed.quantize(h, torch.empty((0, 64), device="cuda"))).shape == (0, 64)


def test_captured_and_replayed_with_other_inputs(h):
    from paper_2511_13778_amd import experts, packed
    r = torch.Generator(device="cuda").manual_seed(9)
    w = weights(r, 96, 256, 128, False, torch.float16, (8,))
    x = torch.randn((24, 256), generator=r, device="cuda").bfloat16()
    scores = torch.randn((24, 8), generator=r, device="cuda")

    def step():
        c = experts.choose(h, scores, 2, balance=False)
        routing = experts.sort_tokens(h, c.ids, 8)
        ys = packed.gemm_grouped(h, experts.gather(h, x, routing), w, routing.offsets)
        return experts.combine(h, ys, routing, c.weights)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(4):
        x.copy_(torch.randn((24, 256), generator=r, device="cuda"))
        scores.copy_(torch.randn((24, 8), generator=r, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(step(), got)


def special(x, codes, scale, zero, group):
    """x W^T with the infinities and NaN that its 64-bit terms have."""
    return x.double() @ ref.values(codes, scale, zero, group).T


def check_special(got, exact, what):
    got = got.double()
    assert torch.equal(got.isnan(), exact.isnan()) and torch.equal(got == float("inf"), exact == float("inf")) and torch.equal(got == -float("inf"), exact == -float("inf")), what


@pytest.mark.parametrize("m,n,k", [(3, 9, 1), (2, 5, 7), (1, 40, 8), (3, 70, 300), (4, 33, 1000), (12, 50, 201), (20, 37, 330), (40, 90, 257), (70, 40, 129)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_infinities_keep_their_sign(h, m, n, k, group, zeros):
    # an infinity times a value is an infinity of the product's sign; NaN where the value is zero (code = zero point) or infinities of both signs meet
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(m + n + k)
    inf = float("inf")
    for dtype in FLOATS:
        w = weights(r, n, k, group, zeros, torch.float32)
        if zeros:
            w.zero.copy_(w.zero.round())
        x = torch.randn((m, k), generator=r, device="cuda").to(dtype)
        y = packed.gemm(h, x, w)
        x[0, k - 1] = inf
        if m > 1:
            x[m - 1, k // 2] = -inf
        if m > 2:
            x[m // 2, 0] = inf
            x[m // 2, k - 1] = -inf
        if m > 3:
            x[1, k // 3] = float("nan")
        if m > 4:
            x[2, 0] = x[2, k - 1] = -inf
        codes = ref.codes_of(w.data, k)
        exact = special(x, codes, w.scale, w.zero, group)
        assert exact.isinf().any()
        for out in {dtype, torch.float32}:
            check_special(packed.gemm(h, x, w, dtype=out), exact, (dtype, out))
        rest = x.isfinite().all(1)
        assert torch.equal(packed.gemm(h, x, w)[rest], y[rest])
        # one row of W alone with a scale that is no number
        w.scale[0, n // 2] = float("nan")
        check_special(packed.gemm(h, x, w), special(x, codes, w.scale, w.zero, group), (dtype, "scale"))


@pytest.mark.parametrize("m,n,k", [(2, 9, 5), (1, 40, 300), (4, 70, 1000), (12, 50, 201), (40, 90, 257)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sums_that_pass_the_range_on_the_way(h, m, n, k, zeros, dtype):
    # x near the type's end, scales that bring the results back: 128 + code, codes or their sums alone would be infinite
    from paper_2511_13778_amd import packed
    r = torch.Generator(device="cuda").manual_seed(m + n + k)
    w = weights(r, n, k, 64, zeros, torch.float32)
    w.scale.copy_(w.scale.clamp(-2.0, 2.0) * 1e-6)
    x = (torch.rand((m, k), generator=r, device="cuda") * 2.0 - 1.0).to(dtype)
    x[::2] *= 1e36
    x[0] *= 300.0
    x[:, 0] = torch.finfo(dtype).max
    codes = ref.codes_of(w.data, k)
    assert x.isfinite().all()
    for out in {dtype, torch.float32}:
        check_product(packed.gemm(h, x, w, dtype=out), x, codes, w.scale, w.zero, 64, (dtype, out))
