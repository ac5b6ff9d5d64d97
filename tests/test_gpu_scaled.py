"""8-bit block-scaled quantiser and products against their definitions in 64 bits, through the public calls."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import scaled_reference as ref  # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def gen(seed):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    return r


def matrix(seed, rows, cols, dtype=E4M3, scale=torch.uint8, block_rows=1, groups=None, pad=0, spread=1.0):
    """A random 8-bit matrix; the padding of its rows and of its scales holds NaN."""
    from paper_2511_13778_amd import scaled
    r = gen(seed)
    lead = () if groups is None else (groups,)
    ld = -(-cols // 16) * 16 + 16 * pad
    x = torch.full(lead + (rows, ld), float("nan"), device="cuda")
    x[..., :cols] = torch.randn(lead + (rows, cols), generator=r, device="cuda") * (ref.TOP[dtype] / 8)
    nb = -(-cols // 128)
    s = torch.full(lead + (-(-rows // block_rows), -(-nb // 4) * 4 + 4 * pad), float("nan"), device="cuda")
    s[..., :nb] = torch.randn(s[..., :nb].shape, generator=r, device="cuda") * spread - 8
    if scale == torch.float32:
        s = torch.exp2(s)
    else:
        s = torch.where(s.isnan(), 255, s.round() + 127).to(torch.uint8)
    return scaled.Scaled(x.clamp(-ref.TOP[dtype], ref.TOP[dtype]).to(dtype), s, cols, block_rows)


def dense(m):
    return ref.dequantize(m.data, m.scale, m.cols, m.block_rows)


# Rounding to the result's type, and what the sums may lose against S = sum |a b|: the 8-bit matrix instruction drops bits below
# 2^-16 of a sum's largest product, at most 128 of them per block, most of them far less (2^-14 S is allowed); sums in 32 bits have at
# most k + 128 roundings of 2^-24 each.
def close(got, exact, size, k):
    unit, loss = {torch.bfloat16: (2.0 ** -8, 2.0 ** -14), torch.float16: (2.0 ** -10, 2.0 ** -14),
                  torch.float32: (2.0 ** -23, (k + 128) * 2.0 ** -24)}[got.dtype]
    err = (got.double() - exact).abs()
    bound = unit * exact.abs() + loss * size + 2.0 ** -24
    assert torch.isfinite(got).all()
    assert (err <= bound).all(), ((err / bound).max().item(), (err > bound).nonzero()[:4].tolist())


SHAPES = [(1, 1, 1), (1, 17, 128), (3, 130, 129), (16, 256, 512), (33, 100, 777), (65, 129, 255), (128, 128, 640), (130, 257, 1000), (200, 300, 260),
          (256, 256, 128), (257, 300, 1300), (300, 513, 384), (512, 256, 2048), (1, 512, 8192), (7, 96, 40000)]


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(h, m, n, k, scale, out):
    from paper_2511_13778_amd import scaled
    seed = m * 7 + n * 3 + k
    for a_type, rows_b in ((E4M3, 128), (E5M2, 1)):
        a, b = matrix(seed, m, k, a_type, scale), matrix(seed + 1, n, k, E4M3, scale, rows_b)
        da, db = dense(a), dense(b)
        exact, size = da @ db.t(), da.abs() @ db.abs().t()
        if out == torch.float16 and size.max() > 30000:        # keep within the type's range
            f = 14
            if scale == torch.uint8:
                b.scale -= f
            else:
                b.scale *= 2.0 ** -f
            db = dense(b)
            exact, size = da @ db.t(), da.abs() @ db.abs().t()
        close(scaled.gemm(h, a, b, dtype=out), exact, size, k)


# sizes that fill the chip with tiles of 256 x 256, 256 x 128 and 128 x 128, ragged, of one step to many, odd and even in number; and few tiles with a
# long k, which is cut
@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,n,k", [(3700, 3650, 100), (3600, 3700, 256), (3601, 3841, 777), (2500, 2600, 128), (2305, 2590, 1290), (2600, 2500, 640), (2100, 2000, 300),
                                   (100, 300, 9000), (300, 70, 20001), (65, 65, 4096), (40, 200, 16500)])
def test_product_large(h, m, n, k, scale, out):
    from paper_2511_13778_amd import scaled
    for a_type, rows_b in ((E4M3, 128), (E5M2, 1)):
        a, b = matrix(m + k, m, k, a_type, scale, spread=0.5), matrix(n, n, k, E4M3, scale, rows_b, spread=0.5)
        if scale == torch.uint8:
            a.scale -= 6                                        # within float16's range
        else:
            a.scale *= 2.0 ** -6
        da, db = dense(a), dense(b)
        exact, size = da @ db.t(), da.abs() @ db.abs().t()
        got = scaled.gemm(h, a, b, dtype=out)
        close(got, exact, size, k)
        if out != torch.float16:
            c = got.clone()
            scaled.gemm(h, a, b, out=c, accumulate=True)
            close(c, exact + got.double(), size + got.double().abs(), k)


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_groups_large(h, scale, out):
    # groups that fill tall tiles, and one that ends inside each kind of tile
    from paper_2511_13778_amd import scaled
    counts, k, n = [700, 0, 1500, 257, 3, 900, 640], 500, 2700
    offsets = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    a, b = matrix(5, sum(counts) + 9, k, E4M3, scale), matrix(6, n, k, E4M3, scale, 128, groups=len(counts))
    got = scaled.gemm_grouped(h, a, b, offsets, dtype=out)
    da, db = dense(a), dense(b)
    for e, c in enumerate(counts):
        rows = slice(int(offsets[e]), int(offsets[e]) + c)
        if c:
            close(got[rows], da[rows] @ db[e].t(), da[rows].abs() @ db[e].abs().t(), k)
    assert not got[sum(counts):].any()
    r = gen(2)
    y, x = torch.randn((sum(counts), 1500), generator=r, device="cuda"), torch.randn((sum(counts), 1400), generator=r, device="cuda")
    qa, qb = (scaled.quantize(h, v, E4M3, scale, which="columns", offsets=offsets) for v in (y, x))
    got = scaled.gemm_grouped_k(h, qa, qb, offsets, dtype=out)
    for e, c in enumerate(counts):
        part = slice(int(offsets[e]), int(offsets[e]) + c)
        if c:
            (qy, ey), (qx, ex) = ref.quantize(y[part].t(), E4M3, 1), ref.quantize(x[part].t(), E4M3, 1)
            dy, dx = (q * ref.power(v).repeat_interleave(128, 1)[:, :c] for q, v in ((qy, ey), (qx, ex)))
            close(got[e], dy @ dx.t(), dy.abs() @ dx.abs().t(), c)
        else:
            assert not got[e].any()


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k,pad", [(5, 70, 200, 1), (130, 260, 500, 3), (300, 290, 777, 2), (512, 512, 256, 0)])
def test_product_with_strides_and_added(h, m, n, k, pad, scale, out):
    from paper_2511_13778_amd import scaled
    a, b = matrix(k, m, k, E4M3, scale, 1, pad=pad), matrix(k + 1, n, k, E4M3, scale, 128, pad=pad)
    da, db = dense(a), dense(b)
    exact, size = da @ db.t(), da.abs() @ db.abs().t()
    r = gen(9)
    whole = torch.randn((m + 2, n + pad + 3), generator=r, device="cuda").to(out)
    before = whole.clone()
    c = whole[1:m + 1, pad:pad + n]
    scaled.gemm(h, a, b, out=c, accumulate=True)
    close(c, exact + before[1:m + 1, pad:pad + n].double(), size + before[1:m + 1, pad:pad + n].double().abs(), k)
    whole[1:m + 1, pad:pad + n] = before[1:m + 1, pad:pad + n]
    assert torch.equal(whole, before)                     # nothing outside the view is written


def test_product_rows_and_blocks_share_scales(h):
    # a matrix scaled by 128 x 128 blocks is the same as one whose rows repeat those scales
    from paper_2511_13778_amd import scaled
    for scale in (torch.uint8, torch.float32):
        a, b = matrix(1, 300, 900, E4M3, scale), matrix(2, 270, 900, E4M3, scale, 128)
        rows = scaled.Scaled(b.data, b.scale.repeat_interleave(128, 0)[:270].contiguous(), 900, 1)
        for out in (torch.bfloat16, torch.float32):
            assert torch.equal(scaled.gemm(h, a, b, dtype=out), scaled.gemm(h, a, rows, dtype=out))


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
def test_nan_scale_and_values_stay_in_their_rows(h, scale, out):
    from paper_2511_13778_amd import scaled
    for m, n, k in ((20, 40, 300), (300, 300, 520)):
        a, b = matrix(3, m, k, E4M3, scale), matrix(4, n, k, E4M3, scale, 1)
        a.scale[3, 1] = 255 if scale == torch.uint8 else float("nan")
        a.data.view(torch.uint8)[5, k - 1] = 0x7F                 # e4m3 NaN
        b.data.view(torch.uint8)[7, 0] = 0xFF
        got = scaled.gemm(h, a, b, dtype=out).isnan()
        want = torch.zeros((m, n), dtype=torch.bool, device="cuda")
        want[3] = want[5] = True
        want[:, 7] = True
        assert torch.equal(got, want)


def test_no_contraction_gives_zero(h):
    from paper_2511_13778_amd import ozdgemm as g, scaled
    a, b = scaled.empty(5, 0), scaled.empty(6, 0, 128)
    c = torch.full((5, 6), 3.0, device="cuda")
    assert torch.equal(scaled.gemm(h, a, b, out=c), torch.zeros_like(c))
    c.fill_(3.0)
    assert torch.equal(scaled.gemm(h, a, b, out=c, accumulate=True), torch.full_like(c, 3.0))
    assert scaled.gemm(h, scaled.empty(0, 128), scaled.empty(6, 128, 128)).shape == (0, 6)
    assert g is not None


GROUPS = [([0, 5, 0, 0, 17, 1], 30, 3), ([128, 0, 129, 300], 700, 0), ([0, 0, 0], 4, 4), ([1] * 40, 260, 2), ([260, 600], 300, 5), ([1000], 128, 0),
          ([3, 700, 64, 16, 15, 0, 33], 200, 6)]


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,k,behind", GROUPS)
def test_rows_in_groups(h, counts, k, behind, scale, out):
    from paper_2511_13778_amd import scaled
    live, m, n = sum(counts), sum(counts) + behind, 270
    offsets = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    a, b = matrix(5, m, k, E4M3, scale), matrix(6, n, k, E4M3, scale, 128, groups=len(counts))
    if behind:
        a.data[live:].fill_(float("nan"))
    got = scaled.gemm_grouped(h, a, b, offsets, dtype=out)
    da, db = dense(a), dense(b)
    for e, c in enumerate(counts):
        rows = slice(int(offsets[e]), int(offsets[e]) + c)
        if c:
            close(got[rows], da[rows] @ db[e].t(), da[rows].abs() @ db[e].abs().t(), k)
    assert torch.equal(got[live:], torch.zeros_like(got[live:]))


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,behind", [(c, b) for c, _, b in GROUPS])
def test_contraction_in_groups(h, counts, behind, scale, out):
    # from quantize: the transposes of two matrices whose rows are in groups
    from paper_2511_13778_amd import scaled
    rows, m, n = sum(counts) + behind, 140, 270
    offsets = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    r = gen(11)
    y, x = torch.randn((rows, m), generator=r, device="cuda"), torch.randn((rows, n), generator=r, device="cuda")
    a = scaled.quantize(h, y, E5M2, scale, which="columns", offsets=offsets)
    b = scaled.quantize(h, x, E4M3, scale, which="columns", offsets=offsets)
    got = scaled.gemm_grouped_k(h, a, b, offsets, dtype=out)
    added = got.clone()
    scaled.gemm_grouped_k(h, a, b, offsets, out=added, accumulate=True)
    at = 0
    for e, c in enumerate(counts):
        part = slice(int(offsets[e]), int(offsets[e]) + c)
        if c:
            (qy, ey), (qx, ex) = ref.quantize(y[part].t(), E5M2, 1), ref.quantize(x[part].t(), E4M3, 1)
            wide = -(-c // 128)
            assert torch.equal(a.values()[:, at * 128:at * 128 + c].float().double(), qy)
            assert torch.equal(ref.scale_values(a.scale[:, at:at + wide]), ref.power(ey))
            dy = qy * ref.power(ey).repeat_interleave(128, 1)[:, :c]
            dx = qx * ref.power(ex).repeat_interleave(128, 1)[:, :c]
            close(got[e], dy @ dx.t(), dy.abs() @ dx.abs().t(), c)
            close(added[e], 2 * (dy @ dx.t()), 2 * dy.abs() @ dx.abs().t(), c)
            at += wide
        else:
            assert not got[e].any() and not added[e].any()


@pytest.mark.parametrize("x_type", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [E4M3, E5M2])
@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 129), (16, 128), (130, 257), (128, 1000), (300, 640)])
def test_quantize(h, rows, cols, scale, dtype, x_type):
    from paper_2511_13778_amd import scaled
    r = gen(rows + cols)
    x = torch.randn((rows, cols), generator=r, device="cuda") * torch.exp2(torch.randint(-9, 9, (rows, cols), generator=r, device="cuda").float())
    x[torch.rand((rows, cols), generator=r, device="cuda") < 0.1] = 0
    x[0, :min(cols, 128)] = 0                                # a block of zeros
    if rows > 2:
        x[2, :100] *= 2.0 ** (-20 if x_type == torch.float16 else -110)
        x[1] = x[1].abs() + 1                            # maxima at either side of the type's largest value
        x[1, 0] = 448.0
        if cols > 128:
            x[1, 128] = 450.0
    x = x.to(x_type)
    for block_rows in (1, 128):
        for which in ("rows", "columns", "both"):
            got = scaled.quantize(h, x, dtype, scale, block_rows, which)
            for m, src in zip(got if which == "both" else (got,), ((x, x.t()) if which == "both" else (x.t(),) if which == "columns" else (x,))):
                v, e = ref.quantize(src, dtype, block_rows)
                assert torch.equal(m.values().float().double(), v)
                assert torch.equal(ref.scale_values(m.scales()), ref.power(e))
                assert not m.data[:, m.cols:].float().any()        # the padding up to 16 is zero


def test_quantize_strided_batched_and_unaligned(h):
    from paper_2511_13778_amd import scaled
    r = gen(4)
    big = torch.randn((70, 400), generator=r, device="cuda").bfloat16()
    for view in (big[3:, 5:305], big[:, 1:2], big[::2, 16:]):
        for which in ("rows", "columns"):
            m = scaled.quantize(h, view, which=which)
            v, e = ref.quantize(view if which == "rows" else view.t(), E4M3, 1)
            assert torch.equal(m.values().float().double(), v) and torch.equal(ref.scale_values(m.scales()), ref.power(e))
    w = torch.randn((3, 200, 300), generator=r, device="cuda")
    a, t = scaled.quantize(h, w, block_rows=128, which="both")
    for i in range(3):
        for m, src in ((a, w[i]), (t, w[i].t())):
            v, e = ref.quantize(src, E4M3, 128)
            assert torch.equal(m.values()[i].float().double(), v) and torch.equal(ref.scale_values(m.scales()[i]), ref.power(e))


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
def test_quantize_infinities_and_nan(h, scale):
    from paper_2511_13778_amd import scaled
    x = torch.randn((200, 300), device="cuda")
    x[3, 5], x[4, 200], x[199, 299] = float("inf"), float("nan"), float("-inf")
    for which, src in (("rows", x), ("columns", x.t())):
        for block_rows in (1, 128):
            m = scaled.quantize(h, x, scale_dtype=scale, block_rows=block_rows, which=which)
            v, e = ref.quantize(src, E4M3, block_rows)
            assert torch.equal(torch.nan_to_num(m.values().float().double(), nan=1e9), torch.nan_to_num(v, nan=1e9))
            assert torch.equal(ref.scale_values(m.scales()).isnan(), e == 128)


def test_quantize_extremes(h):
    # the largest and least numbers of float32: scales at the ends of their range
    from paper_2511_13778_amd import scaled
    x = torch.zeros((4, 128), device="cuda")
    x[0, 3], x[1, 4], x[2, 5], x[3, 6] = torch.finfo(torch.float32).max, 1e-38, 1e-45, 2.0 ** -126
    for dtype in (E4M3, E5M2):
        m = scaled.quantize(h, x, dtype, torch.uint8)
        v, e = ref.quantize(x, dtype, 1)
        assert torch.equal(m.values().float().double(), v) and torch.equal(ref.scale_values(m.scales()), ref.power(e))


def test_other_stream(h):
    from paper_2511_13778_amd import scaled
    a, b = matrix(1, 300, 512), matrix(2, 300, 512, block_rows=128)
    want = scaled.gemm(h, a, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = scaled.gemm(h, a, b)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def test_refusals(h):
    from paper_2511_13778_amd import ozdgemm as g, scaled
    a, b = matrix(1, 32, 256), matrix(2, 48, 256, block_rows=128)
    good = torch.empty((32, 48), device="cuda")

    def call(**change):
        args = dict(m=32, n=48, k=256, a=a, b=b, c=good.data_ptr(), ldc=48, t=g.OZ_F32, acc=0) | change
        h.call("oz_scaled_gemm", 0, args["m"], args["n"], args["k"], args["a"].desc if args["a"] else None, args["b"].desc if args["b"] else None,
               args["c"], args["ldc"], args["t"], args["acc"], None, 0)

    def but(m, **change):
        class M:
            desc = g.oz_scaled_t(*[change.get(f, getattr(m.desc, f)) for f, _ in g.oz_scaled_t._fields_])
        return M
    call()
    for bad in (dict(m=-1), dict(k=(1 << 24) + 1), dict(ldc=47), dict(t=g.OZ_E4M3), dict(acc=2), dict(c=None), dict(c=good.data_ptr() + 1), dict(a=None),
                dict(a=but(a, ld=250)), dict(a=but(a, ld=264)), dict(a=but(a, data=a.data.data_ptr() + 8)), dict(a=but(a, scale_ld=1)),
                dict(a=but(a, scale_ld=6)), dict(a=but(a, type=g.OZ_BF16)), dict(a=but(a, scale_type=g.OZ_F32)), dict(a=but(a, block_rows=64)),
                dict(b=but(b, type=g.OZ_E5M2)), dict(b=but(b, reserved_=1)), dict(a=but(a, scale=None)), dict(b=but(b, data=None))):
        with pytest.raises(g.OzError) as e:
            call(**bad)
        assert e.value.status == 1, bad
    x = torch.zeros((8, 8), device="cuda")
    for bad in (dict(which="sideways"), dict(dtype=torch.float16), dict(scale_dtype=torch.float16)):
        with pytest.raises(ValueError):
            scaled.quantize(h, x, **bad)
    with pytest.raises(ValueError):
        scaled.quantize(h, x.t()[:, ::2])
    with pytest.raises(ValueError):
        scaled.quantize(h, x.double())
    with pytest.raises(ValueError):
        scaled.quantize(h, x.cpu())
    with pytest.raises(ValueError):
        scaled.gemm(h, a, matrix(2, 48, 200, block_rows=128))
    with pytest.raises(ValueError):
        scaled.gemm(h, a, b, accumulate=True)
    with pytest.raises(ValueError):
        scaled.Scaled(a.data, a.scale[:4], 256)
    with pytest.raises(g.OzError):
        scaled.quantize(h, x, block_rows=128, which="columns", offsets=torch.tensor([0, 8], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
