"""Every kernel of the 8-bit products, each at sizes of its own (scaled_routes), against 64 bits: values, sums added to what is there, views, groups with
uneven loads, NaN, and what the sums keep.

Tolerances.  The 8-bit matrix instruction adds products by eights and cuts each off at 2^-13 of the largest of the eight, so the other seven lose
less than 7 2^-13 of it, which is at most the eight's part of S = sum |a b|; the losses of different eights are independent.
  an element               16 bits: a rounding of at most `unit`, and 7 2^-13 S / sqrt(eights);  32 bits: k + 128 roundings of 2^-24 S
  root mean square,        16 bits: roundings evenly spread, unit / sqrt(3), and losses: 2^-13 / sqrt(3) of the largest, which is about three times
  against the results'     the root mean square;  32 bits: a rounding of 2^-24 of a partial sum for every eight and for every block's scale,
                           independent: 2^-24 sqrt(k / 8 + k / 128 + 8)."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import scaled_reference as ref  # noqa: E402
import scaled_routes as sr  # noqa: E402
from test_gpu_scaled import E4M3, E5M2, dense, gen, matrix  # noqa: E402

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
CASES = [(label, size, scale, out) for label, sizes in sr.DENSE.items() for size in sizes for kind, (scale, outs) in
         enumerate([(torch.uint8, (torch.bfloat16, torch.float16)), (torch.float32, (torch.bfloat16, torch.float16)), (torch.uint8, (torch.float32,)),
                    (torch.float32, (torch.float32,))]) if kind in sr.HAS.get(sr.ROUTE[label], sr.KINDS) for out in outs]
NAMES = ["%s-%s-%s-%s" % (label, "x".join(map(str, size)), str(scale)[6:], str(out)[6:]) for label, size, scale, out in CASES]


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def close(got, exact, size, k):
    err = (got.double() - exact).abs()
    if got.dtype == torch.float32:
        bound = 2.0 ** -23 * exact.abs() + (k + 128) * 2.0 ** -24 * size
    else:
        bound = UNIT[got.dtype] * exact.abs() + 7 * 2.0 ** -13 * (-(-k // 8)) ** -0.5 * size
    assert torch.isfinite(got).all()
    assert (err <= bound + 2.0 ** -24).all(), (err / bound).max().item()


def near(got, exact, size, k):
    close(got, exact, size, k)
    rms = lambda t: t.double().square().mean().sqrt().item()  # noqa: E731
    bound = 2.0 ** -24 * (k / 8 + k / 128 + 8) ** 0.5 if got.dtype == torch.float32 else (UNIT[got.dtype] + 3 * 2.0 ** -13) / 3 ** 0.5
    if got.numel() >= 256:
        assert rms(got.double() - exact) <= bound * rms(exact), (rms(got.double() - exact) / rms(exact), bound)


def small(m, by=4):
    """The matrix with scales that keep products within float16."""
    if m.scale.dtype == torch.uint8:
        m.scale -= by
    else:
        m.scale *= 2.0 ** -by
    return m


@pytest.mark.parametrize("label,size,scale,out", CASES, ids=NAMES)
def test_values_and_sums(h, label, size, scale, out):
    from paper_2511_13778_amd import scaled
    m, n, k = size
    for a_type, rows_b in ((E4M3, 128), (E5M2, 1)):
        a, b = small(matrix(m + k, m, k, a_type, scale, spread=0.5)), matrix(n + 1, n, k, E4M3, scale, rows_b, spread=0.5)
        da, db = dense(a), dense(b)
        exact, total = da @ db.t(), da.abs() @ db.abs().t()
        got = scaled.gemm(h, a, b, dtype=out)
        near(got, exact, total, k)
        assert torch.equal(scaled.gemm(h, a, b, dtype=out), got)           # the same bits again
        # added to a view whose rows start at odd elements; what lies around stays
        whole = torch.randn((m + 2, n + 5), generator=gen(k), device="cuda").to(out)
        before = whole.clone()
        view = whole[1:m + 1, 3:n + 3]
        scaled.gemm(h, a, b, out=view, accumulate=True)
        old = before[1:m + 1, 3:n + 3].double()
        near(view, exact + old, total + old.abs(), k)
        view.copy_(before[1:m + 1, 3:n + 3])
        assert torch.equal(whole, before)


@pytest.mark.parametrize("label,size,scale,out", [(a, b, s, o) for a, b, s, o in CASES if b == sr.DENSE[a][-1]],
                         ids=[n for n, (a, b, _, _) in zip(NAMES, CASES) if b == sr.DENSE[a][-1]])
def test_nan_scales_and_values_stay_in_their_rows(h, label, size, scale, out):
    from paper_2511_13778_amd import scaled
    m, n, k = size
    for rows_b in (1, 128):
        a, b = small(matrix(3, m, k, E4M3, scale)), matrix(4, n, k, E4M3, scale, rows_b)
        nb = -(-k // 128)
        want = torch.zeros((m, n), dtype=torch.bool, device="cuda")
        a.scale[m // 2, nb - 1] = 255 if scale == torch.uint8 else float("nan")
        a.data.view(torch.uint8)[m - 1, k - 1] = 0x7F                 # e4m3 NaN
        b.data.view(torch.uint8)[n // 3, 0] = 0xFF
        b.scale[-1, nb // 2] = 255 if scale == torch.uint8 else float("nan")
        want[m // 2] = want[m - 1] = True
        want[:, n // 3] = True
        want[:, n - 1 if rows_b == 1 else (n - 1) // 128 * 128:] = True
        assert torch.equal(scaled.gemm(h, a, b, dtype=out).isnan(), want)


def cancelling(rows, k, high, low_type, generator):
    """Whole numbers: +high and -high (by turns of the factor) in the first two places of every block, 0, 1 or 2 behind them."""
    x = torch.zeros((rows, -(-k // 16) * 16), device="cuda")
    x[:, :k] = torch.randint(0, 3, (rows, k), generator=generator, device="cuda").float()
    for b in range(0, k - 1, 128):
        x[:, b] = high
        x[:, b + 1] = high
    return x.to(low_type)


@pytest.mark.parametrize("label", sr.DENSE)
def test_what_sums_keep_where_large_products_cancel(h, label):
    # each block has 2^16 and -2^16 among small whole numbers; every partial sum is below 2^24.  A float32 result is the exact one; one in 16 bits loses at
    # most 2^-13 of the largest product for each of the others of its eight, and does lose it
    from paper_2511_13778_amd import scaled
    m, n, k = max(sr.DENSE[label], key=lambda s: s[2])
    nb = -(-k // 128)
    r = gen(7)
    lost = 0
    for a_type in (E4M3, E5M2):
        xa, xb = cancelling(m, k, 256.0, a_type, r), cancelling(n, k, 256.0, E4M3, r)
        for b in range(0, k - 1, 128):
            xb[:, b + 1] = torch.full((), -256.0, device="cuda").to(E4M3)
        exact = xa[:, :k].double() @ xb[:, :k].double().t()
        for scale in (torch.uint8, torch.float32):
            one = [torch.full((v, -(-nb // 4) * 4), 127, dtype=torch.uint8, device="cuda") if scale == torch.uint8 else torch.ones((v, nb), device="cuda") for v in (m, n)]
            a, b = scaled.Scaled(xa, one[0], k), scaled.Scaled(xb, one[1], k)
            for out in (torch.float32, torch.bfloat16):
                got = scaled.gemm(h, a, b, dtype=out).double()
                if out == torch.float32:
                    assert torch.equal(got, exact)
                else:
                    off = (got - exact).abs()
                    assert (off <= 2.0 ** -8 * exact.abs() + nb * 7 * 2.0 ** -13 * 2.0 ** 16 + 2.0 ** -8 * nb * 56).all()
                    lost += int((off > 2.0 ** -8 * exact.abs()).any())
    if k >= 8:
        assert lost, "the 8-bit instruction keeps more than is stated"


GROUPS = [(label, i, scale, out) for label, sizes in sr.ROWS.items() for i in range(len(sizes)) for scale in (torch.uint8, torch.float32)
          for out in (torch.bfloat16, torch.float32)]


@pytest.mark.parametrize("label,i,scale,out", GROUPS)
def test_rows_in_uneven_groups(h, label, i, scale, out):
    from paper_2511_13778_amd import scaled
    counts, behind, n, k = sr.ROWS[label][i]
    live, ends = sum(counts), [sum(counts[:j]) for j in range(len(counts) + 1)]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for a_type, rows_b in ((E4M3, 128), (E5M2, 1)):
        a, b = matrix(5, live + behind, k, a_type, scale, spread=0.5), matrix(6, n, k, E4M3, scale, rows_b, groups=len(counts), spread=0.5)
        if behind:
            a.data[live:].fill_(float("nan"))
        got = scaled.gemm_grouped(h, a, b, offsets, dtype=out)
        da, db = dense(a), dense(b)
        for e, c in enumerate(counts):
            rows = slice(ends[e], ends[e] + c)
            if c:
                near(got[rows], da[rows] @ db[e].t(), da[rows].abs() @ db[e].abs().t(), k)
        assert not got[live:].any()


@pytest.mark.parametrize("label,scale,out", [(label, scale, out) for label in sr.CONTRACTION for scale in (torch.uint8, torch.float32)
                                             for out in (torch.bfloat16, torch.float32)])
def test_contraction_in_uneven_groups(h, label, scale, out):
    from paper_2511_13778_amd import scaled
    for counts, behind, m, n in sr.CONTRACTION[label]:
        rows, ends = sum(counts) + behind, [sum(counts[:j]) for j in range(len(counts) + 1)]
        offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        y, x = torch.randn((rows, m), generator=gen(11), device="cuda"), torch.randn((rows, n), generator=gen(12), device="cuda")
        a = scaled.quantize(h, y, E5M2, scale, which="columns", offsets=offsets)
        b = scaled.quantize(h, x, E4M3, scale, which="columns", offsets=offsets)
        assert a.cols == sr.columns(counts, behind)
        got = scaled.gemm_grouped_k(h, a, b, offsets, dtype=out)
        added = torch.full_like(got, 0.5)
        scaled.gemm_grouped_k(h, a, b, offsets, out=added, accumulate=True)
        for e, c in enumerate(counts):
            if not c:
                assert not got[e].any() and (added[e] == 0.5).all()
                continue
            part = slice(ends[e], ends[e] + c)
            (qy, ey), (qx, ex) = ref.quantize(y[part].t(), E5M2, 1), ref.quantize(x[part].t(), E4M3, 1)
            dy, dx = (q * ref.power(v).repeat_interleave(128, 1)[:, :c] for q, v in ((qy, ey), (qx, ex)))
            exact, total = dy @ dx.t(), dy.abs() @ dx.abs().t()
            near(got[e], exact, total, c)
            close(added[e], exact + 0.5, total + 0.5, c)
