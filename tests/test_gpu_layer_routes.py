"""Every way in which products with 4-bit weights and orthogonal updates are cut up, against 64-bit forms."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
import layer_routes as lr  # noqa: E402
from test_gpu_orthogonal import EPS, QUINTIC, check_five, gradient, parts_of  # noqa: E402
from test_gpu_packed import check_product, check_special, special, weights  # noqa: E402


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


@pytest.mark.parametrize("at", sorted(lr.PACKED), ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_packed_products(h, at, dtype):
    from paper_2511_13778_amd import packed
    for counts, behind, n, k, group, kinds in lr.PACKED[at]:
        if dtype.itemsize not in kinds:
            continue
        r = torch.Generator(device="cuda").manual_seed(n + k + group)
        zeros = group != 64
        w = weights(r, n, k, group, zeros, torch.float16, (len(counts),) if counts else ())
        m = sum(counts) + behind
        x = torch.randn((m, k), generator=r, device="cuda").to(dtype)
        if not counts:
            check_product(packed.gemm(h, x, w), x, ref.codes_of(w.data, k), w.scale, w.zero, group, (at, n, k))
            continue
        offsets = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
        y = packed.gemm_grouped(h, x, w, offsets)
        first = 0
        for e, c in enumerate(counts):
            if c:
                check_product(y[first:first + c], x[first:first + c], ref.codes_of(w.data[e], k), w.scale[e], w.zero[e] if zeros else None, group, (at, n, k, e))
            first += c
        assert not y[first:].any()


@pytest.mark.parametrize("dtype,at", [(torch.bfloat16, i) for i in range(len(lr.ORTHO[1]))] + [(torch.float32, i) for i in range(len(lr.ORTHO[2]))])
def test_tiles_of_orthogonal_updates(h, dtype, at):
    from paper_2511_13778_amd import orthogonal
    sizes = list(lr.ORTHO[parts_of(dtype)].values())
    batch, rows, cols = sizes[at]
    r = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = gradient(r, batch, rows, cols).to(dtype)
    got = orthogonal.orthogonalize(h, x, steps=1, eps=EPS)
    if rows != cols:                          # (square ones are taken as they are: their other product with themselves)
        turned = orthogonal.orthogonalize(h, x.transpose(1, 2).contiguous(), steps=1, eps=EPS)
        assert torch.equal(turned.transpose(1, 2), got)
    for i in range(batch):
        exact, bound = ref.orthogonalize_bound(x[i], QUINTIC, EPS, parts_of(dtype))
        err = (got[i].double() - exact).abs()
        bound = bound + ref.rounded(exact, dtype)
        assert (err <= bound).all(), (i, (err / bound).max().item())
    five = orthogonal.orthogonalize(h, x)
    assert torch.equal(five, orthogonal.orthogonalize(h, x))
    for i in (0, batch - 1):
        check_five(five[i], x[i])


def product_of(h, x, w, counts):
    from paper_2511_13778_amd import packed
    if not counts:
        return packed.gemm(h, x, w), torch.zeros(x.shape[0], dtype=torch.int64)
    offsets = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    return packed.gemm_grouped(h, x, w, offsets), torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts))


@pytest.mark.parametrize("at", sorted(lr.PACKED), ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_infinities_in_packed_products(h, at, dtype):
    for counts, behind, n, k, group, kinds in lr.PACKED[at]:
        if dtype.itemsize not in kinds:
            continue
        r = torch.Generator(device="cuda").manual_seed(n + k + group)
        zeros = group != 64
        w = weights(r, n, k, group, zeros, torch.float32, (len(counts),) if counts else ())
        if zeros:
            w.zero.copy_(w.zero.round())
        m = sum(counts) + behind
        x = torch.randn((m, k), generator=r, device="cuda").to(dtype)
        x[::3, k - 1] = float("inf")
        x[1::7, k // 2] = -float("inf")
        x[5::11, 0] = float("nan")
        y, of = product_of(h, x, w, counts)
        for e in range(max(1, len(counts))):
            mine = (of == e).nonzero()[:, 0].cuda()
            pick = (lambda v: v[e]) if counts else (lambda v: v)
            exact = special(x[mine], ref.codes_of(pick(w.data), k), pick(w.scale), pick(w.zero) if zeros else None, group)
            check_special(y[mine], exact, (at, n, k, e))
        assert not y[len(of):].any()


@pytest.mark.parametrize("at", sorted(lr.PACKED), ids=str)
def test_float32_rows_lose_nothing(h, at):
    # 1 in one column of W and nothing elsewhere: that column of x bit for bit, whichever block, part of a block, strip or wave it lies in
    for counts, behind, n, k, group, kinds in lr.PACKED[at]:
        if 4 not in kinds:
            continue
        r = torch.Generator(device="cuda").manual_seed(n + k)
        w = weights(r, n, k, group, False, torch.float32, (len(counts),) if counts else ())
        m = sum(counts) + behind
        x = torch.randn((m, k), generator=r, device="cuda") * 10.0 ** torch.randint(-25, 30, (m, 1), generator=r, device="cuda")
        w.data.fill_(0x88)
        w.scale.fill_(1.0)
        for col in {0, k // 2, k // 128 * 128 - 1, k // 128 * 128, k - 1}:
            if not 0 <= col < k:
                continue
            w.data[..., col // 2] = 0x98 if col % 2 else 0x89
            y, of = product_of(h, x, w, counts)
            assert torch.equal(y[:len(of)], x[:len(of), col:col + 1].expand(-1, n)), (at, n, k, col)
            w.data[..., col // 2] = 0x88
