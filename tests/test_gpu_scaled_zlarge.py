"""Matrices of more than 2^32 bytes and elements, through the quantiser, the products and the routing.  Their rows repeat, so that the first ones,
checked elsewhere, say what the others are."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

COPIES, BASE, WIDE = 8200, 128, 4224          # 1 049 600 rows of 4224: 4.43e9
ROWS = COPIES * BASE


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()
    torch.cuda.empty_cache()


def repeated(base):
    out = torch.empty((COPIES, *base.shape), dtype=base.dtype, device="cuda")
    out.copy_(base.unsqueeze(0).expand_as(out))
    return out.view(-1, base.shape[1])


def all_like_the_first(t, first):
    """Rows of t, `first` over and over; in pieces, because comparing takes memory."""
    return all(torch.equal(part, first.unsqueeze(0).expand_as(part)) for part in t.view(COPIES, *first.shape).split(1025))


def test_quantise_and_multiply(h):
    from paper_2511_13778_amd import scaled
    assert ROWS * WIDE > 1 << 32
    base = torch.randn((BASE, WIDE), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    few, few_t = scaled.quantize(h, base, which="both")
    x = repeated(base)
    a, t = scaled.quantize(h, x, which="both")
    assert torch.equal(scaled.quantize(h, x).data.view(torch.uint8)[-BASE:], few.data.view(torch.uint8))
    del x
    assert all_like_the_first(a.data.view(torch.uint8), few.data.view(torch.uint8)) and all_like_the_first(a.scales(), few.scales())
    for part in t.data.view(torch.uint8).view(WIDE, COPIES, BASE).split(256):          # columns repeat
        assert torch.equal(part, part[:, :1].expand_as(part))
    assert torch.equal(t.data.view(torch.uint8)[:, -BASE:], few_t.data.view(torch.uint8)) and torch.equal(t.scales()[:, -1:], few_t.scales())
    b = scaled.quantize(h, torch.randn((48, WIDE), device="cuda"), block_rows=128)
    want = scaled.gemm(h, few, b, dtype=torch.float32)
    got = scaled.gemm(h, a, b, dtype=torch.float32)
    # tiles of other sizes add in another order
    assert all_like_the_first(got, got[:BASE]) and (got[-BASE:] - want).abs().max() <= 1e-5 * want.abs().max()
    # rows in groups, the last ones past 2^32 bytes
    offsets = torch.tensor([0, 5, ROWS - 200, ROWS - 100, ROWS], dtype=torch.int32, device="cuda")
    w = scaled.quantize(h, torch.randn((4, 48, WIDE), device="cuda"), block_rows=128)
    got = scaled.gemm_grouped(h, a, w, offsets, dtype=torch.float32)
    for lo, hi, g in ((0, 5, 0), (ROWS - 200, ROWS - 100, 2), (ROWS - 100, ROWS, 3)):
        rows = scaled.Scaled(a.data[lo:hi], a.scale[lo:hi], WIDE)
        alone = scaled.gemm(h, rows, scaled.Scaled(w.data[g], w.scale[g], WIDE, 128), dtype=torch.float32)
        assert (got[lo:hi] - alone).abs().max() <= 1e-5 * alone.abs().max()


def test_results_past_32_bits(h):
    from paper_2511_13778_amd import scaled
    r = torch.Generator(device="cuda").manual_seed(2)
    base = scaled.quantize(h, torch.randn((BASE, 256), generator=r, device="cuda"))
    a = scaled.Scaled(repeated(base.data.view(torch.uint8)).view(torch.float8_e4m3fn), repeated(base.scale), 256)
    b = scaled.quantize(h, torch.randn((WIDE, 256), generator=r, device="cuda"), block_rows=128)
    c = scaled.gemm(h, a, b)
    want = scaled.gemm(h, base, b)
    assert c.numel() > 1 << 32
    assert all_like_the_first(c, c[:BASE]) and (c[-BASE:].float() - want.float()).abs().max() <= 2.0 ** -7 * want.abs().max().float()


def test_routed_rows(h):
    from paper_2511_13778_amd import experts as ex
    r = torch.Generator(device="cuda").manual_seed(3)
    tokens = ROWS // 2
    ids = torch.randint(0, 7, (tokens, 2), generator=r, device="cuda")
    routing = ex.sort_tokens(h, ids, 7)
    x = torch.empty((COPIES // 2, BASE, WIDE), dtype=torch.float16, device="cuda")
    x.copy_(torch.randn((BASE, WIDE), generator=r, device="cuda").half().unsqueeze(0).expand_as(x))
    x = x.view(tokens, WIDE)
    x[:, 0] = (torch.arange(tokens, device="cuda") % 2000).half()                     # tells tokens apart
    xs = ex.gather(h, x, routing)
    assert xs.numel() > 1 << 32
    place = routing.place.long()
    for part in range(0, tokens, 65600):
        s = slice(part, part + 65600)
        assert torch.equal(xs[place[s, 0]], x[s]) and torch.equal(xs[place[s, 1]], x[s])
    assert torch.equal(ex.combine(h, xs, routing), x * 2)                             # two choices, exact in 16 bits
    dxs, dw = ex.combine_backward(h, x, xs, routing, torch.ones((tokens, 2), device="cuda"))
    assert torch.equal(dxs, xs)
    last = x[-500:].double().square().sum(1, keepdim=True)
    assert ((dw[-500:].double() - last).abs() <= WIDE * 2.0 ** -24 * last).all()
