"""A layer of experts through all of the 8-bit and routing calls: outputs and gradients against the layer in 64 bits.

An element in e4m3 is off by at most 2^-4 of itself, evenly spread, so by less than 2^-4 / sqrt(3) = 3.6 % in the root mean square, in
e5m2 by twice that.  Independent errors of a product's two operands add in squares, and every product passes its own on: y has two
products in a row, four such errors, 7.2 %; dw2 one of e5m2 with what y's first product gives, 9.5 %; dw1 and dx have one more
product of e5m2 and e4m3 in front of theirs, 12.5 %.  2 % more for silu and the 16-bit results in between."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def off(got, exact):
    return ((got.double() - exact).norm() / exact.norm()).item()


@pytest.mark.parametrize("scale", [torch.uint8, torch.float32])
def test_layer_and_its_gradients(scale):
    from paper_2511_13778_amd import experts as ex, ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    h = g.Handle(0)
    r = torch.Generator(device="cuda").manual_seed(5)
    tokens, width, inner, experts, topk = 300, 260, 390, 6, 2
    w1, w2 = (torch.randn(s, generator=r, device="cuda") * s[-1] ** -0.5 for s in ((experts, inner, width), (experts, width, inner)))
    x, dy = (torch.randn((tokens, width), generator=r, device="cuda").bfloat16() for _ in range(2))
    ids = torch.rand((tokens, experts - 1), generator=r, device="cuda").topk(topk, dim=1).indices      # the last expert gets nothing
    ids[torch.rand(ids.shape, generator=r, device="cuda") < 0.05] = -1
    p = torch.rand((tokens, topk), generator=r, device="cuda")
    layer = ex.ExpertLayer(h, w1, w2, scale)
    y, kept = layer.forward(x, ids, p)
    dx, dp, dw1, dw2 = layer.backward(dy, kept)
    again = layer.backward(dy, kept, dw1.clone(), dw2.clone())
    assert torch.equal(layer.serve(x, ids, p), y)

    leaves = [t.double().requires_grad_() for t in (x, p, w1, w2)]
    ex_, ep, e1, e2 = leaves
    e = ids.clamp(min=0)
    hidden = torch.nn.functional.silu((e1[e] @ ex_.unsqueeze(1).unsqueeze(3)).squeeze(3))
    ey = ((e2[e] @ hidden.unsqueeze(3)).squeeze(3) * (ep * (ids >= 0)).unsqueeze(2)).sum(1)
    ey.backward(dy.double())
    for name, got, exact, bound in (("y", y, ey, 0.092), ("dweights", dp, ep.grad, 0.092), ("dw2", dw2, e2.grad, 0.115), ("dw1", dw1, e1.grad, 0.145),
                                    ("dx", dx, ex_.grad, 0.145)):
        assert off(got, exact) < bound, (name, off(got, exact))
    assert not dw1[experts - 1].any() and not dw2[experts - 1].any()
    for a, b in ((again[2], dw1), (again[3], dw2)):            # added to what is there, rounded once
        assert torch.allclose(a, 2 * b, rtol=2 ** -22, atol=1e-6)
    h.close()
