"""Ends of the ranges of sizes and values: rows without columns, through the public calls."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


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
