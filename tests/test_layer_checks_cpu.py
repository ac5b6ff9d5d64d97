"""What the router's choice, 4-bit weights and orthogonal updates refuse before anything is enqueued: no GPU is needed."""
import ctypes as C
import warnings

import pytest

torch = pytest.importorskip("torch")

from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

from test_abi_cpu import lib  # noqa: E402,F401
from test_scaled_checks_cpu import Nowhere, made  # noqa: E402

F32, I32, U8 = torch.float32, torch.int32, torch.uint8
ERR_ARG = 1


class Here(Nowhere):
    def choose_experts_workspace_bytes(self, *a):
        return 0

    def orthogonalize_workspace_bytes(self, *a):
        return 0


def packed_on(device, rows, cols, groups=(), group=32):
    from paper_2511_13778_amd import packed
    blocks = -(-cols // group)
    return packed.Packed(made(U8, device, *groups, rows, -(-cols // 32) * 16), made(F32, device, *groups, blocks, rows), None, cols=cols, group=group)


def choice_on(device, tokens, topk, experts, live=None):
    from paper_2511_13778_amd import experts as ex
    return ex.Choice(made(I32, device, tokens, topk), made(F32, device, tokens, topk), made(I32, device, experts), made(I32, device, 1), live=live)


@pytest.fixture()
def mode(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    with FakeTensorMode():
        yield


pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer")


def test_tensors_on_another_gpu(mode):
    from paper_2511_13778_amd import experts as ex, orthogonal, packed
    h = Here()
    calls = {
        "choose": (lambda s, l: ex.choose(h, s, 2, live=l), lambda d: made(F32, d, 5, 8), lambda d: made(torch.bool, d, 5)),
        "choose_backward": (lambda s, c, w, l: ex.choose_backward(h, s, c, w, l), lambda d: made(F32, d, 5, 8), lambda d: choice_on(d, 5, 2, 8),
                            lambda d: made(F32, d, 5, 2), lambda d: made(F32, d)),
        "choose_backward live": (lambda s, l: ex.choose_backward(h, s, choice_on("cuda:0", 5, 2, 8, live=l), None, 1.0), lambda d: made(F32, d, 5, 8),
                                 lambda d: made(torch.bool, d, 5)),
        "quantize": (lambda x: packed.quantize(h, x), lambda d: made(F32, d, 6, 64)),
        "unpack": (lambda w, o: packed.unpack(h, w, out=o), lambda d: packed_on(d, 6, 64), lambda d: made(F32, d, 6, 64)),
        "gemm": (lambda x, w, o: packed.gemm(h, x, w, out=o), lambda d: made(F32, d, 3, 64), lambda d: packed_on(d, 6, 64), lambda d: made(F32, d, 3, 6)),
        "gemm_grouped": (lambda x, w, f, o: packed.gemm_grouped(h, x, w, f, out=o), lambda d: made(F32, d, 3, 64), lambda d: packed_on(d, 6, 64, (2,)),
                         lambda d: made(I32, d, 3), lambda d: made(F32, d, 3, 6)),
        "orthogonalize": (lambda x, o: orthogonal.orthogonalize(h, x, out=o), lambda d: made(F32, d, 3, 64), lambda d: made(F32, d, 3, 64)),
    }
    for name, (call, *args) in calls.items():
        for odd in [*range(len(args)), None]:
            where = ["cuda:1" if odd in (i, None) else "cuda:0" for i in range(len(args))]
            with pytest.raises(ValueError):
                call(*(a(d) for a, d in zip(args, where)))
                pytest.fail("%s: %s" % (name, where))
        with pytest.raises(AssertionError, match="enqueued"):
            call(*(a("cuda:0") for a in args))


def test_lost_gradients_are_told(mode):
    from paper_2511_13778_amd import experts as ex, orthogonal, packed
    h, d = Here(), "cuda:0"
    x = made(F32, d, 6, 64)
    for call in (lambda x: ex.choose(h, x, 2), lambda x: packed.quantize(h, x), lambda x: packed.gemm(h, x, packed_on(d, 5, 64)),
                 lambda x: orthogonal.orthogonalize(h, x), lambda x: orthogonal.orthogonalize(h, x[None])):
        with pytest.warns(UserWarning, match="requires gradients"), pytest.raises(AssertionError, match="enqueued"):
            call(x.detach().requires_grad_())
        with warnings.catch_warnings():
            warnings.filterwarnings("error", message=".*requires gradients")
            with torch.no_grad(), pytest.raises(AssertionError, match="enqueued"):
                call(x.detach().requires_grad_())
            with pytest.raises(AssertionError, match="enqueued"):
                call(x)


def refused(call, *args):
    with pytest.raises((ValueError, TypeError)):
        call(*args)
        pytest.fail(str(args))


def test_choices_that_do_not_fit(mode):
    from paper_2511_13778_amd import experts as ex
    h, d = Here(), "cuda:0"
    s = made(F32, d, 5, 8)
    for topk in (0, -1, 9, 65):
        refused(lambda: ex.choose(h, s, topk))
    refused(lambda: ex.choose(h, made(F32, d, 5, 100), 65))
    for odd in (made(torch.float64, d, 5, 8), made(F32, d, 8), made(F32, d, 8, 5).T, made(F32, "cpu", 5, 8)):
        refused(lambda: ex.choose(h, odd, 2))
    for live in (made(torch.bool, d, 4), made(F32, d, 5), made(torch.bool, d, 5, 2)[:, 0], made(torch.bool, "cpu", 5)):
        refused(lambda: ex.choose(h, s, 2, live=live))
    c = choice_on(d, 5, 2, 8)
    refused(lambda: ex.choose_backward(h, made(F32, d, 4, 8), c, None, 1.0))
    refused(lambda: ex.choose_backward(h, made(F32, d, 5, 9), c, None, 1.0))            # counts of 8 experts
    for w in (made(F32, d, 5, 3), made(torch.bfloat16, d, 5, 2), made(F32, d, 2, 5).T):
        refused(lambda: ex.choose_backward(h, s, c, w))
    for loss in (made(F32, d, 2), made(torch.bfloat16, d), made(F32, "cpu")):
        refused(lambda: ex.choose_backward(h, s, c, None, loss))
    none = ex.Choice(c.ids, c.weights)
    refused(lambda: ex.choose_backward(h, s, none, None, 1.0))
    for ids, weights in ((c.ids[:4], c.weights), (c.ids.long(), c.weights), (c.ids, c.weights.double()), (c.ids.T.contiguous().T, c.weights)):
        refused(lambda: ex.choose_backward(h, s, ex.Choice(ids, weights), c.weights))


def test_packed_matrices_that_do_not_fit(mode):
    from paper_2511_13778_amd import orthogonal, packed
    h, d = Here(), "cuda:0"
    data, scale = made(U8, d, 6, 32), made(F32, d, 2, 6)
    packed.Packed(data, scale, cols=64, group=32)
    packed.Packed(data, scale, scale, cols=33, group=32)
    for bad in ((data, scale, None, 65, 32), (data, scale, None, 64, 16), (data, scale[:1], None, 64, 32), (data, scale[:, :5], None, 64, 32), (data.to(torch.int8), scale, None, 64, 32),
                (data, scale.double(), None, 64, 32), (data, scale, scale.half(), 64, 32), (data, scale, scale[:1], 64, 32), (data[None], scale, None, 64, 32),
                (data[:, :24], scale, None, 48, 32), (data, scale, None, -1, 32), (made(U8, d, 6, 64)[:, ::2], scale, None, 64, 32)):
        refused(lambda: packed.Packed(*bad[:3], cols=bad[3], group=bad[4]))
    refused(lambda: packed.empty(4, 64, group=48))
    for part in ("data", "scale", "zero", "cols", "group"):          # what the C ABI is given was looked at when the matrix was made
        with pytest.raises(AttributeError):
            setattr(packed.Packed(data, scale, cols=64, group=32), part, None)
    w, ws, x = packed_on(d, 6, 64), packed_on(d, 6, 64, (2,)), made(F32, d, 3, 64)
    for bad in (made(F32, d, 3, 63), made(torch.float64, d, 3, 64), made(F32, d, 64), made(F32, d, 64, 3).T):
        refused(lambda: packed.gemm(h, bad, w))
        refused(lambda: packed.quantize(h, bad)) if bad.shape != (3, 63) else None
    refused(lambda: packed.gemm(h, x, ws))
    refused(lambda: packed.gemm_grouped(h, x, ws, made(I32, d, 4)))
    refused(lambda: packed.gemm_grouped(h, x, ws, made(torch.int64, d, 3)))
    refused(lambda: packed.gemm(h, x, w, dtype=torch.float64))
    for out in (made(F32, d, 3, 5), made(torch.float64, d, 3, 6), made(F32, d, 6, 3).T):
        refused(lambda: packed.gemm(h, x, w, out=out))
        refused(lambda: packed.unpack(h, w, out=out))
    for bad in (made(torch.float64, d, 3, 4), made(F32, d, 4), made(F32, d, 2, 2, 3, 4), made(F32, d, 4, 3).T, made(F32, "cpu", 3, 4)):
        refused(lambda: orthogonal.orthogonalize(h, bad))
    refused(lambda: orthogonal.orthogonalize(h, x, out=made(F32, d, 64, 3)))
    refused(lambda: orthogonal.orthogonalize(h, x, out=made(torch.bfloat16, d, 3, 64)))


def test_c_entries_without_a_handle(lib):              # noqa: F811
    g, dll = lib
    w = g.oz_packed_t()
    assert C.sizeof(w) == 7 * 8 + 3 * 4 + 4
    assert dll.oz_choose_experts_workspace_bytes(None, 4, 4) == 0 and dll.oz_orthogonalize_workspace_bytes(None, 1, 4, 4, 0) == 0
    n = None
    assert dll.oz_choose_experts(n, n, 4, 4, 2, n, 4, 0, n, 1, n, n, n, n, n, n, n, 0) == ERR_ARG
    assert dll.oz_choose_experts_grad(n, n, 4, 4, 2, n, 4, 0, n, 1, n, n, n, n, n, n, 1.0, n, 4) == ERR_ARG
    assert dll.oz_pack4(n, n, 4, 4, n, 4, 0, 1, 0, C.byref(w)) == ERR_ARG and dll.oz_pack4(n, n, 4, 4, n, 4, 0, 1, 0, n) == ERR_ARG
    assert dll.oz_unpack4(n, n, 4, 4, n, 4, 0, 1, 0, C.byref(w)) == ERR_ARG and dll.oz_unpack4(n, n, 4, 4, n, 4, 0, 1, 0, n) == ERR_ARG
    assert dll.oz_packed_gemm(n, n, 0, n, 4, 4, 4, n, 4, 0, n, n, 4, 0) == ERR_ARG
    assert dll.oz_orthogonalize(n, n, 1, 4, 4, 0, n, 4, 16, n, 4, 16, 5, 1.0, 0.0, 0.0, 0.0, n, 0) == ERR_ARG
