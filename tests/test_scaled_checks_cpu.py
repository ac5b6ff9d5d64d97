"""What the calls on tensors refuse before anything is enqueued, with tensors that have a device but no memory: no GPU is needed."""
import pytest

torch = pytest.importorskip("torch")

from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

E4M3 = torch.float8_e4m3fn


class Nowhere:
    """A handle of cuda:0 whose calls are not allowed to be reached."""
    device = 0

    def call(self, *a):
        raise AssertionError("enqueued")

    def scaled_gemm_workspace_bytes(self, *a):
        return 0

    def sort_tokens_workspace_bytes(self, *a):
        return 0


def made(kind, device, *shape):
    return torch.empty(shape, dtype=kind, device=device)


def routing_on(device):
    from paper_2511_13778_amd import experts as ex
    return ex.Routing(made(torch.int32, device, 4), made(torch.int32, device, 6), made(torch.int32, device, 3, 2), 2)


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
def test_tensors_on_another_gpu(monkeypatch):
    # each argument in turn on the second GPU, the others on the handle's; all of them there; and none, which goes through
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    from paper_2511_13778_amd import experts as ex, scaled
    h, f32, i32 = Nowhere(), torch.float32, torch.int32

    def matrix(device, rows, groups=()):
        return scaled.Scaled(made(E4M3, device, *groups, rows, 128), made(torch.uint8, device, *groups, rows, 4))
    calls = {
        "quantize": (lambda x, o: scaled.quantize(h, x, which="columns", offsets=o), lambda d: made(f32, d, 6, 128), lambda d: made(i32, d, 4)),
        "quantize routed": (lambda x, r: scaled.quantize(h, x, routing=r), lambda d: made(f32, d, 3, 128), routing_on),
        "gemm": (lambda a, b, c: scaled.gemm(h, a, b, out=c), lambda d: matrix(d, 6), lambda d: matrix(d, 5), lambda d: made(f32, d, 6, 5)),
        "gemm_grouped": (lambda a, b, o, c: scaled.gemm_grouped(h, a, b, o, out=c), lambda d: matrix(d, 6), lambda d: matrix(d, 5, (3,)), lambda d: made(i32, d, 4),
                         lambda d: made(f32, d, 6, 5)),
        "gemm_grouped_k": (lambda a, b, o, c: scaled.gemm_grouped_k(h, a, b, o, out=c), lambda d: matrix(d, 6), lambda d: matrix(d, 5), lambda d: made(i32, d, 4),
                           lambda d: made(f32, d, 3, 6, 5)),
        "sort_tokens": (lambda i: ex.sort_tokens(h, i, 3), lambda d: made(torch.int64, d, 3, 2)),
        "gather": (lambda x, r, y: ex.gather(h, x, r, out=y), lambda d: made(f32, d, 3, 8), routing_on, lambda d: made(f32, d, 6, 8)),
        "combine": (lambda x, r, w, y: ex.combine(h, x, r, w, out=y), lambda d: made(f32, d, 6, 8), routing_on, lambda d: made(f32, d, 3, 2), lambda d: made(f32, d, 3, 8)),
        "combine_backward": (lambda dy, x, r, w: ex.combine_backward(h, dy, x, r, w), lambda d: made(f32, d, 3, 8), lambda d: made(f32, d, 6, 8), routing_on,
                             lambda d: made(f32, d, 3, 2)),
    }
    with FakeTensorMode():
        for name, (call, *args) in calls.items():
            for odd in [*range(len(args)), None]:
                where = ["cuda:1" if odd in (i, None) else "cuda:0" for i in range(len(args))]
                with pytest.raises(ValueError):
                    call(*(a(d) for a, d in zip(args, where)))
                    pytest.fail("%s: %s" % (name, where))
            with pytest.raises(AssertionError, match="enqueued"):
                call(*(a("cuda:0") for a in args))
        for odd in range(3):
            d = ["cuda:1" if i == odd else "cuda:0" for i in range(3)]
            with pytest.raises(ValueError):
                ex.Routing(made(i32, d[0], 4), made(i32, d[1], 6), made(i32, d[2], 3, 2), 2)


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
def test_lost_gradients_are_told(monkeypatch):
    # every floating-point argument that a gradient would flow to; not where none is recorded anyway
    import warnings
    from paper_2511_13778_amd import experts as ex, scaled
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    h, f32, d = Nowhere(), torch.float32, "cuda:0"
    with FakeTensorMode():
        r = routing_on(d)
        xs, x, w = made(f32, d, 6, 8), made(f32, d, 3, 8), made(f32, d, 3, 2)
        calls = [(lambda x: scaled.quantize(h, x), x), (lambda x: scaled.quantize(h, x, which="both", routing=r), x), (lambda x: ex.gather(h, x, r), x),
                 (lambda xs, w: ex.combine(h, xs, r, w), xs, w), (lambda dy, xs, w: ex.combine_backward(h, dy, xs, r, w), x, xs, w)]
        for call, *args in calls:
            for asked in range(len(args)):
                given = [a.detach().requires_grad_(i == asked) for i, a in enumerate(args)]
                with pytest.warns(UserWarning, match="requires gradients") as seen, pytest.raises(AssertionError, match="enqueued"):
                    call(*given)
                assert all(s.filename == __file__ for s in seen if "requires gradients" in str(s.message))
                with warnings.catch_warnings():
                    warnings.filterwarnings("error", message=".*requires gradients")
                    with torch.no_grad(), pytest.raises(AssertionError, match="enqueued"):
                        call(*given)
                    with pytest.raises(AssertionError, match="enqueued"):
                        call(*args)
