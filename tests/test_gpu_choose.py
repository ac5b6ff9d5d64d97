"""The router's choice, its balance loss and their gradient, against loops in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402

F = 2.0 ** -24
# An exponential below 2^-126 is taken as 0 (the hardware's exp2 has no numbers below that), and so is off by less than 2^-126, times what it is
# multiplied by next, which is below 16 here; no relative bound covers that.
LEAST = 2.0 ** -126


@pytest.fixture(scope="module")
def h():
    from paper_2511_13778_amd import ozdgemm as g
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
    handle = g.Handle(0)
    yield handle
    handle.close()


def scores_of(seed, tokens, experts, dtype, spread=2.0):
    r = torch.Generator().manual_seed(seed)
    return (torch.randn((tokens, experts), generator=r) * spread + torch.randn((experts,), generator=r)).to(dtype)


def close(got, exact, bound, what):
    err = (got.double().cpu() - exact).abs()
    assert got.shape == exact.shape and (err <= bound).all(), (what, (err - bound).max().item(), err.max().item())


def check(h, scores, topk, live=None, normalize=True, dloss=0.7, view=None):
    """Everything that there is of one batch.  Relative errors: a quotient of exponentials, each of a difference that is off by half a step of the
    spread, with 2 steps of exp; sums over up to 32 values of a lane and 6 folds."""
    from paper_2511_13778_amd import experts as ex
    tokens, experts = scores.shape
    ids, w, p, counts, counted = ref.choose(scores, topk, live, normalize)
    finite = scores.double()[scores.double().isfinite()]
    spread = (finite.max() - finite.min()).item() if finite.numel() else 0.0
    rel = (2 * spread + 2 * 4 + 40) * F
    d_live = None if live is None else live.cuda()
    x = scores.cuda() if view is None else view(scores)
    c = ex.choose(h, x, topk, live=d_live, normalize=normalize)
    assert torch.equal(c.ids.cpu().long(), ids)
    close(c.weights, w, rel * w + LEAST, "weights")
    assert torch.equal(c.counts.cpu().long(), counts) and c.counted.item() == counted
    shares, loss, f = ref.balance(p, counts, counted)
    rel_sum = rel + (tokens / 8192 + 24) * F
    close(c.shares, shares, rel_sum * shares + LEAST, "shares")
    close(c.loss, loss, rel_sum * loss + LEAST * experts, "loss")
    plain = ex.choose(h, x, topk, live=d_live, normalize=normalize, balance=False)
    assert torch.equal(plain.ids, c.ids) and torch.equal(plain.weights, c.weights) and plain.loss is None
    r = torch.Generator().manual_seed(1)
    dw = torch.randn((tokens, topk), generator=r)
    for weights, dl in ((dw, dloss), (dw, None), (None, dloss)):
        exact, size = ref.choose_grad(ids, w, p, f, counted, (dw if weights is not None else 0 * dw).double(), dl, normalize)
        d = ex.choose_backward(h, x, c, None if weights is None else weights.cuda(), dl)
        assert d.dtype == scores.dtype
        close(d, exact, (2 * rel + (topk + 16) * F) * size + ref.rounded(exact, scores.dtype) + 16 * LEAST, "dscores")
    return c


# experts around each width of a lane's part and of a token's lanes
SIZES = [(1, 1, 1), (1, 2, 1), (3, 5, 5), (24, 16, 4), (33, 17, 2), (17, 32, 4), (40, 60, 6), (100, 64, 8), (16, 65, 1), (50, 128, 8), (19, 129, 3), (70, 256, 8), (9, 257, 5),
         (30, 384, 6), (5, 512, 64), (7, 513, 33), (6, 1000, 64), (4, 1024, 17), (2, 64, 64), (3, 30, 30)]


@pytest.mark.parametrize("tokens,experts,topk", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("normalize", [True, False])
def test_sizes(h, tokens, experts, topk, dtype, normalize):
    check(h, scores_of(tokens * experts + topk, tokens, experts, dtype), topk, normalize=normalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_many_tokens(h, dtype):
    # more tokens than one pass of all workgroups takes
    check(h, scores_of(7, 20011, 24, dtype), 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_ties_go_to_the_lowest(h, dtype):
    x = torch.zeros((40, 130))
    x[10:20] = torch.arange(130) // 7 % 3
    x[20:30, ::2] = -0.0                      # equal to +0
    x[30:, 64:] = 1.0
    check(h, x.to(dtype), 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("normalize", [True, False])
def test_padding_and_experts_that_are_not_there(h, dtype, normalize):
    x = scores_of(3, 60, 40, dtype)
    live = torch.rand(60, generator=torch.Generator().manual_seed(2)) < 0.6
    live[4:20] = True
    x[5] = float("-inf")                      # nobody
    x[6, 1:] = float("-inf")                  # one
    x[7, 3:] = float("-inf")                  # fewer than are asked for
    x[8, ::2] = float("-inf")
    c = check(h, x, 4, live, normalize)
    assert (c.ids[5] == -1).all() and c.ids[7].tolist()[3] == -1
    dead = (~live).nonzero()[:, 0]
    x[dead] = float("nan")
    x[dead[::2]] = float("inf")
    got = check(h, x, 4, live, normalize)
    assert torch.equal(got.ids, c.ids) and torch.equal(got.weights, c.weights) and torch.equal(got.loss, c.loss)
    check(h, x, 4, torch.zeros(60, dtype=torch.bool), normalize)          # nobody at all
    check(h, x[:0], 4, None, normalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_not_a_number(h, dtype):
    from paper_2511_13778_amd import experts as ex
    x = scores_of(4, 8, 20, dtype)
    x[2, 7] = x[2, 11] = float("nan")
    x[5, 3] = float("inf")
    x[6, 4] = -float("nan")
    c = ex.choose(h, x.cuda(), 3)
    ids = ref.choose(x, 3)[0]
    assert torch.equal(c.ids.cpu().long(), ids) and ids[2].tolist()[:2] == [7, 11] and ids[6, 0] == 4 and ids[5, 0] == 3
    bad = c.weights.isnan().any(1).cpu()
    assert bad.tolist() == [False, False, True, False, False, True, True, False]
    assert c.loss.isnan() and c.shares.isnan().all()
    d = ex.choose_backward(h, x.cuda(), c, torch.ones((8, 3), device="cuda")).cpu()
    assert d.isnan().any(1).tolist() == bad.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_far_scores(h, dtype):
    # softmax without overflow, and experts whose probability is nothing
    x = scores_of(5, 30, 48, dtype, spread=60.0)
    check(h, x, 4)
    check(h, x, 4, normalize=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_strides_and_alignment(h, dtype):
    x = scores_of(6, 37, 45, dtype)

    def inside(ld, start):
        def view(s):
            big = torch.full((s.shape[0] * ld + start + 64,), float("nan"), dtype=dtype, device="cuda")
            v = big[start:start + s.shape[0] * ld].view(s.shape[0], ld)[:, :s.shape[1]]
            v.copy_(s)
            return v
        return view
    for ld, start in ((45, 1), (46, 3), (47, 0), (64, 5)):
        check(h, x, 5, view=inside(ld, start))


def test_gradient_by_differences(h):
    from paper_2511_13778_amd import experts as ex
    x = scores_of(8, 6, 10, torch.float32).double()
    dw = torch.randn((6, 3), generator=torch.Generator().manual_seed(9)).double()
    for normalize in (True, False):
        def value(s):
            ids, w, p, counts, counted = ref.choose(s, 3, None, normalize)
            return ids, (w * dw).sum() + 0.5 * ref.balance(p, counts, counted)[1]
        ids, _ = value(x)
        c = ex.choose(h, x.float().cuda(), 3, normalize=normalize)
        d = ex.choose_backward(h, x.float().cuda(), c, dw.float().cuda(), 0.5).cpu()
        step = 1e-5
        for t in range(6):
            for e in range(10):
                up, down = x.clone(), x.clone()
                up[t, e] += step
                down[t, e] -= step
                (i, a), (j, b) = value(up), value(down)
                assert torch.equal(i, ids) and torch.equal(j, ids)
                # third derivatives are below 10: the difference is off by 10 step^2, the inputs by their rounding to 32 bits
                assert abs((a - b).item() / (2 * step) - d[t, e].item()) < 1e-5


def test_loss_gradient_on_the_gpu_and_counts_of_several(h):
    from paper_2511_13778_amd import experts as ex
    x = scores_of(10, 300, 16, torch.float32)
    c = ex.choose(h, x.cuda(), 2)
    scalar = torch.tensor(0.25, device="cuda")
    assert torch.equal(ex.choose_backward(h, x.cuda(), c, None, scalar), ex.choose_backward(h, x.cuda(), c, None, 0.25))
    # another GPU's choices added in: its f_e, this one's mean
    ids, w, p, counts, counted = ref.choose(x, 2)
    other = torch.arange(16) * 40
    c.counts = (c.counts.cpu() + other).to(torch.int32).cuda()
    f = (counts + other).double() / (counts + other).sum()
    exact, size = ref.choose_grad(ids, w, p, f, counted, torch.zeros((300, 2)).double(), 0.25, True)
    close(ex.choose_backward(h, x.cuda(), c, None, 0.25), exact, 200 * F * size + ref.rounded(exact, torch.float32), "dscores")


def test_same_bits_again_and_on_another_stream(h):
    from paper_2511_13778_amd import experts as ex
    x = scores_of(11, 30000, 60, torch.bfloat16).cuda()
    dw = torch.randn((30000, 6), device="cuda")
    a = ex.choose(h, x, 6)
    da = ex.choose_backward(h, x, a, dw, 0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = ex.choose(h, x, 6)
        db = ex.choose_backward(h, x, b, dw, 0.1)
    torch.cuda.synchronize()
    for m, n in ((a.ids, b.ids), (a.weights, b.weights), (a.counts, b.counts), (a.shares, b.shares), (a.loss, b.loss), (da, db)):
        assert torch.equal(m, n)


def test_captured_and_replayed_with_other_inputs(h):
    from paper_2511_13778_amd import experts as ex
    x = scores_of(12, 500, 64, torch.float32).cuda()
    dw = torch.randn((500, 4), device="cuda")

    def step():
        c = ex.choose(h, x, 4)
        return c.ids, c.weights, c.counts, c.shares, c.loss, ex.choose_backward(h, x, c, dw, 0.3)
    step()
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    with torch.cuda.graph(other):
        got2 = step()
    for seed in range(4):
        x.copy_(scores_of(20 + seed, 500, 64, torch.float32))
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(step(), got, got2):
            assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("tokens,experts,topk", [(20, 200, 9), (11, 256, 40), (13, 250, 8), (37, 131, 8), (9, 255, 64), (300, 9, 9)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("normalize", [True, False])
def test_more_of_a_lane_than_half(h, tokens, experts, topk, dtype, normalize):
    # chosen experts that are neighbours: all of one lane's
    x = scores_of(11, tokens, experts, dtype)
    x[::2, experts // 3:experts // 3 + topk] += 20.0
    check(h, x, topk, normalize=normalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("experts", [20, 250, 500])
def test_the_types_largest_and_zeros_of_both_signs(h, dtype, experts):
    from paper_2511_13778_amd import experts as ex
    big = torch.finfo(dtype).max
    x = torch.zeros((6, experts), dtype=dtype)
    x[:, 1::2] = -0.0                          # equal: the lowest expert first
    x[1, 5:9], x[1, 11] = big, -big
    x[2] = -big                                # above -infinity
    x[3, 7:] = float("-inf")
    x[4, 3], x[4, 12] = -big, big
    x[5] = big
    for normalize in (True, False):
        c = ex.choose(h, x.cuda(), 8, normalize=normalize)
        ids, w, p, counts, counted = ref.choose(x, 8, None, normalize)
        assert torch.equal(c.ids.cpu().long(), ids) and counted == 6
        # differences are zero or further than any exponential reaches: shares are quotients of whole numbers
        close(c.weights, w, 4 * F * w, "weights")
        dw = torch.randn((6, 8), generator=torch.Generator().manual_seed(1))
        shares, loss, f = ref.balance(p, counts, counted)
        exact, size = ref.choose_grad(ids, w, p, f, counted, dw.double(), 0.5, normalize)
        d = ex.choose_backward(h, x.cuda(), c, dw.cuda(), 0.5)
        close(d, exact, 64 * F * size + ref.rounded(exact, dtype) + 16 * LEAST, "dscores")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_tokens_and_nothing_live(h, dtype):
    from paper_2511_13778_amd import experts as ex
    for tokens, live in ((0, None), (5, torch.zeros(5, dtype=torch.bool, device="cuda"))):
        x = torch.full((tokens, 200), float("nan"), device="cuda", dtype=dtype)
        c = ex.choose(h, x, 8, live=live)
        assert (c.ids == -1).all() and not c.weights.any() and not c.counts.any() and c.counted.item() == 0 and not c.shares.any() and c.loss.item() == 0
        d = ex.choose_backward(h, x, c, torch.ones((tokens, 8), device="cuda"), 1.0)
        assert d.shape == x.shape and not d.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("experts,topk", [(1, 1), (20, 3), (200, 8), (300, 20)])
@pytest.mark.parametrize("normalize", [True, False])
def test_not_a_number_in_all_of_a_row(h, dtype, experts, topk, normalize):
    # NaN in every score, NaN beside -infinity alone, one NaN and one +infinity among numbers: probabilities that are NaN, so all of the token's gradient is
    from paper_2511_13778_amd import experts as ex
    nan, inf = float("nan"), float("inf")
    x = scores_of(13, 9, experts, dtype)
    x[1] = nan
    x[2] = -inf
    x[2, experts // 2] = nan
    x[3] = -nan
    x[4, experts - 1] = nan
    x[5, experts // 3] = inf
    x[6] = -inf                                # nobody to be had: padding, not NaN
    x[7, :experts // 2] = -inf
    bad = torch.tensor([False, True, True, True, True, True, False, False, False])
    c = ex.choose(h, x.cuda(), topk, normalize=normalize)
    ids, w = ref.choose(x, topk, None, normalize)[:2]
    assert torch.equal(c.ids.cpu().long(), ids)
    assert torch.equal(c.weights.isnan().any(1).cpu(), bad) and c.loss.isnan() and c.shares.isnan().all() and c.counted.item() == 8
    dw = torch.randn((9, topk), generator=torch.Generator().manual_seed(1)).cuda()
    for weights, dloss in ((dw, 0.5), (dw, None), (None, 0.5)):
        d = ex.choose_backward(h, x.cuda(), c, weights, dloss).cpu()
        assert d[bad].isnan().all(), (weights is None, dloss, d.isnan().sum(1).tolist())
        assert d[~bad].isfinite().all() and not d[6].any() and not d[7, :experts // 2].any()
    # a token that is not live may have any scores
    live = torch.ones(9, dtype=torch.bool)
    live[bad] = False
    c = ex.choose(h, x.cuda(), topk, live=live.cuda(), normalize=normalize)
    for weights, dloss in ((dw, 0.5), (dw, None), (None, 0.5)):
        assert not ex.choose_backward(h, x.cuda(), c, weights, dloss).cpu()[bad].any()


def test_results_hold_no_workspace(h):
    from paper_2511_13778_amd import experts as ex
    x = scores_of(14, 20000, 256, torch.bfloat16).cuda()
    need = h.choose_experts_workspace_bytes(20000, 256)
    assert need > 100000
    c = ex.choose(h, x, 4)
    for part in (c.counts, c.counted, c.shares, c.loss):
        assert part.untyped_storage().nbytes() <= 4 * (2 * 256 + 64)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    kept = [ex.choose(h, x, 4).loss for _ in range(50)]
    assert torch.cuda.memory_allocated() - before < 50 * 8192 and all(torch.equal(a, kept[0]) for a in kept)
