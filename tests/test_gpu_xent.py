"""Cross entropy over a vocabulary against its definition in 64 bits.

Bounds, from the arithmetic: a product of bf16 numbers is exact in fp32, one of fp32 numbers is off by 2^-21 of it at most (binary16
planes); adding n products in fp32 loses at most n 2^-24 of the sum of their magnitudes.  In the bf16 path G and the outputs are rounded
once each (bf16 has eight bits: 2^-8 at most)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

IGNORE = -100
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# rows, vocabulary, width: one and less than a tile, each side of the tiles' edges, odd widths, several tiles
SHAPES = [(1, 1, 1), (1, 7, 3), (3, 130, 17), (16, 300, 64), (17, 511, 50), (31, 1025, 130), (64, 128, 256), (65, 700, 72), (128, 257, 64),
          (129, 513, 331), (257, 2049, 192), (300, 640, 65)]


@pytest.fixture(scope="module")
def ops():
    from paper_2204_00595_amd import autograd, binding
    return autograd, binding


def inputs(rows, vocab, width, dtype, seed=0, ignored=0.0, sharp=2.0):
    gen = torch.Generator().manual_seed(1000 * rows + vocab + width + seed)
    x = torch.randn((rows, width), generator=gen).to(DTYPES[dtype])
    W = (torch.randn((vocab, width), generator=gen) * (sharp / width ** 0.5)).to(DTYPES[dtype])
    target = torch.randint(0, vocab, (rows,), generator=gen)
    target[torch.rand((rows,), generator=gen) < ignored] = IGNORE
    return x, W, target


class Exact:
    """Loss, gradients and the bounds on them, in 64 bits."""

    def __init__(self, x, W, target, g, dtype):
        x, W, g = x.double(), W.double(), g.double()
        rows, width = x.shape
        counts = target != IGNORE
        x = torch.where(counts[:, None], x, 0.0)
        hit = torch.where(counts, target, 0)
        logits, size = x @ W.t(), x.abs() @ W.abs().t()
        self.lse = torch.logsumexp(logits, 1)
        self.loss = torch.where(counts, self.lse - logits.gather(1, hit[:, None])[:, 0], 0.0)
        one = torch.zeros_like(logits).scatter_(1, hit[:, None], 1.0)
        g = torch.where(counts, g, 0.0)[:, None]
        p = (logits - self.lse[:, None]).exp()
        G, mag = (p - one) * g, (p + one) * g.abs()
        self.dx, self.dW = G @ W, G.t() @ x
        bits = 2.0 ** -21 if dtype == "f32" else 0.0
        off = (bits + width * 2.0 ** -24) * size.amax() + 2.0 ** -21 * self.lse.abs().amax()  # of a logit less its lse
        self.row_bound = 2 * off + 2.0 ** -22 * (1 + self.lse.abs().amax())
        half = 0.0 if dtype == "f32" else 2.0 ** -8
        off = half + bits + 4 * off + 2.0 ** -20
        self.dx_bound = (off + W.shape[0] * 2.0 ** -24) * (mag @ W.abs()) + half * self.dx.abs() * 1.01 + 1e-30
        self.dW_bound = (off + rows * 2.0 ** -24) * (mag.t() @ x.abs()) + half * self.dW.abs() * 1.01 + 1e-30


def within(got, want, bound, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    worst = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
    assert worst <= 1.0, (what, worst)


def run(binding, x, W, target, g, **more):
    xd, Wd, td = x.cuda(), W.cuda(), target.cuda()
    loss, lse = binding.monarch_xent_fwd(xd, Wd, td)
    dx, dW = binding.monarch_xent_bwd(xd, Wd, td, lse, g.cuda(), **more)
    return loss, lse, dx, dW


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_loss_and_gradients(ops, shape, dtype):
    x, W, target = inputs(*shape, dtype, ignored=0.3 if shape[0] > 2 else 0.0)
    g = torch.rand((shape[0],), generator=torch.Generator().manual_seed(7)) - 0.3
    want = Exact(x, W, target, g, dtype)
    loss, lse, dx, dW = run(ops[1], x, W, target, g)
    within(loss, want.loss, want.row_bound, "loss")
    counts = target != IGNORE
    within(lse.cpu()[counts], want.lse[counts], want.row_bound, "lse")
    assert dx.dtype == x.dtype and dW.dtype == W.dtype
    within(dx, want.dx, want.dx_bound, "dx")
    within(dW, want.dW, want.dW_bound, "dW")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_short_workspace_takes_the_vocabulary_in_pieces(ops, dtype):
    _, binding = ops
    code = 0 if dtype == "f32" else 1
    rows, vocab, width = 200, 1500, 96
    x, W, target = inputs(rows, vocab, width, dtype, ignored=0.1)
    g = torch.ones(())
    want = Exact(x, W, target, torch.ones(rows), dtype)
    need = binding.monarch_xent_bwd_workspace_bytes(rows, vocab, width, code)

    def serves(bytes_):
        try:
            return run(binding, x, W, target, g, workspace=torch.empty(bytes_, dtype=torch.uint8, device="cuda"))
        except binding.MonarchError as e:
            assert "workspace" in str(e)
            return None
    refused, least = 0, need      # the shortest that serves
    while least - refused > 256:
        middle = (refused + least) // 2
        refused, least = (refused, middle) if serves(middle) else (middle, least)
    assert least < need
    for bytes_ in (need, (need + least) // 2, least):
        _, _, dx, dW = serves(bytes_)
        within(dx, want.dx, want.dx_bound, "dx")
        within(dW, want.dW, want.dW_bound, "dW")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 150])
def test_what_ignored_rows_hold_has_no_influence(ops, dtype, rows):
    x, W, target = inputs(rows, 400, 80, dtype)
    target[::3] = IGNORE
    g = torch.ones(rows)
    want = Exact(x, W, target, g, dtype)
    x[0] = float("nan")
    x[3, 5] = float("inf")
    loss, _, dx, dW = run(ops[1], x, W, target, g)
    within(loss, want.loss, want.row_bound, "loss")
    within(dx, want.dx, want.dx_bound, "dx")
    within(dW, want.dW, want.dW_bound, "dW")
    assert (dx[::3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_row_counts(ops, dtype):
    autograd, binding = ops
    x, W, target = inputs(70, 300, 64, dtype, ignored=1.0)
    assert (target == IGNORE).all()
    xd, Wd = x.cuda().requires_grad_(), W.cuda().requires_grad_()
    for reduction in ("mean", "sum", "none"):
        loss = autograd.vocab_cross_entropy(xd, Wd, target.cuda(), reduction=reduction)
        dx, dW = torch.autograd.grad(loss.sum(), (xd, Wd))
        assert (loss == 0).all() and (dx == 0).all() and (dW == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(ops, dtype):
    autograd, binding = ops
    x = torch.empty((0, 48), device="cuda", dtype=DTYPES[dtype], requires_grad=True)
    W = torch.ones((30, 48), device="cuda", dtype=DTYPES[dtype], requires_grad=True)
    target = torch.empty((0,), dtype=torch.int64, device="cuda")
    for reduction in ("mean", "sum"):
        loss = autograd.vocab_cross_entropy(x, W, target, reduction=reduction)
        dx, dW = torch.autograd.grad(loss, (x, W))
        assert loss.item() == 0 and dx.shape == x.shape and (dW == 0).all()
    assert autograd.vocab_cross_entropy(x, W, target, reduction="none").shape == (0,)


def test_a_target_outside_the_vocabulary_is_not_a_number(ops):
    for bad in (400, -1, 1 << 40):
        x, W, target = inputs(9, 400, 64, "bf16")
        target[4] = bad
        loss, lse, dx, dW = run(ops[1], x, W, target, torch.ones(9))
        keep = torch.arange(9) != 4
        assert torch.isnan(loss[4]) and torch.isfinite(loss.cpu()[keep]).all() and torch.isfinite(lse).all()
        assert torch.isnan(dx[4]).all() and torch.isfinite(dx.cpu()[keep]).all() and torch.isnan(dW).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wide_ranges(ops, dtype):
    """Rows of x, and of W, that differ by factors of thousands, and logits in the hundreds."""
    rows, vocab, width = 140, 600, 100
    x, W, target = inputs(rows, vocab, width, dtype)
    x = (x.float() * torch.logspace(-3, 2, rows)[:, None]).to(x.dtype)
    W = (W.float() * torch.logspace(0.5, -4, vocab)[:, None]).to(W.dtype)
    g = torch.logspace(-6, 3, rows)
    want = Exact(x, W, target, g, dtype)
    loss, lse, dx, dW = run(ops[1], x, W, target, g)
    within(loss, want.loss, want.row_bound, "loss")
    within(lse, want.lse, want.row_bound, "lse")
    # planes of G and of what it is multiplied with share a power of two: what is 2^-25 of the largest is not kept apart
    rest = torch.full((), 2.0 ** -38 if dtype == "f32" else 0.0, dtype=torch.float64)
    within(dx, want.dx, want.dx_bound + rest * g.max() * vocab * W.double().abs().max(), "dx")
    within(dW, want.dW, want.dW_bound + rest * g.max() * rows * x.double().abs().max(), "dW")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_autograd(ops, dtype, reduction):
    autograd, _ = ops
    x, W, target = inputs(6 * 35, 900, 72, dtype, ignored=0.2)
    count = int((target != IGNORE).sum())
    g = {"mean": torch.full((210,), 2.5 / count), "sum": torch.full((210,), 2.5),
         "none": torch.linspace(-1, 2, 210)}[reduction]
    want = Exact(x, W, target, g, dtype)
    xd, Wd = x.cuda().view(6, 35, 72).requires_grad_(), W.cuda().requires_grad_()
    loss = autograd.vocab_cross_entropy(xd, Wd, target.cuda().view(6, 35), reduction=reduction)
    assert loss.dtype == torch.float32
    if reduction == "none":
        loss.backward(g.cuda().view(6, 35))
        within(loss.view(-1), want.loss, want.row_bound, "loss")
    else:
        (2.5 * loss).backward()
        whole = want.loss.sum() / (count if reduction == "mean" else 1)
        assert abs(loss.item() - whole.item()) <= want.row_bound.item() * (1 if reduction == "mean" else 210) + 1e-6 * abs(whole.item())
    within(xd.grad.view(-1, 72), want.dx, want.dx_bound + 2.0 ** -22 * want.dx.abs(), "dx")
    within(Wd.grad, want.dW, want.dW_bound + 2.0 ** -22 * want.dW.abs(), "dW")


def test_autograd_of_views_and_of_one_side(ops):
    autograd, _ = ops
    x, W, target = inputs(40, 500, 64, "bf16")
    want = Exact(x, W, target, torch.ones(40), "bf16")
    wide = torch.zeros((40, 130), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:65] = x.cuda()
    wide.requires_grad_()
    Wd = torch.cat([torch.zeros(1, dtype=torch.bfloat16), W.view(-1)]).cuda()[1:].view(500, 64)   # not on 16 bytes
    spread = torch.stack([target, target], 1).cuda()[:, 0]
    autograd.vocab_cross_entropy(wide[:, 1:65], Wd, spread, reduction="none").sum().backward()
    within(wide.grad[:, 1:65], want.dx, want.dx_bound, "dx")
    assert (wide.grad[:, 0] == 0).all() and (wide.grad[:, 65:] == 0).all()
    Wd = W.cuda().requires_grad_()
    autograd.vocab_cross_entropy(x.cuda(), Wd, target.cuda(), reduction="sum").backward()
    within(Wd.grad, want.dW, want.dW_bound, "dW")


def test_gradient_against_differences(ops):
    """The loss along a random direction of x and of W, by central differences: the third derivative of the log of a sum of exponentials
    along a direction is at most the cube of the logits' range along it."""
    _, binding = ops
    rows, vocab, width = 33, 260, 40
    x, W, target = inputs(rows, vocab, width, "f32")
    gen = torch.Generator().manual_seed(3)
    ex, eW = torch.randn(x.shape, generator=gen), torch.randn(W.shape, generator=gen) / width ** 0.5
    _, _, dx, dW = run(binding, x, W, target, torch.ones(rows))
    step = 2.0 ** -7

    def total(sx, sW):
        return binding.monarch_xent_fwd((x + sx * ex).cuda(), (W + sW * eW).cuda(), target.cuda())[0].double().sum().item()
    for (sx, sW), grad, e, along in (((step, 0), dx, ex, ex @ W.t()), ((0, step), dW, eW, x @ eW.t())):
        slope = (total(sx, sW) - total(-sx, -sW)) / (2 * step)
        rest = step ** 2 / 6 * (2 * along.abs().amax(1).double()).pow(3).sum().item() + rows * 20 * 2.0 ** -22 / step
        assert abs(slope - (grad.double().cpu() * e.double()).sum().item()) <= rest


def test_weight_gradient_in_fp32_and_twice_the_same(ops):
    _, binding = ops
    x, W, target = inputs(180, 777, 128, "bf16", ignored=0.2)
    want = Exact(x, W, target, torch.ones(180), "bf16")
    first = run(binding, x, W, target, torch.ones(180), flags=binding.MONARCH_FLAG_WGRAD_F32)
    assert first[3].dtype == torch.float32
    within(first[3], want.dW, want.dW_bound, "dW")
    for a, b in zip(first, run(binding, x, W, target, torch.ones(180), flags=binding.MONARCH_FLAG_WGRAD_F32)):
        assert torch.equal(a, b)


def test_on_another_stream_and_in_a_graph(ops):
    _, binding = ops
    x, W, target = inputs(100, 600, 64, "bf16")
    eager = run(binding, x, W, target, torch.ones(100))
    xd, Wd, td, g = x.cuda(), W.cuda(), target.cuda(), torch.ones(100, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, lse = binding.monarch_xent_fwd(xd, Wd, td, stream=side)
    dx, dW = binding.monarch_xent_bwd(xd, Wd, td, lse, g, stream=side)
    side.synchronize()
    for a, b in zip(eager, (loss, lse, dx, dW)):
        assert torch.equal(a, b)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            loss, lse = binding.monarch_xent_fwd(xd, Wd, td)
            dx, dW = binding.monarch_xent_bwd(xd, Wd, td, lse, g)
    for _ in range(3):
        for t in (loss, lse, dx, dW):
            t.fill_(7)
        (torch.randn(1000, device="cuda") @ torch.randn(1000, 50, device="cuda")).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, (loss, lse, dx, dW)):
            assert torch.equal(a, b)


def test_refusals(ops):
    autograd, binding = ops
    x, W, target = (t.cuda() for t in inputs(8, 50, 64, "bf16"))
    with pytest.raises(TypeError):
        binding.monarch_xent_fwd(x, W.float(), target)
    with pytest.raises(TypeError):
        binding.monarch_xent_fwd(x.half(), W.half(), target)
    with pytest.raises(TypeError):
        binding.monarch_xent_fwd(x, W, target.int())
    with pytest.raises(ValueError):
        binding.monarch_xent_fwd(x, W[:, :32], target)
    with pytest.raises(ValueError):
        binding.monarch_xent_fwd(x, W, target[:5])
    with pytest.raises(ValueError):
        binding.monarch_xent_fwd(x.t().contiguous().t(), W, target)
    with pytest.raises(ValueError):
        binding.monarch_xent_fwd(x.cpu(), W, target)
    with pytest.raises(ValueError):
        autograd.vocab_cross_entropy(x, W, target, reduction="most")
    with pytest.raises(ValueError):
        autograd.vocab_cross_entropy(x, W, target[:4])
    lse = torch.zeros(8, device="cuda")
    with pytest.raises(ValueError):
        binding.monarch_xent_bwd(x, W, target, lse, torch.ones(3, device="cuda"))
    with pytest.raises(TypeError):
        binding.monarch_xent_bwd(x, W, target, lse, torch.ones(8, device="cuda").bfloat16())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, ignored", [(40, 0.5), (200, 0.0), (1500, 0.4), (3000, 0.95), (300, 1.0)])
def test_ignored_rows_left_out(ops, dtype, rows, ignored):
    """The forward that computes nothing for them gives the losses, and the lse of the others, of the one that does."""
    _, binding = ops
    x, W, target = inputs(rows, 450, 72, dtype, ignored=ignored)
    x[target == IGNORE] = float("nan")
    want = Exact(x, W, target, torch.ones(rows), dtype)
    xd, Wd, td = x.cuda(), W.cuda(), target.cuda()
    loss, lse = binding.monarch_xent_fwd(xd, Wd, td, flags=binding.MONARCH_FLAG_SKIP_IGNORED)
    counts = target != IGNORE
    within(loss, want.loss, want.row_bound, "loss")
    within(lse.cpu()[counts], want.lse[counts], want.row_bound, "lse")
    dx, dW = binding.monarch_xent_bwd(xd, Wd, td, lse, torch.ones(rows, device="cuda"))
    within(dx, want.dx, want.dx_bound, "dx")
    within(dW, want.dW, want.dW_bound, "dW")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1025, 4097, 5000, 9001])
def test_more_rows_than_are_taken_at_once(ops, dtype, rows):
    """Workgroups that take several rows each, the last ones fewer or none, and some nothing but ignored ones."""
    x, W, target = inputs(rows, 90, 10, dtype, ignored=0.3)
    target[1:300] = IGNORE
    g = torch.rand((rows,), generator=torch.Generator().manual_seed(7)) - 0.3
    want = Exact(x, W, target, g, dtype)
    for more in ({}, {"flags": ops[1].MONARCH_FLAG_SKIP_IGNORED}):
        xd, Wd, td = x.cuda(), W.cuda(), target.cuda()
        loss, lse = ops[1].monarch_xent_fwd(xd, Wd, td, **more)
        dx, dW = ops[1].monarch_xent_bwd(xd, Wd, td, lse, g.cuda())
        within(loss, want.loss, want.row_bound, "loss")
        within(dx, want.dx, want.dx_bound, "dx")
        within(dW, want.dW, want.dW_bound, "dW")


@pytest.mark.parametrize("shape, dtype", [((3000, 9000, 190), "f32"), ((6000, 9000, 150), "bf16"), ((8000, 9000, 150), "bf16")])
def test_widths_that_leave_room_in_the_square_tiles(ops, shape, dtype):
    """dx and dW of some hundred features and many rows: tiles of 192 features, shares of the sums."""
    x, W, target = inputs(*shape, dtype, ignored=0.2)
    g = torch.rand((shape[0],), generator=torch.Generator().manual_seed(7)) - 0.3
    want = Exact(x.cuda(), W.cuda(), target.cuda(), g.cuda(), dtype)
    loss, _, dx, dW = run(ops[1], x, W, target, g)
    within(loss, want.loss.cpu(), want.row_bound.cpu(), "loss")
    within(dx, want.dx.cpu(), want.dx_bound.cpu(), "dx")
    within(dW, want.dW.cpu(), want.dW_bound.cpu(), "dW")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(300, 33500, 40), (513, 22100, 33)])
def test_a_vocabulary_that_ends_in_smaller_tiles(ops, shape, dtype):
    x, W, target = inputs(*shape, dtype, ignored=0.1)
    target[:40] = shape[1] - 1 - torch.arange(40) * 20
    want = Exact(x.cuda(), W.cuda(), target.cuda(), torch.ones(shape[0]).cuda(), dtype)
    counts = target != IGNORE
    for flags in (0, ops[1].MONARCH_FLAG_SKIP_IGNORED):
        loss, lse = ops[1].monarch_xent_fwd(x.cuda(), W.cuda(), target.cuda(), flags=flags)
        within(loss, want.loss.cpu(), want.row_bound.cpu(), "loss")
        within(lse.cpu()[counts], want.lse.cpu()[counts], want.row_bound.cpu(), "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape, ignored", [((1, 70, 33), 0.0), ((40, 300, 96), 1.0), ((150, 1100, 64), 0.3), ((150, 1100, 65), 1.0), ((300, 700, 40), 0.95)])
def test_what_the_workspace_holds_has_no_influence(ops, shape, ignored, dtype):
    _, binding = ops
    x, W, target = (t.cuda() for t in inputs(*shape, dtype, ignored=ignored))
    code, g = 0 if dtype == "f32" else 1, torch.rand((shape[0],), generator=torch.Generator().manual_seed(7)).cuda()
    results = []
    for fill in (0, 255):  # (255: not a number in every type)
        ws = torch.full((binding.monarch_xent_fwd_workspace_bytes(*shape, code),), fill, dtype=torch.uint8, device="cuda")
        loss, lse = binding.monarch_xent_fwd(x, W, target, workspace=ws)
        ws = torch.full((binding.monarch_xent_bwd_workspace_bytes(*shape, code),), fill, dtype=torch.uint8, device="cuda")
        results.append([loss, lse] + list(binding.monarch_xent_bwd(x, W, target, lse, g, workspace=ws)))
    for a, b in zip(*results):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 200, 1), (2, 300, 31), (20, 260, 702), (32, 129, 197), (33, 129, 5), (50, 300, 77), (63, 1000, 385), (64, 127, 130)])
def test_few_rows_that_start_anywhere(ops, shape, dtype):
    """Forward of up to 64 rows whose width is no whole number of 16-byte pieces: one step and less, several, each of the two tiles."""
    x, W, target = inputs(*shape, dtype, ignored=0.2 if shape[0] > 2 else 0.0)
    want, counts = Exact(x, W, target, torch.ones(shape[0]), dtype), target != IGNORE
    loss, lse = ops[1].monarch_xent_fwd(x.cuda(), W.cuda(), target.cuda())
    within(loss, want.loss, want.row_bound, "loss")
    within(lse.cpu()[counts], want.lse[counts], want.row_bound, "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(512, 33500, 40), (1000, 17000, 33)])
def test_the_same_with_rows_that_fill_the_tiles(ops, shape, dtype):
    test_a_vocabulary_that_ends_in_smaller_tiles(ops, shape, dtype)
