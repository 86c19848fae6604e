"""orthogonalize against its definition in 64 bits, and with the layer whose weight it updates."""

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402
from paper_2607_24062_gb300 import api  # noqa: E402

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
QUINTIC = (3.4445, -4.7750, 2.0315)


def _update(shape, seed, dtype=F32, strong=8, weak=0.1, size=1e-3, gap=0):
    """A few strong directions and many weak ones; what lies between the rows is NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    *b, m, n = shape
    r = min(strong, m, n)
    x = torch.randn((*b, m, r), generator=g, device=DEV) * 0.6 ** torch.arange(r, device=DEV)
    x = x @ torch.randn((*b, r, n), generator=g, device=DEV) + weak * torch.randn((*b, m, n), generator=g, device=DEV)
    to = torch.full((*b, m, (n + 7) // 8 * 8 + gap), float("nan"), device=DEV, dtype=dtype)
    to[..., :n] = x * size
    return to[..., :n]


def _steps(g, steps, coeffs, eps, scale, off=0.0, seed=0):
    """The definition in 64 bits; with `off` every operand of every product is off by up to that part of it."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    about = lambda t: t if off == 0.0 else t * (1 + off * (2 * torch.rand(t.shape, generator=gen, device=DEV, dtype=t.dtype) - 1))   # noqa: E731
    x = g.double()
    x = x if x.dim() == 3 else x[None]
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    norm = x.square().sum((1, 2), keepdim=True).sqrt() + eps
    x = torch.where(norm == 0, torch.zeros_like(x), x / norm)
    for a, b, c in (coeffs if len(coeffs) == steps and hasattr(coeffs[0], "__len__") else [coeffs] * steps):
        p = about(x)
        gram = p @ about(x).mT
        p = about(gram)
        q = a * torch.eye(x.shape[1], device=DEV, dtype=x.dtype) + b * gram + c * (p @ about(gram).mT)
        x = about(q) @ about(x)
    x = scale * (x.mT if tall else x)
    return x if g.dim() == 3 else x[0]


def _check(out, g, steps=5, coeffs=QUINTIC, eps=1e-7, scale=1.0):
    """Every operand is held to 2^-16 of it (two bf16 numbers: 2^-8 of 2^-8) and the product of both small parts, 2^-16 as well, is
    left out: 2^-15 for an operand covers both.  What such errors do to the result, whose small singular values the steps
    amplify, is the definition's own answer to them; four times the largest of three trials, and the rounding to bf16."""
    exact = _steps(g, steps, coeffs, eps, scale)
    moved = max(float((_steps(g, steps, coeffs, eps, scale, 2.0 ** -15, s) - exact).abs().max()) for s in (1, 2, 3))
    off = 2.0 ** -8 * exact.abs() + 4 * moved + 1e-38
    bad = ~((out.double() - exact).abs() <= off)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4], out[bad][:4], exact[bad][:4], moved)
    # and nothing is off by more than the rounding on the whole: uniform errors of up to 2^-8 are 2^-8 / sqrt(3) on average
    assert float((out.double() - exact).norm()) <= 2.0 ** -8 * float(exact.norm()) + 4 * moved * exact.numel() ** 0.5


SHAPES = [(1, 1), (1, 7), (9, 1), (3, 5), (8, 8), (17, 130), (64, 64), (130, 17), (65, 300), (128, 129), (257, 256), (300, 515),
          (515, 258), (512, 512), (200, 3000), (2051, 260), (700, 1030)]


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF])
def test_matrices(m, n, dtype):
    g = _update((m, n), m + 3 * n, dtype, gap=8)
    flags = api.new_flags()
    out = acrl.orthogonalize(g, flags=flags)
    assert out.dtype == BF and out.shape == g.shape and acrl.read_flags(flags) == 0
    _check(out, g)


@pytest.mark.parametrize("B,m,n", [(1, 40, 72), (3, 100, 67), (5, 67, 130), (2, 300, 520), (20, 33, 24)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_batches(B, m, n, dtype):
    g = _update((B, m, n), 5, dtype)
    g = g * 10.0 ** torch.arange(B, device=DEV).view(-1, 1, 1).remainder(5).to(dtype)
    g = _aligned(g)
    out = acrl.orthogonalize(g)
    _check(out, g)
    _check(acrl.orthogonalize(g[B - 1]), g[B - 1])


@pytest.mark.parametrize("B,m,n", [(30, 512, 512), (12, 512, 700), (9, 700, 512), (24, 1024, 1024)])
def test_more_matrices_than_pairs_of_processors(B, m, n):
    """Where the steps of many matrices overlap, and their products have tiles of 256 x 256 on the diagonal: the same every time,
    and each matrix as by itself."""
    g = _update((B, m, n), 9)
    flags = api.new_flags()
    out = acrl.orthogonalize(g, flags=flags)
    for _ in range(20):
        assert torch.equal(acrl.orthogonalize(g, flags=flags), out)
    assert acrl.read_flags(flags) == 0
    for z in (0, B // 2, B - 1):
        _check(out[z], g[z])
    x = out.float()
    x = x if m <= n else x.mT
    gram = x @ x.mT
    assert float((gram - torch.diag_embed(gram.diagonal(dim1=1, dim2=2))).abs().max()) < 1.0 and bool(torch.isfinite(out).all())


def _aligned(t, gap=0):
    to = torch.full((*t.shape[:-1], (t.shape[-1] + 7) // 8 * 8 + gap), float("nan"), dtype=t.dtype, device=DEV)[..., : t.shape[-1]]
    return to.copy_(t)


@pytest.mark.parametrize("shape", [(5, 7), (33, 129), (131, 67), (3, 40, 53), (2, 65, 31), (300, 515)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_of_any_alignment(shape, dtype):
    """Rows one after the other, and a view that starts anywhere: the update's and the result's."""
    g = _update(shape, 21, dtype).contiguous()
    want = acrl.orthogonalize(_aligned(g))
    _check(acrl.orthogonalize(g), g)
    n = g.numel()
    flat = torch.full((n + 6,), float("nan"), dtype=dtype, device=DEV)
    flat[3: 3 + n] = g.flatten()
    out = torch.full((n + 6,), 7.0, dtype=BF, device=DEV)
    got = acrl.orthogonalize(flat[3: 3 + n].view(shape), out=out[1: 1 + n].view(shape))
    _check(got, g)
    assert torch.equal(got, want) and bool((out[:1] == 7.0).all()) and bool((out[1 + n:] == 7.0).all())


@pytest.mark.parametrize("steps,coeffs,eps,scale", [(1, (1.5, -0.5, 0.0), 0.0, 1.0), (1, QUINTIC, 1e-7, -2.5), (3, QUINTIC, 0.0, 0.2),
                                                    (8, (1.875, -1.25, 0.375), 1e-7, 1.0),
                                                    (3, [(4.0, -6.0, 2.5), (3.0, -3.5, 1.4), (1.875, -1.25, 0.375)], 1e-3, 1.0)])
@pytest.mark.parametrize("m,n", [(40, 72), (300, 130)])
def test_steps_and_coefficients(steps, coeffs, eps, scale, m, n):
    g = _update((m, n), 7)
    _check(acrl.orthogonalize(g, steps=steps, coeffs=coeffs, eps=eps, scale=scale), g, steps, coeffs, eps, scale)


def test_singular_values_come_near_one():
    g = _update((200, 333), 3, weak=0.3)
    s = torch.linalg.svdvals(acrl.orthogonalize(g).double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25       # where the quintic of five steps puts what is not tiny
    # the cubic's limit is the polar factor: U V^T
    u, _, v = torch.linalg.svd(g.double(), full_matrices=False)
    out = acrl.orthogonalize(g, steps=30, coeffs=(1.5, -0.5, 0.0)).double()
    assert bool(((out - u @ v).abs() <= 2.0 ** -8 * (u @ v).abs() + 2.0 ** -11).all())


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("eps", [0.0, 1e-7])
def test_updates_of_any_size(size, eps):
    """Sums of squares beyond fp32's range, either way, in matrices that are not."""
    g = _update((65, 130), 9, size=size)
    _check(acrl.orthogonalize(g, eps=eps), g, eps=eps)


def test_very_long_rows():
    """The Gram matrix of rows of a million columns: its sums are split, however many tiles there are."""
    for m, n in ((40, 2 ** 20 + 24), (2 ** 17 + 40, 300)):
        g = _update((m, n), 17, BF)
        _check(acrl.orthogonalize(g), g)


def test_zeros_infinities_and_nan():
    for m, n in ((40, 72), (300, 130)):
        g = _update((5, m, n), 11)
        g[1] = 0.0
        want = acrl.orthogonalize(g)
        assert not bool(want[1].any()) and bool(want.isfinite().all())
        assert not bool(acrl.orthogonalize(g, eps=0.0)[1].any())
        g[0, 3, 5], g[3, 0, 0], g[4, m - 1, n - 1] = float("nan"), float("inf"), float("-inf")
        flags = api.new_flags()
        out = acrl.orthogonalize(g, flags=flags)
        assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
        assert bool(out[[0, 3, 4]].isnan().all()) and torch.equal(out[[1, 2]], want[[1, 2]])
        # rows and columns of zeros stay zeros
        g = _update((m, n), 12)
        g[5], g[:, 7] = 0.0, 0.0
        out = acrl.orthogonalize(g)
        assert not bool(out[5].any()) and not bool(out[:, 7].any())
        _check(out, g)


def test_output_in_place_and_what_is_beyond_it():
    for shape in ((37, 50), (130, 67), (3, 40, 52)):
        g = _update(shape, 13, BF)
        want = acrl.orthogonalize(g)
        big = torch.full((*shape[:-2], shape[-2] + 1, (shape[-1] + 7) // 8 * 8 + 8), 7.0, dtype=BF, device=DEV)
        view = big[..., : shape[-2], : shape[-1]]
        assert acrl.orthogonalize(g, out=view) is view
        assert torch.equal(view, want)
        assert bool((big[..., shape[-2]:, :] == 7.0).all()) and bool((big[..., shape[-1]:] == 7.0).all())
        acrl.orthogonalize(g, out=g)
        assert torch.equal(g, want)


def test_streams_graphs_and_repetition():
    g, h = _update((260, 300), 1), _update((3, 130, 72), 2, BF)
    want = [acrl.orthogonalize(t).clone() for t in (g, h)]
    for _ in range(3):
        assert all(torch.equal(w, acrl.orthogonalize(t)) for w, t in zip(want, (g, h)))
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    for _ in range(20):
        big = torch.tanh(big @ big)
    for _ in range(3):
        torch.empty(api.orthogonalize_workspace_bytes(1, 260, 300), dtype=torch.uint8, device=DEV).fill_(255)
    got = [acrl.orthogonalize(t, stream=side) for t in (g, h)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs, outs = [], []
    for t in (g, h):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(acrl.orthogonalize(t))
        graphs.append(graph)
    for _ in range(5):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_two_at_once_that_each_fill_the_gpu():
    """On two streams, eagerly and from graphs, beside layers on a third: the CTAs of a call wait for one another, never for those
    of another call."""
    sets = [_update((30, 512, 512), 1), _update((16, 1024, 512), 2, BF)]
    x, w = (torch.randn(n, 2048, device=DEV).to(BF) for n in (1024, 4096))
    flags = [api.new_flags() for _ in sets]
    want = [acrl.orthogonalize(t).clone() for t in sets]
    y = acrl.linear(x, w).clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got.append([acrl.orthogonalize(t, flags=f, stream=s) for t, f, s in zip(sets, flags, streams)])
        got[-1].append(acrl.linear(x, w, stream=streams[2]))
    torch.cuda.synchronize()
    assert [acrl.read_flags(f) for f in flags] == [0, 0]
    assert all(torch.equal(a, b) for g in got for a, b in zip(want + [y], g))
    graphs, outs = [], []
    for t, f in zip(sets, flags):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(acrl.orthogonalize(t, flags=f))
        graphs.append(graph)
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert [acrl.read_flags(f) for f in flags] == [0, 0]
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_nothing_and_refusals():
    g = _update((40, 72), 1)
    assert acrl.orthogonalize(g[:0]).shape == (0, 72) and acrl.orthogonalize(g[:, :0]).shape == (40, 0)
    assert acrl.orthogonalize(g[None][:0]).shape == (0, 40, 72)
    for call in (lambda: acrl.orthogonalize(g.double()), lambda: acrl.orthogonalize(g.cpu()), lambda: acrl.orthogonalize(g[0]),
                 lambda: acrl.orthogonalize(g.t()), lambda: acrl.orthogonalize(g, steps=0), lambda: acrl.orthogonalize(g, steps=65),
                 lambda: acrl.orthogonalize(g, eps=-1.0), lambda: acrl.orthogonalize(g, eps=float("nan")),
                 lambda: acrl.orthogonalize(g, scale=float("inf")), lambda: acrl.orthogonalize(g, coeffs=(1.5, -0.5)),
                 lambda: acrl.orthogonalize(g, coeffs=(1.5, float("nan"), 0.0)),
                 lambda: acrl.orthogonalize(g, steps=3, coeffs=[QUINTIC, QUINTIC]),
                 lambda: acrl.orthogonalize(g, out=torch.empty_like(g)),
                 lambda: acrl.orthogonalize(g, out=torch.empty((40, 80), dtype=BF, device=DEV)),
                 lambda: acrl.orthogonalize(g[None].expand(3, 40, 72), out=torch.empty((1, 40, 72), dtype=BF, device=DEV).expand(3, 40, 72)),
                 lambda: acrl.orthogonalize(g, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(acrl.AcrlError):
            call()


def test_layers_trained_with_it():
    """Two layers with a residual, their gradients, and updates that are orthogonalised: against the same in 64 bits from the
    same gradients, step by step."""
    T, H, W = 90, 72, 200
    gen = torch.Generator(device=DEV).manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)   # noqa: E731
    x, target = rnd(T, H).to(BF), rnd(T, H)
    up, down = rnd(W, H) * H ** -0.5, rnd(H, W) * W ** -0.5
    bias = torch.zeros(W, device=DEV)
    moment = [torch.zeros_like(up), torch.zeros_like(down)]
    for step in range(4):
        a, c, b = up.to(BF).requires_grad_(), down.to(BF).requires_grad_(), bias.clone().requires_grad_()
        y = acrl.linear_layer(acrl.linear_layer(x, a, b, "gelu"), c, residual=x)
        ((y.float() - target) ** 2).mean().backward()
        # the same forward and backward by torch, in 64 bits
        a64, c64, b64 = (t.detach().double().requires_grad_() for t in (a, c, b))
        hidden = torch.nn.functional.gelu(x.double() @ a64.t() + b64)
        ((hidden @ c64.t() + x.double() - target) ** 2).mean().backward()
        for t, ref in ((a, a64), (c, c64), (b, b64)):
            # several roundings to bf16 on the way (the hidden state, the output, two incoming gradients, the weight's), 2^-8 each
            assert float((t.grad.double() - ref.grad).norm()) <= 6 * 2.0 ** -8 * float(ref.grad.norm())
        with torch.no_grad():
            for m, t, w in zip(moment, (a, c), (up, down)):
                m.mul_(0.9).add_(t.grad.float())
                o = acrl.orthogonalize(m)
                _check(o, m)
                w.sub_(0.05 * o.float())
            bias -= 0.05 * b.grad
