"""Orthogonalised updates on the GPU against their float64 definition: types,
shapes, ranges, and the gradients they are made for.

Bounds.  A product of operands that carry 22 bits or more, accumulated in
float32, errs by at most (2^-20 + K 2^-24) sqrt(k) of the operands' spectral
sizes in norm for a k x K times K x r product; with A, A A and B X and the
coefficients (3.4445 + 4.775 + 2.0315 = 10.3 of them, the gain of one step in
size) a step adds at most 10.3 times three of these, and every later step
magnifies it by at most its slope; over all steps that is `gain` times for the
first and less for the others, 1.5 gain in all (a geometric sum with ratio
1 / 3.4445).  So |X - ref|_2 <= 31 * 1.5 gain (2^-20 + K 2^-24) as the worst
case.  Rounding errors of a product are random in sign; their sum over K
products grows as its root, and a random matrix of entrywise errors e has
spectral norm 2 sqrt(r) e instead of r e, which leaves

    max |X - ref| <= gain (2^-20 + sqrt(K) 2^-24) max |ref|

for each entry.  An output's rounding adds half a step of its type.
"""
import numpy as np
import pytest

import oracle
from oracle import ortho_oracle as oo
from paper_2309_16318_amd import deeppcr, synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SHAPES = [(1, 1, 1), (3, 1, 5), (2, 5, 1), (4, 2, 2), (5, 16, 16), (3, 17, 17), (7, 32, 32),
          (2, 31, 33), (3, 64, 64), (2, 40, 64), (2, 100, 100), (3, 128, 128), (2, 128, 16),
          (2, 16, 128), (2, 50, 100), (2, 90, 120), (2, 120, 70), (2, 60, 20), (2, 129, 129), (1, 96, 200), (2, 200, 96), (1, 256, 256), (1, 1, 300),
          (1, 333, 130), (1, 520, 264), (1, 130, 1025),
          # more large tiles than CUs
          (270, 128, 250), (260, 250, 120), (90, 250, 256)]


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def cpu(t):
    return t.detach().double().cpu().numpy()


def check(got, ref, dtype, steps=5, coeffs=oo.COEFFS):
    got, half = cpu(got), torch.finfo(dtype).eps / 2
    K = max(ref.shape[-2:])
    top = np.max(np.abs(ref), axis=(-2, -1), keepdims=True)
    e = max(1.0, oo.gain(steps, coeffs)) * (2.0 ** -20 + np.sqrt(K) * 2.0 ** -24)
    assert np.all(np.isfinite(got)) and got.shape == ref.shape
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    bad = np.abs(got - ref) - (e * top + half * np.abs(ref) + tiny)
    assert np.max(bad) <= 0, np.max(np.abs(got - ref) / top)


def gradient(N, m, n, dtype, dev, seed=0):
    gen = torch.Generator().manual_seed(seed + 13 * m + n)
    return (torch.randn(N, m, n, generator=gen) * 0.02).to(dtype).to(dev)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", list(TYPES))
def test_shapes(dev, shape, kind):
    G = gradient(*shape, TYPES[kind], dev)
    check(deeppcr.deeppcr_orthogonalize(G), oo.orthogonalize(cpu(G)), TYPES[kind])


@pytest.mark.parametrize("w", [12, 128, 160])
def test_steps_and_coefficients(dev, w):
    G = gradient(2, w, w, torch.float32, dev)
    for steps, coeffs in ((0, oo.COEFFS), (1, oo.COEFFS), (2, (1.5, -0.5, 0.0)),
                          (6, (1.875, -1.25, 0.375))):
        got = deeppcr.deeppcr_orthogonalize(G, steps=steps, coeffs=coeffs)
        check(got, oo.orthogonalize(cpu(G), steps, coeffs), torch.float32, steps, coeffs)
    one = deeppcr.deeppcr_orthogonalize(G[1])
    assert torch.equal(one, deeppcr.deeppcr_orthogonalize(G)[1])


@pytest.mark.parametrize("w", [16, 64, 128, 150])
def test_range(dev, w):
    """Gradients far below and above the squares' float32 range, a zero
    matrix, rank one, and non-finite ones that stay alone."""
    G = gradient(8, w, w, torch.float32, dev)
    G[0] *= 1e-37 / 0.02
    G[1] = G[1] * 50 * 1e37
    G[2] = 0
    G[3] = torch.outer(G[3, 0], G[3, 1])
    got = deeppcr.deeppcr_orthogonalize(G, eps=0.0)
    ref = oo.orthogonalize(cpu(G), eps=0.0)
    check(got, ref, torch.float32)
    assert torch.all(got[2] == 0)
    check(deeppcr.deeppcr_orthogonalize(G), oo.orthogonalize(cpu(G)), torch.float32)
    G[4, 0, 0] = float("nan")
    G[5, w - 1, 2] = float("inf")
    bad = deeppcr.deeppcr_orthogonalize(G, eps=0.0)
    keep = [0, 1, 2, 3, 6, 7]
    assert torch.equal(bad[keep], got[keep])
    assert torch.isnan(bad[4]).any() and torch.isnan(bad[5]).any()


@pytest.mark.parametrize("w", [16, 30, 64, 128, 150])
def test_gradients_below_eps(dev, w):
    """|G| / eps from 10 down to 1e-20: X is small, and moved by its linear term
    until it has grown; its own size bounds its error."""
    scale = 10.0 ** torch.arange(1.0, -21.0, -3.0)
    G = gradient(len(scale), w, w, torch.float32, dev)
    G *= (scale * 1e-7).to(dev)[:, None, None] / torch.linalg.matrix_norm(G)[:, None, None]
    for steps, coeffs in ((5, oo.COEFFS), (12, (1.5, -0.5, 0.0)), (3, (0.5, 0.25, 0.0))):
        got = deeppcr.deeppcr_orthogonalize(G, steps=steps, coeffs=coeffs)
        check(got, oo.orthogonalize(cpu(G), steps, coeffs), torch.float32, steps, coeffs)


@pytest.mark.parametrize("w", [16, 30, 64, 150])
def test_a_linear_term_that_counts_least(dev, w):
    """Iterates that the cubic term makes, far larger than the linear term alone
    would have them.  They are held to the bound u -> |a| u + |b| u^3 + |c| u^5 of
    their norms, here far above them: a step adds an error of 2^-20 u' (its
    operands' 22 bits, against their bounds), and later steps magnify it by at most
    their slope |a| + 3 |b| u^2 + 5 |c| u^4 <= 5 u' / u, so that three steps end
    within (25 + 5 + 1) 2^-20 of the last bound."""
    G = gradient(3, w, w, torch.float32, dev)
    G[1] *= 1e-7 / torch.linalg.matrix_norm(G[1])          # X = 1 / 2
    G[2] = torch.outer(G[2, 0], G[2, 1]) * 1e-6            # one singular value, small
    for coeffs in ((0.0625, 0.9375, 0.0), (0.0625, 1.0, -0.1), (-0.0625, 0.0, 1.0)):
        got = cpu(deeppcr.deeppcr_orthogonalize(G, steps=3, coeffs=coeffs))
        ref = oo.orthogonalize(cpu(G), 3, coeffs)
        norm = np.linalg.norm(cpu(G), axis=(1, 2))
        u = norm / (norm + 1e-7)
        for _ in range(3):
            u = abs(coeffs[0]) * u + abs(coeffs[1]) * u ** 3 + abs(coeffs[2]) * u ** 5
        err = np.max(np.abs(got - ref), axis=(1, 2))
        assert np.all(np.isfinite(got)) and np.all(err <= 31 * 2.0 ** -20 * u), (coeffs, err / u)


def test_more_matrices_than_a_launch_works_on(dev):
    """The stack goes through the workspace in parts."""
    N, m, n = 9000, 3, 130
    few = deeppcr.orthogonalize_workspace_bytes(100, m, n) / 100
    assert deeppcr.orthogonalize_workspace_bytes(N, m, n) < few * N
    G = gradient(N, m, n, torch.float32, dev)
    got = deeppcr.deeppcr_orthogonalize(G)
    for part in (slice(0, 4), slice(7000, 7400), slice(N - 4, N)):
        assert torch.equal(got[part], deeppcr.deeppcr_orthogonalize(G[part].contiguous()))


def test_in_place_and_same_bits(dev):
    for shape in ((40, 24, 24), (3, 128, 128), (2, 300, 140)):
        G = gradient(*shape, torch.float32, dev)
        first = deeppcr.deeppcr_orthogonalize(G)
        for _ in range(3):
            assert torch.equal(first, deeppcr.deeppcr_orthogonalize(G))
        X = G.clone()
        assert deeppcr.deeppcr_orthogonalize(X, X=X) is X and torch.equal(X, first)


def test_captured(dev):
    for shape in ((5, 64, 64), (2, 200, 140)):
        G = gradient(*shape, torch.bfloat16, dev)
        X = torch.empty_like(G)
        ws = torch.empty(deeppcr.orthogonalize_workspace_bytes(*shape), dtype=torch.uint8,
                         device=dev)
        deeppcr.deeppcr_orthogonalize(G, X=X, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            deeppcr.deeppcr_orthogonalize(G, X=X, workspace=ws)
        for _ in range(3):
            G.copy_(torch.randn_like(G))
            want = deeppcr.deeppcr_orthogonalize(G)
            X.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(X, want)


def test_update_of_the_mlp_gradients(dev):
    """dW of the library's own backward pass, every layer's update."""
    B, L, w = 4, 12, 24
    d = {k: torch.from_numpy(v).to(dev) for k, v in synth.mlp_inputs(B, L, w, seed=5).items()}
    res = deeppcr.deeppcr_mlp_forward(d["W"], d["bias"], d["z0"])
    dW = deeppcr.deeppcr_mlp_backward(d["W"], d["bias"], d["z0"], res.Z, d["G"])[2]
    check(deeppcr.deeppcr_orthogonalize(dW, eps=0.0), oo.orthogonalize(cpu(dW), eps=0.0),
          torch.float32)


@pytest.mark.parametrize("shape", [(3, 5, 700), (2, 700, 5), (4, 32, 129), (2, 5000, 32), (1, 1, 8192),
                                   (5, 17, 300), (2, 31, 257), (700, 2, 140)], ids=str)
@pytest.mark.parametrize("kind", list(TYPES))
def test_long_matrices(dev, shape, kind):
    G = gradient(*shape, TYPES[kind], dev)
    for steps in (5, 1, 0):
        got = deeppcr.deeppcr_orthogonalize(G, steps=steps)
        check(got, oo.orthogonalize(cpu(G), steps), TYPES[kind], steps)
        X = G.clone()
        assert torch.equal(deeppcr.deeppcr_orthogonalize(X, X=X, steps=steps), got)


@pytest.mark.parametrize("m, n", [(20, 300), (400, 6)])
def test_long_matrices_range(dev, m, n):
    """Far below and above the squares' range, far below eps, zero, not finite."""
    G = gradient(7, m, n, torch.float32, dev)
    G[0] *= 1e-37 / 0.02
    G[1] = G[1] * 50 * 1e37
    G[2] = 0
    got = deeppcr.deeppcr_orthogonalize(G, eps=0.0)
    check(got, oo.orthogonalize(cpu(G), eps=0.0), torch.float32)
    assert torch.all(got[2] == 0)
    low = deeppcr.deeppcr_orthogonalize(G * 1e-9)
    check(low[3:], oo.orthogonalize(cpu(G * 1e-9))[3:], torch.float32)
    G[3, 0, 0] = float("nan")
    G[4, m - 1, 2] = float("inf")
    bad = deeppcr.deeppcr_orthogonalize(G, eps=0.0)
    keep = [0, 1, 2, 5, 6]
    assert torch.equal(bad[keep], got[keep])
    assert torch.isnan(bad[3]).any() and torch.isnan(bad[4]).any()


@pytest.mark.parametrize("shape", [(129, 129), (20, 300), (70, 400), (1024, 1024)], ids=str)
def test_squares_that_add_up_beyond_float32(dev, shape):
    """Elements whose squares are in float32's range and their sum is not, alone, in
    a single row, and beside larger ones; with no steps too (X = G / |G|)."""
    scales = [1e13, 1e15, 1e16, 1e17, 3e17, 1e18, 2e18, 1e19, 1e20]
    G = gradient(len(scales) + 2, *shape, torch.float32, dev) * 50
    for i, s in enumerate(scales):
        G[i] *= s
    G[-2, 0] *= 1e18
    G[-1] *= 1e17
    G[-1, :, 1] *= 1e3
    for steps in (5, 0):
        got = deeppcr.deeppcr_orthogonalize(G, eps=0.0, steps=steps)
        check(got, oo.orthogonalize(cpu(G), steps, eps=0.0), torch.float32, steps)


def float32_products(G, steps=5, coeffs=oo.COEFFS, eps=1e-7):
    """The update with float32 products."""
    X = G / (torch.sqrt((G * G).sum((1, 2), keepdim=True)) + eps)
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2).contiguous()
    a, b, c = coeffs
    for _ in range(steps):
        A = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.bmm(b * A + c * torch.bmm(A, A), X)
    return X.transpose(1, 2) if tall else X


# a value has all of its 24 bits up to 32 rows: no more than float32's roundings, and
# a quarter for chance; two parts round to 2^-23 of a value, twice float32's 2^-24
PRECISION = [((1000, 4, 4), 1.25), ((300, 11, 11), 1.25), ((200, 16, 16), 1.25), ((100, 24, 24), 1.25),
             ((100, 4, 69), 1.25), ((60, 32, 32), 1.25), ((40, 128, 17), 1.25), ((40, 5, 755), 1.25),
             ((20, 32, 2000), 1.25), ((20, 20, 300), 1.25),
             ((60, 33, 64), 2), ((30, 64, 64), 2), ((20, 100, 100), 2), ((20, 128, 128), 2),
             ((16, 33, 130), 2), ((16, 33, 1024), 2), ((8, 48, 2048), 2), ((8, 33, 8192), 2),
             ((8, 4096, 64), 2), ((8, 64, 1024), 2), ((4, 128, 8192), 2), ((2, 256, 8192), 2),
             ((3, 512, 512), 2), ((300, 128, 512), 2)]


@pytest.mark.parametrize("shape, times", PRECISION, ids=str)
def test_errs_like_float32_products(dev, shape, times):
    """The error of whole matrices against that of float32 products, over enough
    entries for chance to average out."""
    gen = torch.Generator().manual_seed(sum(shape))
    N, m, n = shape
    G = (torch.randn(N, m, n, generator=gen) * torch.exp(0.5 * torch.randn(N, 1, n, generator=gen))).to(dev)
    want = oo.orthogonalize(cpu(G))
    err = lambda X: np.linalg.norm(cpu(X) - want) / np.linalg.norm(want)
    got, plain = err(deeppcr.deeppcr_orthogonalize(G)), err(float32_products(G))
    assert got <= times * plain, (got, plain, got / plain)


@pytest.mark.parametrize("shape, most", [((7500, 33, 129), 7281), ((9000, 130, 3), 8192)], ids=str)
def test_parts_of_a_stack(dev, shape, most):
    """Stacks of which the workspace holds `most` matrices at a time: the second
    turn uses all of it again."""
    N, m, n = shape
    need = deeppcr.orthogonalize_workspace_bytes
    assert need(most - 1, m, n) < need(most, m, n) == need(most + 1, m, n) == need(N, m, n)
    G = gradient(N, m, n, torch.float32, dev)
    got = deeppcr.deeppcr_orthogonalize(G)
    for part in (slice(0, 4), slice(most - 150, most + 150), slice(N - 4, N)):
        assert torch.equal(got[part], deeppcr.deeppcr_orthogonalize(G[part].clone()))
    check(got[most - 2:most + 2], oo.orthogonalize(cpu(G[most - 2:most + 2])), torch.float32)
    assert torch.equal(deeppcr.deeppcr_orthogonalize(G, X=G), got)


@pytest.mark.parametrize("shape", [(2, 33, 200), (3, 300, 40), (1, 64, 129), (2, 48, 1025), (1, 64, 8192),
                                   (1, 5001, 33), (1, 1100, 2100), (1, 2049, 513)], ids=str)
@pytest.mark.parametrize("kind", list(TYPES))
def test_thin_and_large_tiles(dev, shape, kind):
    """33 to 64 rows or columns beside longer ones (products of four steps), and
    sides beyond 2048."""
    G = gradient(*shape, TYPES[kind], dev)
    for steps in (5, 1, 0) if shape[0] > 1 else (5,):
        got = deeppcr.deeppcr_orthogonalize(G, steps=steps)
        check(got, oo.orthogonalize(cpu(G), steps), TYPES[kind], steps)


@pytest.mark.parametrize("m, n", [(40, 300), (400, 64)])
def test_thin_tiles_range(dev, m, n):
    """Far below and above the squares' range, far below eps, zero, not finite."""
    G = gradient(7, m, n, torch.float32, dev)
    G[0] *= 1e-37 / 0.02
    G[1] = G[1] * 50 * 1e37
    G[2] = 0
    got = deeppcr.deeppcr_orthogonalize(G, eps=0.0)
    check(got, oo.orthogonalize(cpu(G), eps=0.0), torch.float32)
    assert torch.all(got[2] == 0)
    low = deeppcr.deeppcr_orthogonalize(G * 1e-9)
    check(low[3:], oo.orthogonalize(cpu(G * 1e-9))[3:], torch.float32)
    G[3, 0, 0] = float("nan")
    G[4, m - 1, 2] = float("inf")
    bad = deeppcr.deeppcr_orthogonalize(G, eps=0.0)
    keep = [0, 1, 2, 5, 6]
    assert torch.equal(bad[keep], got[keep])
    assert torch.isnan(bad[3]).any() and torch.isnan(bad[4]).any()


@pytest.mark.parametrize("shape", [(16, 16), (100, 120), (30, 100), (150, 200), (40, 300), (20, 400)], ids=str)
@pytest.mark.parametrize("columns", [False, True])
def test_rows_far_below_the_others(dev, shape, columns):
    """Rows or columns 1e-2 to 1e-8 of the rest, each to its own precision or to the
    parts' floor.  X, A and B are off by up to 2^-35 an entry.  A step's effect on a
    small row is at most |a| + |X col| (1 + |b| + 2 |c| |A|) of that, with |X| and
    |A| up to 1.2 and 1.4 the factor 3.5 + 1.2 (1 + 4.8 + 5.7) < 18, and every later
    step magnifies it by at most 3.45: 18 (3.45^5 - 1) / 2.45 < 2^12 in all."""
    m, n = shape
    G = gradient(5, m, n, torch.float32, dev)
    low = slice(0, n // 8) if columns else slice(0, m // 8)
    for i, s in enumerate((1e-2, 1e-4, 1e-5, 1e-6, 1e-8)):
        (G[i].t() if columns else G[i])[low] *= s
    got, ref = cpu(deeppcr.deeppcr_orthogonalize(G, eps=0.0)), oo.orthogonalize(cpu(G), eps=0.0)
    if columns:
        got, ref = got.swapaxes(1, 2), ref.swapaxes(1, 2)
    e = oo.gain() * (2.0 ** -20 + np.sqrt(max(m, n)) * 2.0 ** -24)
    top = np.max(np.abs(ref), axis=2, keepdims=True)
    assert np.all(np.abs(got - ref)[:, low] <= (e * top + 2.0 ** (12 - 35))[:, low])
