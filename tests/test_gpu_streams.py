"""Calls with a stream of their own: what the binding allocates belongs to that
stream, and memory that crosses between two streams is given out again only when
both are past it.  Nothing here depends on who wins a race: the tests look at
which stream asked for memory, and at addresses."""
import pytest

from paper_2309_16318_amd import deeppcr, generic, synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
SLEEP = 1 << 27    # cycles that keep a stream busy, some tens of milliseconds


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def calls(dev):
    """name: call(stream), for every entry point that allocates."""
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen).to(dev)
    B, L, w = 2, 600, 40
    a, u, x, g, x0 = r(B, L, w), r(B, L, w), r(B, L, w), r(B, L, w), r(B, w)
    dW = r(3, 40, 200)
    ones, rs = torch.ones(w, device=dev), torch.ones(B, L, device=dev)
    m = {k: torch.from_numpy(v).to(dev) for k, v in synth.mlp_inputs(2, 12, 16, seed=5).items()}
    W, bias, z0, G = m["W"], m["bias"], m["z0"], m["G"]
    Z = deeppcr.deeppcr_mlp_forward(W, bias, z0).Z
    R = deeppcr.deeppcr_resnet_forward(W, bias, z0, 3).Z
    J, rhs = 0.1 * r(2, 12, 16, 16), r(2, 12, 16)
    d = deeppcr
    return {
        "scan": lambda s: d.deeppcr_gated_scan_forward(a, u, x0=x0, stream=s),
        "scan_backward": lambda s: d.deeppcr_gated_scan_backward(a, u, x, g, stream=s),
        "scan_step": lambda s: d.deeppcr_gated_scan_step(a[:, 0], u[:, 0], x0.clone(), stream=s),
        "norm": lambda s: d.deeppcr_residual_norm_forward(x, g, a, ones, ones, ones, gate=1, stream=s),
        "norm_backward": lambda s: d.deeppcr_residual_norm_backward(
            x, g, rs, rs, a, u, a, ones, ones, ones, gate=1, stream=s),
        "update": lambda s: d.deeppcr_orthogonalize(dW, stream=s),
        "solve": lambda s: d.pcr_solve_block_bidiag(J, rhs, stream=s),
        "solve_chunked": lambda s: d.pcr_solve_block_bidiag_chunked(J, rhs, 3, stream=s),
        "mlp": lambda s: d.deeppcr_mlp_forward(W, bias, z0, stream=s),
        "mlp_residual": lambda s: d.deeppcr_mlp_forward_residual(W, bias, z0, stream=s),
        "mlp_backward": lambda s: d.deeppcr_mlp_backward(W, bias, z0, Z, G, stream=s),
        "newton_step": lambda s: d.deeppcr_newton_step(J, rhs, rhs.clone(), stream=s),
        "resnet": lambda s: d.deeppcr_resnet_forward(W, bias, z0, 3, stream=s),
        "resnet_backward": lambda s: d.deeppcr_resnet_backward(W, z0, R, G, 3, stream=s),
        "resnet_seq": lambda s: d.deeppcr_resnet_seq_forward(W, bias, z0, 3, stream=s),
        "resnet_seq_backward": lambda s: d.deeppcr_resnet_seq_backward(W, z0, R, G, 3, stream=s),
        "seq": lambda s: d.deeppcr_seq_forward(W, bias, z0, stream=s),
        "seq_backward": lambda s: d.deeppcr_seq_backward(W, bias, z0, Z, G, stream=s),
        "generic": lambda s: generic.newton_generic(
            lambda p: 0.5 * p, lambda p: 0.5 * torch.eye(16, device=dev).expand(2, 12, 16, 16),
            rhs[:, 0].contiguous(), 12, stream=s),
    }


def test_every_call_allocates_on_its_stream(dev, monkeypatch):
    side, asked = torch.cuda.Stream(), []

    def noted(make):
        def call(*args, **kw):
            asked.append(torch.cuda.current_stream(dev))
            return make(*args, **kw)
        return call

    everything = calls(dev)
    torch.cuda.synchronize()
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, noted(getattr(torch, name)))
    for name, call in everything.items():
        asked.clear()
        want = list(deeppcr._tensors(call(None)))
        assert all(s != side for s in asked), name
        made = len(asked)
        side.wait_stream(torch.cuda.current_stream())
        asked.clear()
        got = list(deeppcr._tensors(call(side)))
        assert len(asked) == made and all(s == side for s in asked), name
        torch.cuda.synchronize()
        assert torch.cuda.current_stream(dev) != side
        assert len(got) == len(want), name
        assert all(torch.equal(p, q) for p, q in zip(got, want)), name


def test_an_output_outlives_its_readers(dev):
    """An output that the caller's stream still reads when it is dropped is not the
    next call's memory; nor is an input that the call's stream still reads."""
    side = torch.cuda.Stream()
    a = torch.rand(2, 3000, 72, device=dev)
    torch.cuda.synchronize()
    x, last = deeppcr.deeppcr_gated_scan_forward(a, a, stream=side)
    at = x.data_ptr()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(SLEEP)          # stands for work that reads x
    del x
    y, _ = deeppcr.deeppcr_gated_scan_forward(a, a, stream=side)
    assert y.data_ptr() != at
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)      # the call will start behind it
    b = a.clone()
    side.wait_stream(torch.cuda.current_stream())
    at = b.data_ptr()
    z, _ = deeppcr.deeppcr_gated_scan_forward(b, b, stream=side)
    del b
    assert torch.empty_like(a).data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(z, y)


def test_a_stream_of_another_device_is_refused(dev):
    class Elsewhere:
        device = torch.device("cuda", 7)

    a = torch.rand(1, 4, 8, device=dev)
    with pytest.raises(ValueError):
        deeppcr.deeppcr_gated_scan_forward(a, a, stream=Elsewhere())


def test_captured_on_a_stream_beside(dev):
    """A captured graph that forks to a stream of its own for the call."""
    a = torch.rand(2, 700, 40, device=dev)
    u = torch.randn(2, 700, 40, device=dev)
    side = torch.cuda.Stream()
    deeppcr.deeppcr_gated_scan_forward(a, u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        x, last = deeppcr.deeppcr_gated_scan_forward(a, u, stream=side)
        here.wait_stream(side)
        y = 2 * x
    for _ in range(3):
        u.copy_(torch.randn_like(u))
        want = deeppcr.deeppcr_gated_scan_forward(a, u)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want[0]) and torch.equal(last, want[1]) and torch.equal(y, 2 * want[0])
