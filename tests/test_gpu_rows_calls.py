"""Norm, its gradient, 8-bit rows and their product as a program calls them: captured into a graph, on other streams, two at a time, on tensors past 2^31 and 2^32 bytes.
Needs an MI355X (-m gpu)."""
import pytest
import torch

from tests.test_gpu_rows import BF16, E4M3, EPS, F32, U, _operands, _rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


def _bits(t):
    return t.contiguous().view(torch.uint8) if t.numel() else t


def _same(a, b):
    return all((x is None and y is None) or torch.equal(_bits(x), _bits(y)) for x, y in zip(a, b))


class Layer:
    """A gated layer in 8 bits, forward, and the gradient of its norm: every call into tensors that the program keeps, or that it makes."""

    def __init__(self, dev, tokens, width, hidden, kept):
        self.dev, self.kept = dev, kept
        self.x, self.r, self.g = (_rows_of(i, tokens, width, BF16) for i in (1, 2, 3))
        self.w = (1 + 0.1 * torch.randn(width, device="cuda")).to(BF16)
        self.up, self.down = (dev.quantize(_rows_of(i, *s, BF16, s[1] ** -0.5), tall=128) for i, s in ((4, (2 * hidden, width)), (5, (width, hidden))))
        self.hidden = hidden
        e = lambda *s, t=BF16: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
        blocks = lambda n: -(-n // 128)  # noqa: E731
        self.room = dict(out=e(tokens, width, t=E4M3), scale=e(tokens, blocks(width), t=F32), total=e(tokens, width), both=e(tokens, 2 * hidden), gated=e(tokens, hidden, t=E4M3),
                         gated_scale=e(tokens, blocks(hidden), t=F32), y=e(tokens, width), dx=e(tokens, width), dw=e(width, t=F32),
                         work=torch.empty(max(1, dev.norm_grad_workspace(self.x)), dtype=torch.uint8, device="cuda"))

    def __call__(self, stream=None):
        d, k = self.dev, self.room if self.kept else {}
        n = d.norm(self.x, self.w, EPS, residual=self.r, eight=True, out=k.get("out"), scale=k.get("scale"), total=k.get("total"), stream=stream)
        both = d.gemm_scaled(n.out, n.scale, *self.up, out=k.get("both"), stream=stream)
        z = d.quantize(both[:, self.hidden:], gate=both[:, :self.hidden], out=k.get("gated"), scale=k.get("gated_scale"), stream=stream)
        y = d.gemm_scaled(z.out, z.scale, *self.down, out=k.get("y"), stream=stream)
        dx, dw = d.norm_grad(n.total, self.w, self.g, EPS, extra=y, dx=k.get("dx"), dweight=k.get("dw"), workspace=k.get("work"), stream=stream)
        return n.out, n.scale, n.total, both, z.out, z.scale, y, dx, dw


SIZES = [(1, 256, 128), (16, 1024, 512), (130, 512, 1408), (4400, 2048, 2304)]


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("tokens, width, hidden", SIZES)
def test_captured(dev, tokens, width, hidden, kept):
    """Replays with new inputs, eager calls and synchronizations between them: each gives what the eager call gives."""
    layer = Layer(dev, tokens, width, hidden, kept)
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = layer()
    eager = Layer(dev, tokens, width, hidden, False)
    for i in range(4):
        for t, mine in zip((layer.x, layer.r, layer.g), (eager.x, eager.r, eager.g)):
            t.copy_(_rows_of(10 + i, *t.shape, BF16))
            mine.copy_(t)
        eager.w.copy_(layer.w)
        for t in made:
            t.view(torch.uint8).fill_(0x55) if t.dtype == E4M3 else t.fill_(3)
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        assert _same(eager(), made)


def test_two_graphs_at_the_same_time(dev):
    layers = [Layer(dev, 700, 1024, 640, False) for _ in range(2)]
    layers[1].x.copy_(_rows_of(77, 700, 1024, BF16))
    want = [[t.clone() for t in layer()] for layer in layers]
    torch.cuda.synchronize()
    graphs, made, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for layer in layers:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            made.append(layer())
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert _same(made[0], want[0]) and _same(made[1], want[1])


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("tokens, width, hidden", SIZES)
def test_on_other_streams(dev, tokens, width, hidden, kept):
    """The current stream is another one than the tensors were made on; and a stream that is named, whichever is current."""
    layer = Layer(dev, tokens, width, hidden, kept)
    want = [t.clone() for t in layer()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = layer()
    s.synchronize()
    assert _same(got, want)
    got = layer(stream=s.cuda_stream)
    s.synchronize()
    assert _same(got, want)


def test_two_streams_at_the_same_time(dev):
    layers = [Layer(dev, 900, 1024, 640, False) for _ in range(2)]
    layers[1].x.copy_(_rows_of(78, 900, 1024, BF16))
    want = [[t.clone() for t in layer()] for layer in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(layers[i]())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(_same(g, want[i]) for g in got[i])


# ---- past 2^31 and 2^32 bytes

def test_rows_past_four_gigabytes(dev):
    """Norm, its gradient and 8 bits of the last rows of 5.2 GB: what they are by themselves."""
    rows, dim = 160000, 16256
    x = torch.empty((rows, dim), dtype=BF16, device="cuda")
    x[:50].normal_()
    x[50:-50] = 0.5
    x[-50:].normal_()
    w, last = torch.ones(dim, dtype=BF16, device="cuda"), x[-50:].clone()
    a, b = dev.norm(x, w, EPS, eight=True), dev.norm(last, w, EPS, eight=True)
    assert torch.allclose(a.scale[-50:], b.scale, rtol=70 * U, atol=0)
    assert (a.out[-50:].float() - b.out.float()).abs().max() <= 32   # (a step at 448)
    wide = dev.norm(x, w, EPS).out[-50:].float()
    assert torch.allclose(wide, dev.norm(last, w, EPS).out.float(), rtol=2 ** -7, atol=0)
    del a
    dx, _ = dev.norm_grad(x, w, x, EPS)
    mine, _ = dev.norm_grad(last, w, last, EPS)
    assert torch.allclose(dx[-50:].float(), mine.float(), rtol=2 ** -7, atol=1e-5)
    del dx
    for tall in (1, 128):
        q, mine = dev.quantize(x, tall=tall), dev.quantize(x[-128:].clone(), tall=tall)
        assert torch.equal(q.scale[-(128 // tall):], mine.scale) and torch.equal(_bits(q.out[-128:]), _bits(mine.out))
        del q


@pytest.mark.parametrize("m, n, k, few", [(290000, 136, 8192, 40), (600, 300000, 8192, 40), (66000, 33000, 128, 30)])
def test_products_past_two_gigabytes(dev, m, n, k, few):
    """A, w or the product of more than 2^31 bytes: the last rows and columns are those of the last operands' rows by themselves."""
    a, sa, w, sw = _operands(5, few, 256, k, True)
    big_a = torch.zeros((m, k), dtype=torch.uint8, device="cuda").view(E4M3)
    big_w = torch.zeros((n, k), dtype=torch.uint8, device="cuda").view(E4M3)
    scale_a, scale_w = torch.ones((m, -(-k // 128)), device="cuda"), torch.ones((-(-n // 128), -(-k // 128)), device="cuda")
    big_a.view(torch.uint8)[-few:] = a.view(torch.uint8).cuda()
    scale_a[-few:] = sa.cuda()
    last = n // 128 * 128 - 128   # a block's first column
    big_w.view(torch.uint8)[last:last + 128] = w[:128].view(torch.uint8).cuda()
    scale_w[last // 128] = sw[0].cuda()
    got = dev.gemm_scaled(big_a, scale_a, big_w, scale_w)
    want = dev.gemm_scaled(a.cuda(), sa.cuda(), w[:128].cuda(), sw[:1].cuda())
    assert torch.equal(got[-few:, last:last + 128], want) and not got[:-few].any() and not got[-few:, :last].any()
