"""The operators of a feed-forward together, as a step calls them: quantized rows and their products, routing, the experts' products
and the joining; eager, captured and replayed, on other streams, with idle rows, and in a decoder with its cache."""
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_products import STEP, whole  # noqa: E402
from tests.test_gpu_rows_quantize import inst  # noqa: E402, F401

BF16 = torch.bfloat16


class Layer:
    """Tensors of one feed-forward of experts, in 16 or in 8 bits."""

    def __init__(self, n, width, inner, experts, k, eight, seed=0, sigmoid=False):
        g, cuda = torch.Generator().manual_seed(seed), dict(device="cuda")
        self.n, self.width, self.inner, self.experts, self.k, self.eight, self.sigmoid = n, width, inner, experts, k, eight, sigmoid
        self.x = torch.randn(n, width, generator=g).to(BF16).cuda()
        self.router = (torch.randn(experts, width, generator=g) / width ** 0.5).to(BF16).cuda()
        self.bias = (torch.randn(experts, generator=g) * 0.1).cuda() if sigmoid else None
        if eight:
            self.up, self.down = whole(g, experts, 2 * inner, width), whole(g, experts, width, inner)
            self.up_scale, self.down_scale = torch.rand(experts, 2 * inner, generator=g).cuda() / (74 * width ** 0.5), torch.rand(experts, width, generator=g).cuda() / (74 * inner ** 0.5)
            self.q, self.scale = torch.empty(n, width, dtype=torch.int8, **cuda), torch.empty(n, **cuda)
            self.hq, self.h_scale = torch.empty(n * k, inner, dtype=torch.int8, **cuda), torch.empty(n * k, **cuda)
        else:
            self.up = (torch.randn(experts, 2 * inner, width, generator=g) / width ** 0.5).to(BF16).cuda()
            self.down = (torch.randn(experts, width, inner, generator=g) / inner ** 0.5).to(BF16).cuda()
        i32 = dict(dtype=torch.int32, **cuda)
        self.expert, self.place, self.token = torch.empty(n, k, **i32), torch.empty(n, k, **i32), torch.empty(n * k, **i32)
        self.start, self.weight = torch.empty(experts + 1, **i32), torch.empty(n, k, **cuda)
        self.h, self.y, self.out = torch.empty(n * k, inner, dtype=BF16, **cuda), torch.empty(n * k, width, dtype=BF16, **cuda), torch.empty(n, width, dtype=BF16, **cuda)

    def run(self, inst, stream=None):  # noqa: F811
        logits = self.x @ self.router.T
        I.maaso_expert_route(inst, logits=logits, bias=self.bias, sigmoid=self.sigmoid, expert=self.expert, weight=self.weight, start=self.start, token=self.token,
                             place=self.place, stream=stream)
        if self.eight:
            I.maaso_rows_quantize(inst, x=self.x, q=self.q, scale=self.scale, stream=stream)
            I.maaso_expert_product(inst, a=self.q, a_scale=self.scale, w=self.up, w_scale=self.up_scale, out=self.h, start=self.start, token=self.token, gated=True,
                                   stream=stream)
            I.maaso_rows_quantize(inst, x=self.h, q=self.hq, scale=self.h_scale, stream=stream)
            I.maaso_expert_product(inst, a=self.hq, a_scale=self.h_scale, w=self.down, w_scale=self.down_scale, out=self.y, start=self.start, stream=stream)
        else:
            I.maaso_expert_product(inst, a=self.x, w=self.up, out=self.h, start=self.start, token=self.token, gated=True, stream=stream)
            I.maaso_expert_product(inst, a=self.h, w=self.down, out=self.y, start=self.start, stream=stream)
        I.maaso_expert_combine(inst, y=self.y, place=self.place, weight=self.weight, out=self.out, residual=self.x, stream=stream)
        return self.out

    def expected(self):
        """In 64 bits from the experts and weights that were chosen, the inner rows rounded as the calls round them."""
        out = self.x.double()
        for e in range(self.experts):
            t, j = torch.nonzero(self.expert == e, as_tuple=True)
            if not len(t):
                continue
            a = self.x[t].double()
            up, down = self.up[e].double(), self.down[e].double()
            if self.eight:
                s = a.abs().amax(1, keepdim=True) / 127
                a, up, down = (a / s).round() * s, up * self.up_scale[e].double()[:, None], down * self.down_scale[e].double()[:, None]
            g, u = (a @ up.T).chunk(2, 1)
            h = (g * torch.sigmoid(g) * u).to(BF16).double()
            if self.eight:
                s = (h.abs().amax(1, keepdim=True) / 127).clamp(min=1e-300)
                h = (h / s).round() * s
            out = out.index_add(0, t, (h @ down.T).to(BF16).double() * self.weight[t, j].double()[:, None])
        return out

    def check(self):
        """Within a rounding of the output, and what one rounding of an inner element (to the other side, to 16 or to 8 bits) moves a sum of `inner`
        of them by: half a step each, of a random sign, four standard deviations, and the row's own roundings to 16 bits, k of them."""
        want = self.expected()
        got = self.out.double()
        largest = (got - self.x.double()).abs().amax(1, keepdim=True)
        off = (got - want).abs()
        assert (off <= STEP[BF16] * want.abs() + 3 * STEP[BF16] * largest * (self.k + 1)).all(), (off / largest).max()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n, width, inner, experts, k, sigmoid", [(1, 256, 96, 4, 2, False), (5, 128, 64, 8, 3, True), (64, 512, 208, 16, 4, False), (300, 256, 128, 5, 2, True),
                                                                  (900, 128, 48, 70, 6, False), (33, 64, 32, 2, 1, False)])
def test_layer(inst, n, width, inner, experts, k, sigmoid, eight):  # noqa: F811
    layer = Layer(n, width, inner, experts, k, eight, sigmoid=sigmoid)
    layer.run(inst)
    layer.check()
    assert I.maaso_instance_status(inst) == 0


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n", [8, 400])
def test_captured_and_replayed(inst, n, eight):  # noqa: F811
    """Two layers in a graph, replayed on other inputs, with the instance's own eager work between the replays."""
    one, two = Layer(n, 256, 96, 8, 2, eight, seed=1), Layer(n, 256, 64, 12, 3, eight, seed=2, sigmoid=True)
    other = Layer(350, 128, 64, 6, 2, not eight, seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one.run(inst)
        two.run(inst)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.x.copy_(one.run(inst))
        two.run(inst)
    for seed in range(4):
        one.x.copy_(torch.randn(n, 256, generator=torch.Generator().manual_seed(seed)).to(BF16))
        other.run(inst)
        other.check()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        one.check()
        two.check()
        kept = [t.clone() for t in (one.out, two.out, two.expert, two.place)]
        two.x.copy_(one.run(inst))
        two.run(inst)
        for a, b in zip(kept, (one.out, two.out, two.expert, two.place)):
            assert torch.equal(a, b)
    assert I.maaso_instance_status(inst) == 0


def test_other_streams(inst):  # noqa: F811
    """Calls that follow each other on unlike streams are in order; what a stream argument names is where they run."""
    layers = [Layer(500, 128, 64, 40, 4, bool(i % 2), seed=i) for i in range(4)]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(3):
        for layer, stream in zip(layers, streams):
            with torch.cuda.stream(stream):
                layer.run(inst, stream=stream)
    torch.cuda.synchronize()
    for layer in layers:
        layer.check()


def test_replays_that_the_caller_has_not_ordered(inst):  # noqa: F811
    """Two graphs that share the workspace and run at once may give wrong orders, but write nothing outside their tensors; calls behind them are right."""
    graphs, held = [], []
    for n, e, k in ((3000, 12, 2), (40000, 60, 4), (1500, 200, 3)):
        logits = torch.randn(n, e, generator=torch.Generator().manual_seed(n)).cuda()
        around = torch.full((4 * n * k,), -77, dtype=torch.int32, device="cuda")
        o = dict(expert=torch.empty(n, k, dtype=torch.int32, device="cuda"), weight=torch.empty(n, k, device="cuda"), start=torch.empty(e + 1, dtype=torch.int32, device="cuda"),
                 token=around[n * k:2 * n * k], place=torch.empty(n, k, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            I.maaso_expert_route(inst, logits=logits, **o)
        graphs.append((graph, torch.cuda.Stream()))
        held.append((logits, around, o, n, k))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for logits, around, o, n, k in held:
        assert (around[:n * k] == -77).all() and (around[2 * n * k:] == -77).all()
        assert ((o["place"] >= -1) & (o["place"] < n * k)).all()
        I.maaso_expert_route(inst, logits=logits, **o)
        best = torch.sort(logits.cpu(), dim=1, descending=True, stable=True)[1][:, :k]
        order = torch.sort(best.flatten(), stable=True)[1]
        assert torch.equal(o["expert"].cpu().long(), best) and torch.equal(o["token"].cpu().long(), order // k)
        assert torch.equal(o["place"].cpu().long().flatten()[order], torch.arange(n * k))
    assert I.maaso_instance_status(inst) == 0


def test_repeats_are_the_same_bits(inst):  # noqa: F811
    layer = Layer(700, 256, 96, 16, 4, False, seed=5)
    first = layer.run(inst).clone()
    for _ in range(5):
        assert torch.equal(layer.run(inst), first)


def test_idle_rows_of_a_step(inst):  # noqa: F811
    """Rows whose logits are all -infinity go to no expert: their output is the residual, their places are nobody's."""
    layer = Layer(40, 128, 64, 8, 2, False, seed=6)
    layer.run(inst)
    whole_out, logits = layer.out.clone(), layer.x @ layer.router.T
    logits[25:] = float("-inf")
    layer.h.fill_(3.0)
    layer.y.fill_(3.0)
    I.maaso_expert_route(inst, logits=logits, expert=layer.expert, weight=layer.weight, start=layer.start, token=layer.token, place=layer.place)
    I.maaso_expert_product(inst, a=layer.x, w=layer.up, out=layer.h, start=layer.start, token=layer.token, gated=True)
    I.maaso_expert_product(inst, a=layer.h, w=layer.down, out=layer.y, start=layer.start)
    I.maaso_expert_combine(inst, y=layer.y, place=layer.place, weight=layer.weight, out=layer.out, residual=layer.x)
    assert layer.start[-1].item() == 50 and (layer.token[50:] == -1).all() and (layer.h[50:] == 3).all() and (layer.y[50:] == 3).all()
    assert torch.equal(layer.out[25:], layer.x[25:]) and torch.equal(layer.out[:25], whole_out[:25])
    assert I.maaso_instance_status(inst) == 0


@pytest.mark.parametrize("options", [dict(experts=4), dict(experts=6, chosen=3, eight=True), dict(eight=True)])
def test_a_decoder_with_experts_and_in_8_bits(options):
    """The example's step, one by one and as replays of a graph, over a prompt, its forks and tokens."""
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
    import measure_instance as M
    m = M.Decoder(layers=2, heads=4, kv_heads=2, dim=64, vocab=500, max_len=256, **options)
    both = []
    for captured in (False, True):
        s = M.Serving(m, rows=3, pages=40, page_size=16, width=10)
        s.step(torch.arange(33, device="cuda"), s.buffers([0], 33))
        b, got = s.buffers([1, 2], 1), []
        I.maaso_kv_fork(s.inst, s.pages, parents=torch.zeros(2, dtype=torch.int32, device="cuda"), children=b["rows"])
        tokens = torch.tensor([7, 9], dtype=torch.int32, device="cuda")

        def one():
            logits = s.step(tokens, b)
            tokens.copy_(b["chosen"])
            return logits

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            one()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = one()
        for _ in range(4):
            if captured:
                graph.replay()
            else:
                out = one()
            torch.cuda.synchronize()
            assert out.isfinite().all()
            got.append((out.clone(), tokens.clone()))
            torch.randn(100, 100, device="cuda").sum()
        both.append(got)
        assert I.maaso_instance_status(s.inst) == 0
    for a, b in zip(*both):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert 0 < M.measure(m, 2, 40, 2, 16) < 1
