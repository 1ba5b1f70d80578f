"""The calls around a compressed gradient as a data-parallel training step makes them: lookup, the embedding's gradient
into the flat gradient, compression by every worker, the receiver's average, and the orthogonalised update of the matrices;
against the same step in 64 bits, from a graph, and from two streams at once."""
import numpy as np
import pytest

from tests.gpu_harness import Device
from tests.test_gpu_orthogonal import exact, view

pytestmark = pytest.mark.gpu

VOCABULARY, WIDTH, HIDDEN, CHUNK = 211, 48, 72, 1 << 12
LR, BETA, DECAY = 0.05, 0.9, 0.01


@pytest.fixture(scope="module")
def dev():
    return Device()


class Model:
    """logits = lookup(tokens) W1 W2; the flat vectors hold the table, W1 and W2 behind each other (odd offsets)"""

    def __init__(self, dev, workers, seed):
        torch, f = dev.torch, dev.f
        self.dev, self.workers = dev, workers
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.at1 = VOCABULARY * WIDTH + 1
        self.at2 = self.at1 + WIDTH * HIDDEN + 3
        self.n = self.at2 + HIDDEN * 10
        self.weights = torch.randn(self.n, device="cuda", generator=gen) * 0.3
        self.momentum = torch.zeros(self.n, device="cuda")
        self.listing = f.matrices([f.Matrix(self.at1, WIDTH, HIDDEN), f.Matrix(self.at2, HIDDEN, 10, gain=1.5)])
        self.tokens = [torch.randint(-1, VOCABULARY, (37 + 5 * w,), device="cuda", generator=gen) for w in range(workers)]
        self.target = [torch.randn(t.numel(), 10, device="cuda", generator=gen) for t in self.tokens]
        self.flat = [torch.zeros(self.n, device="cuda") for _ in range(workers)]
        self.out = [torch.empty(t.numel(), WIDTH, device="cuda") for t in self.tokens]
        nb = f.packed_bytes(self.n, CHUNK, 1.0, 32)
        self.packed = [torch.zeros(nb, dtype=torch.uint8, device="cuda") for _ in range(workers)]
        self.mean = torch.zeros(self.n, device="cuda")
        self.ws = dev.workspace(max(f.workspace_bytes_accumulate(self.n, CHUNK, 32, workers), f.workspace_bytes(self.n, CHUNK, 32)))
        self.ws_e = [dev.workspace(f.workspace_bytes_embedding(VOCABULARY, WIDTH, t.numel())) for t in self.tokens]
        self.ws_o = dev.workspace(f.workspace_bytes_orthogonal(self.listing))

    def parts(self, flat):
        return (flat[:VOCABULARY * WIDTH].view(VOCABULARY, WIDTH), flat[self.at1:self.at1 + WIDTH * HIDDEN].view(WIDTH, HIDDEN),
                flat[self.at2:self.at2 + HIDDEN * 10].view(HIDDEN, 10))

    def gradients(self):
        """every worker's flat gradient of the mean squared error"""
        f = self.dev.f
        table, w1, w2 = self.parts(self.weights)
        for w in range(self.workers):
            f.embedding(table, self.tokens[w], self.out[w], 2.0)
            x = self.out[w]
            h = x @ w1
            d = (h @ w2 - self.target[w]) / x.shape[0]
            g_table, g1, g2 = self.parts(self.flat[w])
            g2.copy_(h.t().contiguous() @ d)
            dh = d @ w2.t().contiguous()
            g1.copy_(x.t().contiguous() @ dh)
            f.embedding_gradient(dh @ w1.t().contiguous(), self.tokens[w], g_table, self.ws_e[w], 2.0)

    def exchange(self):
        f = self.dev.f
        for w in range(self.workers):
            f.compress(self.flat[w], CHUNK, 1.0, 32, self.packed[w], self.ws)     # all bins, 32 bits: only rounding is lost
        f.decompress_accumulate(self.packed, self.packed[0].numel(), 1.0 / self.workers, self.mean, CHUNK, 1.0, 32, self.ws)

    def update(self):
        self.dev.f.orthogonal_step(self.mean, self.momentum, self.weights, self.listing, self.ws_o, LR, BETA, DECAY)
        n = VOCABULARY * WIDTH
        self.weights[:n].add_(self.mean[:n], alpha=-LR)                            # the table's rows: plain descent

    def step(self):
        self.gradients()
        self.exchange()
        self.update()


def reference(model):
    """the step in 64 bits from the model's present state: (mean gradient, momentum, weights, errors allowed of the last two)"""
    torch = model.dev.torch
    weights = model.weights.double()
    table, w1, w2 = (p.detach().clone().requires_grad_() for p in model.parts(weights))
    loss = 0
    for w in range(model.workers):
        inside = model.tokens[w] >= 0
        x = 2.0 * table[torch.where(inside, model.tokens[w], 0)] * inside[:, None]
        loss = loss + ((x @ w1 @ w2 - model.target[w].double()) ** 2).sum() / x.shape[0] / 2
    (loss / model.workers).backward()
    mean = torch.zeros(model.n, dtype=torch.float64, device="cuda")
    for part, p in zip(model.parts(mean), (table, w1, w2)):
        part.copy_(p.grad)
    return mean


def test_a_step_of_three_workers(dev):
    torch = dev.torch
    model = Model(dev, 3, 1)
    for _ in range(3):
        want = reference(model)
        before, momentum = model.weights.clone(), model.momentum.clone()
        model.gradients()
        model.exchange()
        # binary32 products of up to 72 terms three deep, sums over 37 rows and the codec's 1e-5: 3e-5 of the gradient's norm
        assert float(torch.linalg.vector_norm(model.mean.double() - want)) <= 3e-5 * float(torch.linalg.vector_norm(want))
        mean = model.mean.clone()
        model.update()
        keep = 1.0 - float(np.float32(LR)) * float(np.float32(DECAY))
        for m in model.listing.array:
            got_m = view(torch, model.momentum, m).double()
            want_m = float(np.float32(BETA)) * view(torch, momentum, m).double() + view(torch, mean, m).double()
            assert bool(((got_m - want_m).abs() <= 2.0 ** -24 * 1.01 * want_m.abs()).all())
            o, bound = exact(torch, (view(torch, mean, m).double() + float(np.float32(BETA)) * got_m).float())
            want_w = keep * view(torch, before, m).double() - float(np.float32(LR)) * m.gain * o
            err = float(torch.linalg.vector_norm(view(torch, model.weights, m).double() - want_w))
            assert err <= LR * m.gain * bound + 2.0 ** -22 * float(torch.linalg.vector_norm(want_w))
        gaps = [VOCABULARY * WIDTH, *range(model.at1 + WIDTH * HIDDEN, model.at2)]
        assert torch.equal(model.weights[gaps], before[gaps]) and bool((model.momentum[gaps] == 0).all())


def test_gradients_agree_with_differences(dev):
    """the flat gradient against the loss's differences along a random direction, both from the calls here"""
    torch, f = dev.torch, dev.f
    model = Model(dev, 1, 2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    direction = torch.randn(model.n, device="cuda", generator=gen)
    model.gradients()
    slope = float((model.flat[0].double() * direction.double())[torch.cat([torch.arange(a, b, device="cuda") for a, b in (
        (0, VOCABULARY * WIDTH), (model.at1, model.at1 + WIDTH * HIDDEN), (model.at2, model.n))])].sum())

    def loss(h):
        table, w1, w2 = model.parts(model.weights + h * direction)
        x = torch.empty_like(model.out[0])
        f.embedding(table.contiguous(), model.tokens[0], x, 2.0)
        return float((((x.double() @ w1.double() @ w2.double() - model.target[0].double()) ** 2).sum() / x.shape[0] / 2))

    h = 1e-3
    # a polynomial of degree six in h: the central difference is off by h^2 / 6 of the third derivative, and the values' 2^-24
    # by 2^-24 / h; the richer difference takes the first away
    central = lambda s: (loss(s) - loss(-s)) / (2 * s)
    rich = (4 * central(h) - central(2 * h)) / 3
    assert abs(rich - slope) <= 1e-3 * abs(slope), (rich, slope)


def test_a_captured_step_replays(dev):
    torch, f = dev.torch, dev.f
    model, twin = Model(dev, 2, 4), Model(dev, 2, 4)
    model.step()                                           # what is created on first use is there
    twin.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gen = torch.Generator(device="cuda").manual_seed(9)
    # the library's calls only: torch's products stay outside, the gradients are given
    grads = [torch.randn(t.numel(), WIDTH, device="cuda", generator=gen) for t in model.tokens]
    rows = [torch.empty(t.numel(), WIDTH, device="cuda") for t in model.tokens]

    def calls(m):
        for w in range(m.workers):
            f.embedding(m.parts(m.weights)[0], m.tokens[w], rows[w], 2.0)
            f.embedding_gradient(grads[w], m.tokens[w], m.parts(m.flat[w])[0], m.ws_e[w], 2.0)
            f.embedding_gradient(grads[w], m.tokens[w], m.parts(m.flat[w])[0], m.ws_e[w], 0.5, base=m.parts(m.flat[w])[0])
        m.exchange()
        f.orthogonal_step(m.mean, m.momentum, m.weights, m.listing, m.ws_o, LR, BETA, DECAY)
        f.orthogonal(m.weights, m.weights, m.listing, m.ws_o)

    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            calls(model)
    torch.cuda.synchronize()
    for replay in range(4):
        for w in range(2):
            grads[w].normal_(generator=gen)
            model.tokens[w].random_(-1, VOCABULARY, generator=gen)
            twin.tokens[w].copy_(model.tokens[w])
        model.ws_o.fill_(0xFF)
        for ws in model.ws_e:
            ws.fill_(0xFF)
        calls(twin)
        eager = [r.clone() for r in rows]
        torch.cuda.synchronize()
        for r in rows:
            r.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for w in range(2):
            assert torch.equal(rows[w], eager[w]), replay
            assert torch.equal(model.flat[w], twin.flat[w]), replay
        assert torch.equal(model.momentum, twin.momentum) and torch.equal(model.weights, twin.weights), replay


def test_sorted_and_sliced_calls_replay_from_a_graph(dev):
    """the larger forms: places that are sorted by several workgroups, tiles whose steps several workgroups share"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(10)
    tokens = torch.randint(-1, 3000, (20000,), device="cuda", generator=gen)
    grad = torch.randn(20000, 40, device="cuda", generator=gen)
    out = torch.empty(3000, 40, device="cuda")
    ws = dev.workspace(f.workspace_bytes_embedding(3000, 40, 20000))
    listing = f.matrices([f.Matrix(0, 300, 20000), f.Matrix(6000000, 150, 9000)])
    x = torch.randn(listing.end, device="cuda", generator=gen)
    y = torch.empty_like(x)
    ws_o = dev.workspace(f.workspace_bytes_orthogonal(listing))

    def calls():
        f.embedding_gradient(grad, tokens, out, ws)
        f.orthogonal(x, y, listing, ws_o)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            calls()
    torch.cuda.synchronize()
    for replay in range(3):
        grad.normal_(generator=gen)
        tokens.random_(-1, 3000, generator=gen)
        x.normal_(generator=gen)
        calls()
        torch.cuda.synchronize()
        want = out.clone(), y.clone()
        out.fill_(1.0)
        y.fill_(1.0)
        ws.fill_(0xFF)
        ws_o.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(y, want[1]), replay


@pytest.mark.parametrize("count", [20, 150])   # a list that travels with the launch, and one that is written down first
def test_steps_of_small_matrices_replay_from_a_graph(dev, count):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(21)
    at, ms = 0, []
    for i in range(count):
        rows, cols = 1 + 7 * i % 64, 1 + 61 * i % 700
        ms.append(f.Matrix(at, *((rows, cols) if i % 2 else (cols, rows))))
        at += rows * cols
    listing = f.matrices(ms)
    g, mom, w = (torch.randn(at, device="cuda", generator=gen) for _ in range(3))
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    f.orthogonal_step(g, mom.clone(), w.clone(), listing, ws, LR, BETA, DECAY)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            f.orthogonal_step(g, mom, w, listing, ws, LR, BETA, DECAY)
    torch.cuda.synchronize()
    for replay in range(3):
        g.normal_(generator=gen)
        want = mom.clone(), w.clone()
        f.orthogonal_step(g, *want, listing, ws, LR, BETA, DECAY)
        torch.cuda.synchronize()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mom, want[0]) and torch.equal(w, want[1]), replay


def test_two_streams_at_once(dev):
    """each with workspaces of its own; the larger forms on both"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(13)
    listing = f.matrices([f.Matrix(0, 200, 12000), f.Matrix(2400000, 500, 700)])
    jobs = []
    for k in range(2):
        tokens = torch.randint(-1, 900, (12000,), device="cuda", generator=gen)
        grad = torch.randn(12000, 64, device="cuda", generator=gen)
        x = torch.randn(listing.end, device="cuda", generator=gen)
        jobs.append(dict(tokens=tokens, grad=grad, x=x, out=torch.empty(900, 64, device="cuda"), y=torch.empty_like(x),
                         ws=dev.workspace(f.workspace_bytes_embedding(900, 64, 12000)),
                         ws_o=dev.workspace(f.workspace_bytes_orthogonal(listing)), stream=torch.cuda.Stream()))

    def run(j, stream):
        f.embedding_gradient(j["grad"], j["tokens"], j["out"], j["ws"], stream=stream)
        f.orthogonal(j["x"], j["y"], listing, j["ws_o"], stream=stream)

    want = []
    for j in jobs:
        run(j, None)
        torch.cuda.synchronize()
        want.append((j["out"].clone(), j["y"].clone()))
        j["out"].fill_(-1.0)
        j["y"].fill_(-1.0)
    torch.cuda.synchronize()
    for _ in range(5):
        for j in jobs:
            run(j, j["stream"])
    torch.cuda.synchronize()
    for j, w in zip(jobs, want):
        assert torch.equal(j["out"], w[0]) and torch.equal(j["y"], w[1])
