"""The dense-layer example: its gradients, its server step, and training through an outage.

With whole numbers, and sums that fp32 holds, forward and backward products are exact in every type that holds the factors; relu keeps them
so.  Gradients are then equal to those in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mlp():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2406_05546_amd import mlp as m
    return m


def whole(g, *shape, top):
    import torch
    return torch.randint(-top, top + 1, shape, generator=g).double()


@pytest.mark.parametrize("sizes,slots", [([5, 0, 9, 1], [1, 0, 2, 1]), ([33], [0]), ([64, 70], [2, 2])])
@pytest.mark.parametrize("widths", [(12, 20, 7), (16, 40, 24, 8)])
def test_gradients_of_whole_numbers(mlp, sizes, slots, widths):
    """Magnitudes: inputs and weights up to 2, at most 40 products a sum, three layers: below 2 (2 40)^3 < 2^20, and with
    gradients of logits up to 1 no sum of 70 rows passes 2^24 either (the last row of the asserts)."""
    import torch
    g = torch.Generator()
    g.manual_seed(len(sizes) * 100 + len(widths))
    server = mlp.MlpServer(widths, 3, 2 * len(sizes), torch.float32, "relu", state_bits=32)
    params = [whole(g, 3, *s, top=1) for s in server.shapes]
    for view, p in zip(server._parts(server.versions), params):
        view.copy_(p)
    rows, n = sum(sizes), len(widths) - 1
    x, dl = whole(g, rows, widths[0], top=2), whole(g, rows, widths[-1], top=1)
    edges = [sum(sizes[:k]) for k in range(len(sizes) + 1)]
    offsets, version = torch.tensor(edges, dtype=torch.int32).cuda(), torch.tensor(slots, dtype=torch.int32).cuda()
    logits, kept = server.forward(x.float().cuda(), offsets, version)
    first = server.backward(dl.float().cuda(), kept, offsets, version)
    again = server.backward(dl.float().cuda(), kept, offsets, version)
    assert (first, again, server.pending) == (range(len(sizes)), range(len(sizes), 2 * len(sizes)), 2 * len(sizes))
    with pytest.raises(RuntimeError):
        server.backward(dl.float().cuda(), kept, offsets, version)
    got = [t.cpu().double() for t in server._parts(server.queue)]
    assert torch.equal(server.queue[:len(sizes)], server.queue[len(sizes):])
    for k, slot in enumerate(slots):
        s = slice(edges[k], edges[k + 1])
        inputs, gates, h = [], [], x[s]
        for i in range(n):
            inputs.append(h)
            z = h @ params[2 * i][slot].t() + params[2 * i + 1][slot]
            gates.append((z > 0).double() if i + 1 < n else torch.ones_like(z))
            h = z * gates[-1]
        assert torch.equal(logits[s].cpu().double(), h)
        d = dl[s]
        for i in reversed(range(n)):
            d = d * gates[i]
            want_w, want_b = d.t() @ inputs[i], d.sum(0)
            assert (d.abs().t() @ inputs[i].abs()).max() < 2 ** 24 if len(d) else True  # the sums are exact in any order
            assert torch.equal(got[2 * i][k], want_w) and torch.equal(got[2 * i + 1][k], want_b)
            d = d @ params[2 * i][slot]
    server.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_takes_all_pending_gradients_and_publishes(mlp, bits):
    """The first step from empty states: m / (1 - beta1) = g and the root of v / (1 - beta2) = |g|, so that every weight moves by lr
    g / (|g| + eps).  Roundings, all in 32 bits: the sum of n rows n, the scale, m, v, root, quotient, two corrections and the
    products with lr about 16 steps of 2^-24 of lr; p's two differences 2^-24 of p each, and decay's two products of lr decay p."""
    import torch
    server = mlp.MlpServer((24, 40, 10), 2, 6, torch.bfloat16, "gelu", state_bits=bits, weight_decay=0.1)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    server.queue.normal_(generator=g)
    before = server.master.clone()
    server.pending, lr, eps = 5, 1e-2, 1e-8
    assert server.apply(lr) == 5 and server.pending == 0 and server.apply(lr) == 0 and server.steps == 1
    mean = server.queue[:5].double().sum(0) / 5
    for old, new, grad, shape in zip(server._parts(before), server._parts(server.master), server._parts(mean), server.shapes):
        decay = 0.1 if len(shape) == 2 else 0.0
        old = old.double()
        want = old - lr * decay * old - lr * grad / (grad.abs() + eps)
        # a sum that nearly cancels is off by 5 steps of its terms, but moves g / |g| only where it is near eps or its sign may turn
        sure = grad.abs() > 1e-4
        assert sure.float().mean() > 0.9
        off = (new.double() - want).abs()
        assert (off[sure] <= 2.0 ** -24 * (3 * want.abs() + 20 * lr)[sure]).all()
    assert torch.equal(server.fresh, server.master.bfloat16())
    assert not torch.equal(server.versions[1], server.fresh)
    server.pull(1)
    assert torch.equal(server.versions[1], server.fresh) and not torch.equal(server.versions[0], server.fresh)
    server.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_training_through_an_outage(mlp, bits):
    """The teacher's ten classes begin near ln 10 = 2.3 of loss; learning takes it below half of that, and while the server is down nothing is
    learned."""
    losses = mlp.train(rounds=60, state_bits=bits)
    assert len(losses) == 60 and all(l == l for l in losses)
    assert losses[-1] < 0.5 * losses[0]


def test_a_buffer_of_one_gradient(mlp):
    import torch
    server = mlp.MlpServer((8, 3), 1, 1, torch.float32, "relu")
    offsets, version = torch.tensor([0, 4], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    loss = server.work(torch.ones(4, 8).cuda(), torch.tensor([0, 1, 2, 0]).cuda(), offsets, version)
    assert loss.shape == (1,) and server.apply(1e-3) == 1
    server.close()


def test_an_outage_leaves_the_weights_alone_and_piles_gradients_up(mlp, monkeypatch):
    """Rounds 3 to 5 without the server: the buffer grows by a gradient for each worker, master weights, published weights and versions keep
    their bytes, and the first round after takes all that piled up in one step."""
    import torch
    log, servers = [], []

    class Watched(mlp.MlpServer):
        def __init__(self, *a, **k):
            super().__init__(*a, **k)
            servers.append(self)

        def work(self, *a):
            before = [t.clone() for t in (self.master, self.fresh, self.versions)]
            loss = super().work(*a)
            assert all(torch.equal(t, b) for t, b in zip((self.master, self.fresh, self.versions), before))
            log.append(("work", self.pending, before))
            return loss

        def apply(self, lr, mean=True):
            n = super().apply(lr, mean)
            log.append(("apply", n, self.steps))
            return n
    monkeypatch.setattr(mlp, "MlpServer", Watched)
    workers, down = 6, range(3, 6)
    mlp.train(rounds=8, down=down, workers=workers, batch=8, widths=(32, 48, 5))
    rounds = [e for e in log if e[0] == "work"]
    assert [e[1] for e in rounds] == [workers * n for n in (1, 1, 1, 1, 2, 3, 4, 1)]
    assert [e[1:] for e in log if e[0] == "apply"] == [(workers, 1), (workers, 2), (workers, 3), (4 * workers, 4), (workers, 5)]
    for r in range(8):
        same = [torch.equal(a, b) for a, b in zip(rounds[r][2], rounds[r - 1][2])] if r else [False]
        assert all(same) if r in range(4, 7) else not any(same[:2])
    assert len(servers) == 1
