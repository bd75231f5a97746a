"""The dense-layer example on tokens and with activations kept in 8 bits: embedding, layers, checkpoints, log probabilities and the server's step
run together, against the same network in 64 bits.

Tolerances.  Everything is in fp32, so a result's error is a few hundred steps of 2^-24 of the sums that it is made of (below 64 terms, three layers,
slopes below 1.13): 1e-4 of a tensor's norm leaves a factor of ten.  With activations in 8 bits the reference is a network whose
backward pass reads what is held in 8 bits, by the definition, from its own pre-activations in 64 bits; those that lie within fp32's error
of a border between two codes may be held as the other one.  A code is off by a step of 2^-3 then, for one value in 2^-3 / 2^-20 = 1e5,
which is none or one of those here and changes a gradient by less than 2^-3 / sqrt(values) of its norm: 1e-2."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mlp():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2406_05546_amd import mlp as m
    return m


def phi(z):
    import torch
    return 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)


def held(x):
    """What 8 bits hold of x."""
    import torch
    from tests.test_gpu_checkpoint import encode64, values_of_e4m3
    code, scale = encode64(x)
    value = torch.cat([values_of_e4m3(), torch.tensor([float("nan")], dtype=torch.float64)])[(code & 127).long()] * torch.where(code > 127, -1.0, 1.0)
    return value * torch.exp2(scale.double() - 127).repeat_interleave(32, 1)[:, :x.shape[1]]


def reference(params, x, labels, vocab, context, n, checkpoint):
    """Loss and gradients of one worker (mean over its rows), and the logits."""
    import math
    import torch
    table = params[0]
    dim = table.shape[1]
    there = ((x >= 0) & (x < vocab))[:, :, None]
    h = (torch.where(there, table[x.clamp(0, vocab - 1)], 0.0) * dim ** 0.5).reshape(len(x), context * dim)
    inputs, pres = [], []
    for i in range(n):
        w, b = params[1 + 2 * i], params[2 + 2 * i]
        inputs.append(h)
        z = h @ w.t() + b
        pres.append(z)
        h = z * phi(z) if i + 1 < n else z
    log_p = torch.log_softmax(h, 1)
    keep = labels >= 0
    loss = -(log_p.gather(1, labels.clamp(min=0)[:, None])[:, 0] * keep).sum() / max(1, len(x))
    d = torch.exp(log_p)
    d[torch.arange(len(x)), labels.clamp(min=0)] -= 1.0
    d = d * keep[:, None] / max(1, len(x))
    grads = [None] * len(params)
    for i in reversed(range(n)):
        z = pres[i]
        if checkpoint:
            z = held(z) if i + 1 < n else z
            before = held(pres[i - 1]) if i else None
            inputs[i] = before * phi(before) if i else held(inputs[0])
        if i + 1 < n:
            d = d * (phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        grads[1 + 2 * i], grads[2 + 2 * i] = d.t() @ inputs[i], d.sum(0)
        d = d @ params[1 + 2 * i]
    dt = torch.zeros_like(table)
    flat, rows = x.reshape(-1), (d.reshape(-1, dim) * dim ** 0.5)
    ok = (flat >= 0) & (flat < vocab)
    dt.index_add_(0, flat[ok], rows[ok])
    grads[0] = dt
    return loss, grads, h


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("sizes,slots", [([5, 0, 9, 1], [1, 0, 2, 1]), ([40, 33], [2, 0])])
def test_gradients(mlp, sizes, slots, checkpoint):
    import torch
    vocab, context, widths = 30, 4, (40, 64, 33, 12)
    server = mlp.MlpServer(widths, 3, 2 * len(sizes), torch.float32, "gelu", state_bits=32, vocab=vocab, context=context, checkpoint=checkpoint)
    assert server.shapes[0] == (30, 10) and server.shapes[1] == (64, 40)
    g = torch.Generator().manual_seed(len(sizes))
    params = [torch.randn(3, *s, generator=g) * (s[1] ** -0.5 if len(s) == 2 else 0.1) for s in server.shapes]
    for view, p in zip(server._parts(server.versions), params):
        view.copy_(p)
    rows = sum(sizes)
    x, labels = torch.randint(-1, vocab + 1, (rows, context), generator=g), torch.randint(0, widths[-1], (rows,), generator=g)
    labels[3] = -100
    edges = [sum(sizes[:k]) for k in range(len(sizes) + 1)]
    offsets, version = torch.tensor(edges, dtype=torch.int32).cuda(), torch.tensor(slots, dtype=torch.int32).cuda()
    logits, kept = server.forward(x.cuda(), offsets, version)
    loss = server.work(x.cuda(), labels.cuda(), offsets, version)
    assert server.pending == len(sizes)
    got = [t.cpu().double() for t in server._parts(server.queue)]
    for k, slot in enumerate(slots):
        s = slice(edges[k], edges[k + 1])
        want_loss, want, h = reference([p[slot].double() for p in params], x[s], labels[s], vocab, context, 3, checkpoint)
        assert (logits[s].cpu().double() - h).norm() <= 1e-4 * h.norm()
        assert abs(loss[k].item() - want_loss.item()) <= 1e-4 * (1 + abs(want_loss.item()))
        for a, b in zip(got, want):
            assert (a[k] - b).norm() <= (1e-2 if checkpoint else 1e-4) * b.norm(), tuple(b.shape)
    server.close()


def test_what_is_kept(mlp):
    """A checkpointed network keeps a byte and a thirty-second for each activation, and no layer's input but the first."""
    import torch
    from paper_2406_05546_amd import dense
    server = mlp.MlpServer((64, 128, 96, 10), 1, 2, vocab=50, context=4, checkpoint=True)
    offsets, version = torch.tensor([0, 20], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    x = torch.randint(0, 50, (20, 4)).cuda()
    _, kept = server.forward(x, offsets, version)
    assert kept[0] is x and [type(v) for layer in kept[1:] for v in layer] == [dense.Checkpoint] * 5 + [type(None)]
    assert kept[1][1] is kept[2][0] and kept[2][1] is kept[3][0]
    server.close()


@pytest.mark.parametrize("vocab,checkpoint", [(64, False), (64, True), (0, True)])
def test_training_runs(mlp, vocab, checkpoint):
    losses = mlp.train(rounds=12, down=range(4, 6), workers=5, batch=16, widths=(64, 96, 10), vocab=vocab, checkpoint=checkpoint)
    assert len(losses) == 12 and all(l == l and l < 100 for l in losses)


def test_a_round_on_bfloat16_in_a_graph(mlp):
    """Forward and backward passes of a round captured and replayed on other tokens and weights."""
    import torch
    server = mlp.MlpServer((64, 128, 1000), 2, 4, vocab=200, context=8, checkpoint=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    offsets, version = torch.tensor([0, 30, 50], dtype=torch.int32).cuda(), torch.tensor([1, 0], dtype=torch.int32).cuda()
    x, dl = torch.randint(0, 200, (50, 8), device="cuda", generator=g), torch.randn(50, 1000, device="cuda", generator=g).bfloat16()

    def run():
        server.pending = 0
        logits, kept = server.forward(x, offsets, version)
        server.backward(dl, kept, offsets, version)
        return logits
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = run()
    for _ in range(3):
        x.copy_(torch.randint(-1, 201, (50, 8), device="cuda", generator=g))
        server.versions.normal_(0, 0.1, generator=g)
        graph.replay()
        torch.cuda.synchronize()
        mine, queue = logits.clone(), server.queue[:2].clone()
        assert torch.equal(run(), mine) and torch.equal(server.queue[:2], queue)
    server.close()
