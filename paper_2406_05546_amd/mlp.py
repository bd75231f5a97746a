"""A network of dense layers trained the parameter server's way on the operators of `dense`: workers compute gradients on the
weight versions that they last pulled, these pile up in rows of a buffer while the server is down, and one AdamW
step takes all of them when it is back.

    python -m paper_2406_05546_amd.mlp            (a GPU is needed; a few seconds)

Everything is allocated when the server is made.  The master weights and the two states of every tensor are part of one
buffer each, a tensor beginning at a multiple of 256 elements (a block of an 8-bit state); a gradient row and a weight version
have the same layout, so the layers' operators read a version's matrices in place and write gradients where the step reads them.

With --vocab the inputs are tokens, so many of them (--context) to a row, whose vectors, rows of a table, are the first layer's
input; with --checkpoint a layer's pre-activations, in 8 bits, are all that is kept for the backward pass, which makes the next layer's input
from them again."""
from __future__ import annotations

import argparse
from typing import List, Optional, Sequence

import torch

from . import dense, tokens

_ALIGN = dense.ADAMW_BLOCK


class MlpServer:
    """widths: features of the input, of every hidden layer (with `activation`) and the logits.  The master weights are fp32, versions and
    gradients of `dtype`.  capacity: gradients that the buffer holds.  vocab: the inputs are rows of `context` tokens (0 .. vocab - 1; others
    are padding), a vector of widths[0] / context features for each.  checkpoint: what the backward pass needs is kept in 8 bits."""

    def __init__(self, widths: Sequence[int], n_versions: int, capacity: int, dtype=torch.bfloat16, activation: str = "gelu",
                 state_bits: int = 8, weight_decay: float = 0.01, seed: int = 0, device: str = "cuda:0", vocab: int = 0, context: int = 1,
                 checkpoint: bool = False):
        if len(widths) < 2 or min(widths) < 1:
            raise ValueError("widths: at least an input and an output, each with a feature or more")
        if n_versions < 1 or capacity < 1:
            raise ValueError("at least one version and room for one gradient")
        if activation not in dense.ACTIVATIONS:
            raise ValueError(f"unknown activation {activation!r}")
        if vocab < 0 or context < 1 or (vocab and widths[0] % context):
            raise ValueError("vocab: none or some tokens; widths[0]: as many features for each token of a row")
        self.vocab, self.context, self.checkpoint = vocab, context, checkpoint
        self.shapes = [(vocab, widths[0] // context)] if vocab else []
        self.layers = len(self.shapes)  # number of the first layer's weights
        for fin, fout in zip(widths, widths[1:]):
            self.shapes += [(fout, fin), (fout,)]
        self.at, total = [], 0
        for i in range(len(self.shapes)):
            self.at.append(total)
            total += -(-self._numel(i) // _ALIGN) * _ALIGN
        self.widths, self.activation, self.n_versions, self.capacity, self.pending, self.steps = list(widths), activation, n_versions, capacity, 0, 0
        self.master = torch.zeros(total, device=device)
        self.fresh = torch.zeros(total, dtype=dtype, device=device)  # the master weights, rounded: what a pull copies
        self.versions = torch.zeros(n_versions, total, dtype=dtype, device=device)
        self.queue = torch.zeros(capacity, total, dtype=dtype, device=device)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        for w, shape in zip(self._parts(self.master), self.shapes):
            if len(shape) == 2:
                w.normal_(0, shape[1] ** -0.5, generator=gen)
        self.fresh.copy_(self.master)
        self.versions.copy_(self.fresh.expand_as(self.versions))
        flat = lambda t: [t[..., a:a + self._numel(i)] for i, a in enumerate(self.at)]  # noqa: E731
        # grads with one row are gradients, not rows: a buffer of one is given as it is
        self.optimizer = dense.ps_adamw_create(flat(self.master), flat(self.queue) if capacity > 1 else flat(self.queue[0]), state_bits=state_bits,
                                               weight_decay=[weight_decay if len(s) == 2 else 0.0 for s in self.shapes], copies=flat(self.fresh))

    def _numel(self, i: int) -> int:
        n = 1
        for s in self.shapes[i]:
            n *= s
        return n

    def _parts(self, t) -> List[torch.Tensor]:
        """Views of every tensor in a flat buffer, or in each row of a matrix of them."""
        return [t[..., a:a + self._numel(i)].unflatten(-1, s) for i, (a, s) in enumerate(zip(self.at, self.shapes))]

    def pull(self, version: int) -> None:
        """Workers on this version have the server's present weights from here on."""
        self.versions[version].copy_(self.fresh)

    def forward(self, x, offsets, version_of_worker):
        """Logits [rows, out] of the workers' rows (worker g has rows offsets[g] .. offsets[g + 1] - 1 and reads version
        version_of_worker[g]), and what `backward` needs.  x: [rows, features], or tokens [rows, context] of int32 or int64."""
        parts, kept, n, at = self._parts(self.versions), [], len(self.widths) - 1, self.layers
        if self.vocab:
            kept.append(x)
            dim = self.shapes[0][1]
            x = tokens.ps_grouped_embedding_forward(x.reshape(-1), offsets * self.context, parts[0], dim ** 0.5, version_of_worker).view(x.shape[0], self.widths[0])
        held = dense.ps_checkpoint_encode(x) if self.checkpoint else x
        for i in range(n):
            pre = None
            if i + 1 < n:
                shape = x.shape[0], self.widths[i + 1]
                pre = dense.ps_checkpoint_empty(*shape, x.device) if self.checkpoint else torch.empty(shape, dtype=x.dtype, device=x.device)
            x = dense.ps_grouped_linear_forward(x, offsets, parts[at + 2 * i], parts[at + 2 * i + 1], None, "none" if pre is None else self.activation, version_of_worker, pre=pre)
            kept.append((held, pre))
            held = pre if self.checkpoint else x
        return x, kept

    def backward(self, dlogits, kept, offsets, version_of_worker) -> range:
        """Appends every worker's gradient to the buffer; returns their rows."""
        workers = offsets.numel() - 1
        if self.pending + workers > self.capacity:
            raise RuntimeError(f"the buffer holds {self.capacity} gradients, {self.pending} are pending and {workers} came")
        rows = range(self.pending, self.pending + workers)
        weights, grads, dy, at = self._parts(self.versions), self._parts(self.queue[rows.start:rows.stop]), dlogits, self.layers
        layers = kept[1:] if self.vocab else kept
        for i in reversed(range(len(layers))):
            x, pre = layers[i]
            dy, _, _ = dense.ps_grouped_linear_backward(dy, x, offsets, weights[at + 2 * i], "none" if pre is None else self.activation, pre, version_of_worker,
                                                        need_dx=i > 0 or self.vocab > 0, dw=grads[at + 2 * i], db=grads[at + 2 * i + 1],
                                                        x_activation=self.activation if self.checkpoint and i else "none")
        if self.vocab:
            dim = self.shapes[0][1]
            tokens.ps_grouped_embedding_backward(dy.view(-1, dim), kept[0].reshape(-1), offsets * self.context, self.vocab, dim ** 0.5, dtable=grads[0])
        self.pending = rows.stop
        return rows

    def work(self, x, labels, offsets, version_of_worker):
        """One minibatch of every worker: the mean cross-entropy's gradients go to the buffer; returns each worker's loss."""
        workers = offsets.numel() - 1
        logits, kept = self.forward(x, offsets, version_of_worker)
        size = (offsets[1:] - offsets[:-1]).long()
        worker = torch.repeat_interleave(torch.arange(workers, device=x.device), size, output_size=x.shape[0])
        p = tokens.ps_logprob_forward(logits, labels)
        dlogits = tokens.ps_logprob_backward(logits, labels, p.norm, (-1.0 / size)[worker], out=logits)
        self.backward(dlogits, kept, offsets, version_of_worker)
        return torch.zeros(workers, device=x.device).index_add_(0, worker, -p.logp) / size.clamp(min=1)

    def apply(self, lr: float, mean: bool = True) -> int:
        """One AdamW step with the sum (or mean) of all pending gradients, which leaves the buffer empty; returns how many there were."""
        n = self.pending
        if n:
            self.steps += 1
            dense.ps_adamw_step(self.optimizer, self.steps, lr, grad_scale=1.0 / n if mean else 1.0, n_rows=n)
            self.pending = 0
        return n

    def close(self) -> None:
        dense.ps_adamw_destroy(self.optimizer)


def train(rounds: int = 60, down: Optional[range] = None, workers: int = 16, batch: int = 64, widths: Sequence[int] = (256, 512, 512, 10),
          state_bits: int = 8, lr: float = 2e-3, seed: int = 1, dtype=torch.bfloat16, say=None, vocab: int = 0, context: int = 8,
          checkpoint: bool = False) -> List[float]:
    """Workers learn a random teacher's labels; worker g pulls every (g % 4 + 1)-th round, as far as the server is there
    (it is not in the rounds of `down`).  With `vocab` the inputs are `context` random tokens, each of which the teacher gives points to
    every class.  Returns the mean loss of every round."""
    down = range(rounds // 2, rounds // 2 + 8) if down is None else down
    server = MlpServer(widths, 4, workers * (len(down) + 1), dtype, state_bits=state_bits, seed=seed, vocab=vocab, context=context if vocab else 1,
                       checkpoint=checkpoint)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    teacher = torch.randn(vocab or widths[0], widths[-1], device="cuda", generator=gen)
    # ragged minibatches: batch, one less, two less, .. rows, and again
    sizes = [max(1, batch - g % 4) for g in range(workers)]
    offsets = torch.tensor([sum(sizes[:g]) for g in range(workers + 1)], dtype=torch.int32).cuda()
    version = torch.tensor([g % 4 for g in range(workers)], dtype=torch.int32).cuda()
    losses = []
    for r in range(rounds):
        if vocab:
            x = torch.randint(0, vocab, (sum(sizes), context), device="cuda", generator=gen)
            labels = teacher[x].sum(1).argmax(1)
        else:
            x = torch.randn(sum(sizes), widths[0], device="cuda", generator=gen)
            x, labels = x.to(dtype), (x @ teacher).argmax(1)
        loss = server.work(x, labels, offsets, version)
        losses.append(loss.mean())
        if r not in down:
            n = server.apply(lr)
            for v in range(4):
                if r % (v + 1) == 0:
                    server.pull(v)
            if say:
                say(f"round {r}: loss {losses[-1].item():.4f}, {n} gradients applied")
        elif say:
            say(f"round {r}: loss {losses[-1].item():.4f}, server down, {server.pending} gradients pending")
    server.close()
    return [v.item() for v in losses]


def main() -> None:
    p = argparse.ArgumentParser(description="trains a small network of dense layers through an outage of the parameter server")
    p.add_argument("--rounds", type=int, default=60)
    p.add_argument("--workers", type=int, default=16)
    p.add_argument("--batch", type=int, default=64)
    p.add_argument("--widths", type=int, nargs="+", default=[256, 512, 512, 10])
    p.add_argument("--state-bits", type=int, choices=[8, 32], default=8)
    p.add_argument("--vocab", type=int, default=0, help="inputs are tokens, so many different ones")
    p.add_argument("--context", type=int, default=8, help="tokens of a row")
    p.add_argument("--checkpoint", action="store_true", help="keep activations in 8 bits for the backward pass")
    a = p.parse_args()
    train(a.rounds, workers=a.workers, batch=a.batch, widths=a.widths, state_bits=a.state_bits, say=lambda m: print(m, flush=True), vocab=a.vocab,
          context=a.context, checkpoint=a.checkpoint)


if __name__ == "__main__":
    main()
