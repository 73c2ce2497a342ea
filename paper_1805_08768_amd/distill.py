"""Rounds of Alg. 1 whose clients learn from a teacher's answers, with weights and products in 4 bits.

What the paper compresses is what goes up: a client's weight update, as a sparse binary message.  Here what
goes down is small as well: the weights of the layer that the clients train are held in microscaled 4-bit
floating point (4.25 bits a weight), and instead of labels the teacher sends its top logits for every
position (8 bytes each, and the log-sum-exp that says how much of its mass they leave out).  The client's
products run in 4 bits, its loss is the divergence from the teacher, and its update goes up through
sbc_compress as in any other round.

HeldLinear, Teacher and Learner are the parts; `distilled_rounds` runs them through rounds.run_rounds on one
GPU, everything in device memory.  All arithmetic but the weights' own addition is the library's
(sbc_mxfp_*, sbc_top_logits, sbc_distill_loss, sbc_compress, sbc_decompress_average).

    python -m paper_1805_08768_amd.distill          # a small run: losses, and bytes up and down per round
"""
from __future__ import annotations

from typing import Callable, List, NamedTuple, Optional, Tuple

import torch

from . import binding as sbc
from . import rounds


class HeldLinear:
    """The weights [outputs, inputs] of a linear layer held in 4 bits."""

    def __init__(self, outputs: int, inputs: int, device: str = "cuda:0"):
        self.q = sbc.Mxfp(outputs, inputs, device=device)

    def hold(self, weight: torch.Tensor) -> "HeldLinear":
        sbc.sbc_mxfp_quantize(weight, self.q)
        return self

    def values(self, out: torch.Tensor) -> torch.Tensor:
        """The weights as they are held: what a client has after the download."""
        sbc.sbc_mxfp_dequantize(self.q, out)
        return out

    def __call__(self, x: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
        """out = Q(x) w^T for one row of x or many."""
        sbc.sbc_mxfp_linear(x, self.q, out)
        return out

    @property
    def nbytes(self) -> int:
        return sbc.sbc_mxfp_bytes(self.q.rows, self.q.cols)


class Answers(NamedTuple):
    """A teacher's answers for a batch: places and values of its top logits, and the log-sum-exp of all."""
    index: torch.Tensor
    top: torch.Tensor
    lse: torch.Tensor

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self)


class Teacher:
    """A layer from hidden states to logits, held in 4 bits, that answers with its k largest logits."""

    def __init__(self, weight: torch.Tensor, k: int, temperature: float):
        self.vocab, self.hidden = weight.shape
        self.k, self.temperature = int(k), float(temperature)
        self.layer = HeldLinear(self.vocab, self.hidden, str(weight.device)).hold(weight)

    def answer(self, hidden: torch.Tensor) -> Answers:
        """Answers for hidden states [positions, hidden]; one position (serving) as many."""
        rows, device = hidden.shape[0], hidden.device
        logits = torch.empty(rows, self.vocab, dtype=hidden.dtype, device=device)
        self.layer(hidden, logits)
        answers = Answers(torch.empty(rows, self.k, dtype=torch.int32, device=device),
                          torch.empty(rows, self.k, dtype=torch.float32, device=device),
                          torch.empty(rows, dtype=torch.float32, device=device))
        sbc.sbc_top_logits(logits, answers.index, answers.top, answers.lse, self.temperature)
        return answers


class Learner:
    """A client's local training: `steps` steps of gradient descent on the layer from the weights it downloaded,
    against a teacher's answers; hidden states in float32.  Buffers are made once."""

    def __init__(self, vocab: int, hidden: int, positions: int, temperature: float, lr: float, steps: int = 1, device: str = "cuda:0"):
        self.temperature, self.lr, self.steps = float(temperature), float(lr), int(steps)
        new = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=device)  # noqa: E731
        self.layer = HeldLinear(vocab, hidden, device)
        self.weight, self.dweight = new(vocab, hidden), new(vocab, hidden)
        self.logits, self.loss = new(positions, vocab), new(positions)
        self.grad_cols = sbc.Mxfp(vocab, positions, device=device)
        self.hidden_cols = sbc.Mxfp(hidden, positions, device=device)

    def gradient(self, hidden: torch.Tensor, answers: Answers, share: torch.Tensor) -> torch.Tensor:
        """dL/dw at self.weight for L = sum(share * loss): products in 4 bits, the logits' gradient in their place."""
        self.layer.hold(self.weight)(hidden, self.logits)
        sbc.sbc_distill_loss(self.logits, answers.index, answers.top, self.temperature, self.loss, grad=self.logits,
                             teacher_lse=answers.lse, weight=share)
        sbc.sbc_mxfp_quantize(self.logits, None, self.grad_cols)
        sbc.sbc_mxfp_matmul(self.grad_cols, self.hidden_cols, self.dweight)
        return self.dweight

    def train(self, weight: torch.Tensor, hidden: torch.Tensor, answers: Answers, share: torch.Tensor, out: torch.Tensor) -> None:
        """Writes the update of the weights into `out`: local weights after training minus the downloaded ones.  `weight`
        are the server's; what is trained from is what 4 bits hold of them.  share[positions]: each position's weight in
        the loss, 0 for padding."""
        self.layer.hold(weight).values(self.weight)
        out.copy_(self.weight).neg_()
        sbc.sbc_mxfp_quantize(hidden, None, self.hidden_cols)
        for _ in range(self.steps):
            self.weight.add_(self.gradient(hidden, answers, share), alpha=-self.lr)
        out.add_(self.weight)


def distilled_rounds(teacher: Teacher, hidden: List[torch.Tensor], p: float, n_rounds: int, lr: float, steps: int = 1,
                     weight: Optional[torch.Tensor] = None, share: Optional[List[torch.Tensor]] = None,
                     on_loss: Optional[Callable[[int, int, torch.Tensor], None]] = None) -> Tuple[torch.Tensor, List[int], int]:
    """n_rounds of Alg. 1 with one client for each of `hidden` (its positions' hidden states, [positions, hidden] each), which
    learn teacher's layer.  weight: the server's first weights [vocab, hidden] (default zeros); share: per client,
    the positions' weights in its loss (default 1 / positions).  on_loss(round, client, losses of the last local step): called
    on the client's stream with the learner's own buffer, which its next step overwrites.
    Returns the final weights, the bytes uploaded per round, and the bytes that the client with the most positions downloads
    for a round with its answers."""
    vocab, width = teacher.vocab, teacher.hidden
    device = str(hidden[0].device)
    if share is None:
        share = [torch.full((h.shape[0],), 1.0 / h.shape[0], device=device) for h in hidden]
    answers = [teacher.answer(h) for h in hidden]
    learners = [Learner(vocab, width, h.shape[0], teacher.temperature, lr, steps, device) for h in hidden]
    down = max(learner.layer.nbytes + a.nbytes for learner, a in zip(learners, answers))

    def local_update(client, rnd, W, out):
        learner = learners[client]
        learner.train(W[0].view(vocab, width), hidden[client], answers[client], share[client], out[0].view(vocab, width))
        if on_loss is not None:
            on_loss(rnd, client, learner.loss)

    start = None if weight is None else [weight.detach().reshape(-1).float().cpu().numpy()]
    W, uploaded = rounds.run_rounds([vocab * width], p, len(hidden), n_rounds, local_update, weights=start, device=device, on_device=True)
    return W[0].view(vocab, width), uploaded, down


def main() -> None:
    vocab, width, positions, clients, n_rounds = 10000, 200, 700, 4, 10
    g = torch.Generator(device="cuda:0").manual_seed(7)
    normal = lambda *s: torch.empty(*s, device="cuda:0").normal_(generator=g)  # noqa: E731
    teacher = Teacher(normal(vocab, width) * (2.0 / width ** 0.5), k=32, temperature=2.0)
    hidden = [normal(positions, width) for _ in range(clients)]
    seen = {}

    def on_loss(rnd, client, loss):
        seen.setdefault(rnd, []).append(loss.sum())

    _, uploaded, down = distilled_rounds(teacher, hidden, p=0.01, n_rounds=n_rounds, lr=3000.0, on_loss=on_loss)
    for rnd in range(n_rounds):
        mean = float(torch.stack(seen[rnd]).mean())
        print("round %2d: loss %.4f, up %d bytes a client, down %d (dense fp32: %d)" % (rnd, mean, uploaded[rnd] // clients, down, 4 * vocab * width))


if __name__ == "__main__":
    main()
