"""A small language model whose feed-forward layers are Monarch matrices, trained from the loss to the optimiser's step with this library's kernels:

    python examples/train_lm.py [--steps 200] [--vocab 5003] [--width 256] [--layers 2] [--tokens 2048]

Token and position embeddings, feed-forward blocks (MonarchLinear, GELU, MonarchLinear) with residuals, and a dense head over the vocabulary.  The
loss is ``vocab_cross_entropy`` (no logits in memory), the factors are stepped by ``Muon``, the embeddings and the head by AdamW.  The data is
synthetic: each token decides the next one in nine cases of ten, so the loss falls from log(vocab) towards what is left to chance.  At the
end a held-out batch is scored one row at a time and all at once (``monarch_xent_fwd``).
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2204_00595_amd import binding  # noqa: E402
from paper_2204_00595_amd.autograd import MonarchLinear, vocab_cross_entropy  # noqa: E402
from paper_2204_00595_amd.optim import Muon  # noqa: E402

IGNORE = -100


class Block(torch.nn.Module):
    def __init__(self, width: int):
        super().__init__()
        self.up = MonarchLinear(width, 4 * width, device="cuda")
        self.down = MonarchLinear(4 * width, width, device="cuda")

    def forward(self, x):
        h = torch.nn.functional.rms_norm(x, x.shape[-1:])
        return x + self.down(torch.nn.functional.gelu(self.up(h), approximate="tanh"))


class Model(torch.nn.Module):
    def __init__(self, vocab: int, width: int, layers: int):
        super().__init__()
        self.tokens = torch.nn.Embedding(vocab, width, device="cuda", dtype=torch.bfloat16)
        self.blocks = torch.nn.ModuleList([Block(width) for _ in range(layers)])
        self.head = torch.nn.Parameter((torch.randn((vocab, width), device="cuda") / math.sqrt(width)).to(torch.bfloat16))

    def forward(self, tokens):
        """The last hidden state; the logits are head times it."""
        x = self.tokens(tokens)
        for block in self.blocks:
            x = block(x)
        return torch.nn.functional.rms_norm(x, x.shape[-1:])


def batch(next_of, tokens, generator):
    """Tokens and what follows each; a tenth of the rows are padding, which has no target."""
    vocab = len(next_of)
    t = torch.randint(0, vocab, (tokens,), generator=generator, device="cuda")
    chance = torch.rand((tokens,), generator=generator, device="cuda")
    target = torch.where(chance < 0.9, next_of[t], torch.randint(0, vocab, (tokens,), generator=generator, device="cuda"))
    target[torch.rand((tokens,), generator=generator, device="cuda") < 0.1] = IGNORE
    return t, target


def train(steps=200, vocab=5003, width=256, layers=2, tokens=2048, seed=0, say=print):
    """The losses of all steps, and of a held-out batch by rows and as a mean."""
    torch.manual_seed(seed)
    generator = torch.Generator(device="cuda")
    generator.manual_seed(seed)
    next_of = torch.randperm(vocab, generator=generator, device="cuda")
    model = Model(vocab, width, layers)
    factors = [p for b in model.blocks for layer in (b.up, b.down) for p in (layer.R, layer.L)]
    taken = {id(p) for p in factors}
    others = [p for p in model.parameters() if id(p) not in taken]
    muon, adam = Muon(factors, lr=0.02), torch.optim.AdamW(others, lr=0.01, weight_decay=0.0)
    losses = []
    for step in range(steps):
        t, target = batch(next_of, tokens, generator)
        loss = vocab_cross_entropy(model(t), model.head, target, ignore_index=IGNORE)
        loss.backward()
        muon.step()
        adam.step()
        muon.zero_grad()
        adam.zero_grad()
        losses.append(loss.detach())
        if say and (step % 20 == 0 or step + 1 == steps):
            say("step %4d  loss %.4f" % (step, loss.item()), flush=True)
    with torch.no_grad():
        t, target = batch(next_of, 64, generator)
        x = model(t)
        whole, _ = binding.monarch_xent_fwd(x, model.head, target, ignore_index=IGNORE)
        single = torch.cat([binding.monarch_xent_fwd(x[i:i + 1], model.head, target[i:i + 1], ignore_index=IGNORE)[0] for i in range(64)])
        mean = binding.monarch_xent_total(whole, target, ignore_index=IGNORE)[0]
    if say:
        say("held out: mean loss %.4f over %d rows; rows one at a time differ by at most %.1e"
            % (mean.item(), int((target != IGNORE).sum()), (whole - single).abs().max().item()), flush=True)
    return torch.stack(losses), whole, single, mean


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 200), ("vocab", 5003), ("width", 256), ("layers", 2), ("tokens", 2048)):
        a.add_argument("--" + name, type=int, default=value)
    train(**vars(a.parse_args()))


if __name__ == "__main__":
    main()
