"""Quantise a small language model's weights with the solver, then train what is left of it through the codes.

A block of two layers (4-bit codes, packed) and a vocabulary (8-bit codes); the embedding and the biases stay in
bfloat16 and learn to predict a synthetic sequence.  No weight is dequantised, the loss
keeps no logits, and the activations wait for the backward pass in 8 bits.  Run on an MI355X:

    python examples/finetune_quantized.py --steps 50
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2202_07471_amd as sq  # noqa: E402


class QuantizedLanguageModel(torch.nn.Module):
    def __init__(self, vocabulary: int, width: int, hidden: int, seed: int = 0):
        super().__init__()
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols):
            return torch.randn(rows, cols, device="cuda", generator=gen) / math.sqrt(cols)

        self.embedding = torch.nn.Parameter(torch.randn(vocabulary, width, device="cuda", generator=gen).bfloat16())
        self.up_bias = torch.nn.Parameter(torch.zeros(hidden, dtype=torch.bfloat16, device="cuda"))
        self.down_bias = torch.nn.Parameter(torch.zeros(width, dtype=torch.bfloat16, device="cuda"))
        self.up = sq.squant_quantize_ex(weight(hidden, width), 4, sq.MODE_EKC, sq.OUT_INT4)
        self.down = sq.squant_quantize_ex(weight(width, hidden), 4, sq.MODE_EKC, sq.OUT_INT4)
        self.head = sq.squant_quantize(weight(vocabulary, width), 8, sq.MODE_EKC)

    def hidden_states(self, tokens: torch.Tensor) -> torch.Tensor:
        x = self.embedding[tokens]
        h = sq.quantized_linear(x, *self.up, self.up_bias, sq.ACT_GELU)
        return sq.quantized_linear(h, *self.down, self.down_bias, residual=x)

    def loss(self, tokens: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        losses = sq.quantized_cross_entropy(self.hidden_states(tokens), *self.head, labels)
        return losses.sum() / (labels != sq.IGNORE_INDEX).sum()

    @torch.no_grad()
    def next_token(self, token: torch.Tensor) -> torch.Tensor:
        """The likeliest next token of each of a few sequences, as a server asks for it."""
        return sq.squant_linear(self.hidden_states(token), *self.head).argmax(-1)


def main(steps: int = 50, vocabulary: int = 1000, width: int = 256, hidden: int = 1024, batch: int = 16, length: int = 65):
    model = QuantizedLanguageModel(vocabulary, width, hidden)
    optimizer = torch.optim.Adam(model.parameters(), lr=2e-2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for step in range(steps):
        start = torch.randint(0, vocabulary, (batch, 1), device="cuda", generator=gen)
        tokens = (start + 7 * torch.arange(length + 1, device="cuda")) % vocabulary
        labels = tokens[:, 1:].clone()
        labels[:, 0] = sq.IGNORE_INDEX  # the first prediction of a sequence does not count
        loss = model.loss(tokens[:, :-1], labels)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    token = torch.arange(4, device="cuda")
    right = (model.next_token(token) == (token + 7) % vocabulary).sum().item()
    print(f"loss {losses[0]:.3f} at first, {losses[-1]:.3f} after {steps} steps; {right} of 4 next tokens right")
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=50)
    main(parser.parse_args().steps)
