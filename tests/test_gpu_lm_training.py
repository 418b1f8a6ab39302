"""The example that uses the operators together (train_lm.py): its gradients agree with plain torch operations, and
it learns its synthetic text."""
import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import train_lm  # noqa: E402

pytestmark = pytest.mark.gpu


class Plain:
    """The operators in torch."""

    @staticmethod
    def embedding(tokens, table, scale):
        return table[tokens] * scale

    @staticmethod
    def layer_norm(x, gain, bias):
        return torch.nn.functional.layer_norm(x.float(), x.shape[-1:], gain, bias).to(x.dtype)

    @staticmethod
    def loss(h, w, targets):
        return torch.nn.functional.cross_entropy(h.flatten(0, -2) @ w.t(), targets.flatten())


def test_gradients_agree_with_plain_operations():
    grads = []
    tokens, targets = train_lm.Text(700).batch(3, 40)
    for ops in (train_lm.Operators(), Plain):
        parts = train_lm.build(700, 64, 2)
        loss = train_lm.loss_of(ops, *parts, tokens, targets, torch.float32)
        loss.backward()
        grads.append([loss.detach()] + [p.grad for part in parts for p in part.values()])
    # Two evaluations in fp32 of the same model, a few hundred terms per sum.
    for a, b in zip(*grads):
        assert (a - b).norm() <= 2e-5 * b.norm() + 1e-9


@pytest.mark.parametrize("bits,dtype", [(8, "bf16"), (32, "fp32")])
def test_it_learns(bits, dtype):
    out = train_lm.train(vocab=512, width=128, blocks=1, rows=32, length=64, steps=60, bits=bits, dtype=dtype)
    losses = out["losses"]
    assert abs(losses[0] - math.log(512)) < 0.5
    # A tenth of the tokens is free: what can be known leaves about 0.1 log 512 + 0.33 = 0.95.
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0], losses
