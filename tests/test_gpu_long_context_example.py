"""The example that trains a small windowed decoder and lets it answer: tokens one by one against the sequence at once, the change of the loss
along the gradient, and that training makes the text more likely."""
import pytest
import torch

import paper_2405_18047_amd as tbp
from paper_2405_18047_amd.examples import long_context as lc

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return g


def test_answering_sees_what_training_saw():
    """Logits of tokens decoded one by one over ring caches are those of the whole sequence's forward at the same places."""
    print("example: decode against forward", flush=True)
    c = lc.Shape(window=20, sinks=3)
    model = lc.Model(c, seq=72, batch=2)
    tokens = torch.randint(0, c.vocab, (2, 72), generator=_gen(3), device="cuda:0")
    want = model.logits(model.hidden(tokens)).float().view(2, 72, -1)
    caches, lengths = model.caches(2), torch.zeros(2, dtype=torch.int32, device="cuda:0")
    for i in range(72):
        lengths += 1
        got = model.next_logits(tokens[:, i], lengths, caches).float()
        # the same operations in another order, each result rounded to bf16: a few 2^-9 of the logits' size
        assert float((got - want[:, i]).abs().max()) < 4e-2 * float(want.abs().max()), i


def test_gradient_follows_the_loss():
    """The mean log probability changes along the negative gradient as the gradient says (to the accuracy of a bf16 model)."""
    print("example: gradient along its own direction", flush=True)
    c = lc.Shape(layers=1)
    model = lc.Model(c, seq=64, batch=8)
    tokens, targets = lc.phrases(8, 64, 16, c.vocab, _gen(4))
    before, grads = model.gradients(tokens, targets)
    slope = float(sum((g.double() ** 2).sum() for g in grads))
    rate = 0.05 / slope                                          # a change of 0.05 by the gradient
    for w, p, g in zip(model.master, model.params, grads):
        w.sub_(g, alpha=rate)
        p.copy_(w)
    after, _ = model.gradients(tokens, targets)
    change = float(after) - float(before)
    assert 0.5 * 0.05 < change < 1.5 * 0.05, change


def test_training_makes_the_text_likelier_and_clips():
    print("example: training", flush=True)
    model = lc.Model(lc.Shape(), seq=128, batch=8)
    gen = _gen(5)
    first = last = None
    for i in range(40):
        tokens, targets = lc.phrases(8, 128, 16, model.c.vocab, gen)
        logp, norm = model.step(tokens, targets, 0.5, max_norm=0.5)
        total = torch.sqrt(sum((g.double() ** 2).sum() for g in model.clipped))
        assert float(norm) > 0 and abs(float(total) - min(float(norm), 0.5)) < 1e-4
        first = float(logp) if first is None else first
        last = float(logp)
    assert last > first + 0.2, (first, last)
    said, weights = model.answer(tokens[:, :32], 3)
    assert said.shape == (8, 3) and bool((weights[..., :-1] >= weights[..., 1:]).all())
