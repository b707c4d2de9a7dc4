"""The example that runs the operators together: it learns, and tokens one by one are those that whole prompts give."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_example_learns_and_continues_a_prompt():
    import torch
    import decay_lm
    model, losses = decay_lm.train(60, say=lambda _: None)
    assert sum(losses[-5:]) / 5 < 0.8 * losses[0]              # (ln 64 = 4.2 at the start)
    prompt = torch.randint(decay_lm.VOCAB, (3 * decay_lm.PERIOD + 2,), generator=torch.Generator().manual_seed(3)).cuda()
    tokens = model.generate(prompt, 6)
    whole = torch.cat([prompt, tokens[:-1]])
    n = whole.numel()
    with torch.no_grad():
        logits = model(whole, torch.arange(n, device="cuda"), torch.tensor([0, n], device="cuda"))[prompt.numel() - 1:]
    chosen, best = logits.gather(1, tokens[:, None]).squeeze(1), logits.max(1).values
    assert tokens.shape == (6,) and (best - chosen <= 0.05 * logits.abs().max()).all()     # (equal but for 16-bit roundings between the two ways)
