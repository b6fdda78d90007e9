"""Decode with drafted tokens end to end: look-up, q/k norms and append, attention, verification, step after step."""
import numpy as np
import pytest
import torch

from paper_2505_21889_b200 import drafted

pytestmark = pytest.mark.gpu


def _prompts(users, vocab, seed):
    rng = np.random.default_rng(seed)
    return [np.tile(rng.integers(0, vocab, 9), 6)[:n].tolist() for n in rng.integers(17, 54, users)]


@pytest.mark.parametrize("temperature", [0.0, 0.8])
@pytest.mark.parametrize("drafts", [0, 1, 4, 9])
def test_generated_text_and_cache(drafts, temperature):
    """What the steps leave is what one pass over the generated text gives: the cache bit for bit (rows of refused drafts are written
    over), and, decoded greedily, every token the likeliest of its row up to the rounding of bf16 logits (2^-8 of values below 16,
    from attention outputs that differ by rounding: 0.1)."""
    model = drafted.Model(3, 504, 8, 2, 64, 300)
    prompts = _prompts(6, 504, drafts)
    session, said, totals = drafted.run(model, prompts, 40, drafts, temperature, seed=5)
    assert all(40 <= len(t) <= 40 + drafts for t in said)
    assert totals["steps"] <= 40 and (drafts > 0 or totals["steps"] == 40)
    texts = [p + t for p, t in zip(prompts, said)]
    for s, t in enumerate(texts):
        assert session.history[s, :len(t)].tolist() == t
    whole = drafted.Session(model, texts, session.history.shape[1] - max(len(t) for t in texts))
    whole.table.copy_(session.table)
    tokens = torch.cat([whole.history[s, :n] for s, n in enumerate(whole.lens)])
    _, out = whole.attend(tokens, np.zeros(len(texts), np.int32), whole.lens)
    logits = model.logits(tokens, out).float()
    torch.cuda.synchronize()
    assert int(whole.status.item()) == 0
    row = 0
    for s, (p, t) in enumerate(zip(prompts, said)):
        n = len(p) + len(t) - 1                                           # the last token's row is not in the cache yet
        pages, slots = session.table[s, torch.arange(n) // 16].long(), torch.arange(n) % 16
        for a, b in ((session.cache.k_pool, whole.cache.k_pool), (session.cache.v_pool, whole.cache.v_pool)):
            assert torch.equal(a[pages, :, slots].view(torch.int16), b[pages, :, slots].view(torch.int16))
        if temperature == 0:
            said_by = logits[row + len(p) - 1:row + n]
            chosen = said_by.gather(1, torch.tensor(t, device="cuda")[:, None])[:, 0]
            assert (said_by.amax(1) - chosen).max() <= 0.1
        row += n + 1


def test_drafts_are_taken_up():
    """Where the text repeats itself, steps with drafts bring more than one token each."""
    model = drafted.Model(4, 304, 4, 4, 128, 400)
    prompts = _prompts(3, 304, 1)
    plain = drafted.run(model, prompts, 60, 0)
    quick = drafted.run(model, prompts, 60, 6)
    assert quick[2]["tokens_per_user_step"] > 1.3 * plain[2]["tokens_per_user_step"] == 1.3
