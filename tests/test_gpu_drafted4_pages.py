"""Pages that a drafted loop over a 4-bit cache holds: those of its text at least, and of the last step's refused drafts at most."""
import pytest
import torch

from paper_2505_21889_b200 import drafted
from tests.test_gpu_drafted4 import _prompts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("drafts", [0, 4, 9])
def test_pages_of_the_text(drafts):
    model = drafted.Model(3, 504, 8, 2, 64, 300)
    prompts = _prompts(6, 504, drafts)
    session, said, _ = drafted.run(model, prompts, 40, drafts, cache_bits=4)
    for s, (p, t) in enumerate(zip(prompts, said)):
        n = len(p) + len(t) - 1                                           # the last token's row is not in the cache yet
        row = session.table[s]
        held = int((row >= 0).sum())
        assert -(-n // 16) <= held <= -(-(n + drafts + 1) // 16)
        assert (row[:held] >= 0).all() and (row[held:] == -1).all()
    assert len(torch.unique(session.table[session.table >= 0])) == int((session.table >= 0).sum())
