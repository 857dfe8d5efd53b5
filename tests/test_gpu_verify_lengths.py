"""Draft verification on the GPU: lengths at the ends of 32 bits."""
import numpy as np
import pytest
import torch

from paper_2510_24824_b200.runner import DraftVerify

pytestmark = pytest.mark.gpu


def test_lengths_of_any_32_bits():
    """Wound back from zero where they lie below it, as the decode step takes them."""
    lens = torch.tensor([-2 ** 31, -2 ** 31 + 1, -1, 0, 1, 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    n, K, V = len(lens), 2, 40
    probs = torch.full((n, K + 1, V), 1.0 / V, device="cuda")
    drafts = torch.zeros(n, K, dtype=torch.int32, device="cuda")
    u = torch.full((n, K), 0.9, device="cuda")               # refuses every draft
    tokens, count, new = (torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((n, K + 1), (n,), (n,)))
    with DraftVerify("f32", n, K, V) as op:
        op.run(probs, drafts, u, torch.full((n,), 0.5, device="cuda"), tokens, count, seq_lens=lens, new_lens=new)
        assert op.check() == 0
    assert (count == 0).all()
    assert np.array_equal(new.cpu().numpy(), [0, 0, 0, 0, 0, 0, 2 ** 31 - 3])
