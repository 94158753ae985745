"""The example that uses the language-model operators together: asynchronous workers distil a teacher."""
import sys

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu

sys.path.insert(0, str(ROOT / "examples"))


def test_the_student_learns_from_stale_snapshots():
    import async_distill

    first, last, _ = async_distill.main(commits=240, verbose=False)
    # a student without training is at the divergence of two unrelated models; a fifth of the commits
    # by four workers bring it well below
    assert last < 0.6 * first, (first, last)


def test_token_by_token_answers_are_the_sequence_s():
    """Generation with the state carried on gives the tokens that a forward pass over the result gives."""
    import async_distill

    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    m = async_distill.Model(300, 16, 40)
    flat = m.init(g)
    first = torch.arange(8, device="cuda")
    out = m.generate(flat, first, 20)
    logits, _ = m.forward(flat, torch.cat([first[:, None], out[:, :-1]], 1))
    two = logits.view(8, 20, -1).topk(2, 2).values
    clear = (two[..., 0] - two[..., 1]) > 1e-3          # apart by more than rounding
    assert bool((logits.view(8, 20, -1).argmax(2) == out)[clear].all()) and float(clear.float().mean()) > 0.9
