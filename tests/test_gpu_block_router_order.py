"""The order of chosen experts whose softmax is equal, or nearly so, in 64 bits: equal choices go by their index, whichever logit is
larger, and whether or not who comes behind them is in doubt."""
import pytest
import torch

import block_reference as ref
from paper_2311_01635_amd import RtpRouter

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ids(l, k, groups):
    T, E = l.shape
    ids, w = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    RtpRouter(E, k, groups=groups, kept_groups=groups).forward(l.to(DEV), ids, w)
    return ids.cpu()


@pytest.mark.parametrize("E,groups", [(8, 2), (16, 4), (60, 5), (256, 8), (1000, 10)])
def test_equal_scores_of_unequal_logits(E, groups):
    """beside a logit of 1 (or of 0) those below 2^-59 all have the same exponential: l - 1 is -1 (e^l is 1) in 64 bits"""
    rows = []
    at = torch.randperm(E, generator=torch.Generator().manual_seed(E))[:6].tolist()
    for top in (1.0, 0.0):
        for values in ((0.0, 1e-18), (1e-20, 2e-20), (3e-20, 1e-20, 2e-20, 1e-18), (-1e-18, 0.0, 1e-25, -1e-30)):
            row = torch.full((E,), -5.0)
            row[at[0]] = top
            for i, x in zip(at[1:], values):
                row[i] = x
            rows.append(row)
    l = torch.stack(rows)
    for k in range(1, 6):        # (with k inside the equals who is last is in doubt, and behind them it is not)
        assert torch.equal(_ids(l, k, groups), ref.route(l, k, groups=groups, kept=groups)[0]), k


@pytest.mark.parametrize("E,groups", [(16, 4), (256, 8)])
def test_order_does_not_hang_on_who_comes_behind(E, groups):
    """logits 2^-36 to 2^-62 apart beside a 1: the first five are in the same order whether five are chosen (and the sixth, as close, is in
    doubt) or all six"""
    g = torch.Generator().manual_seed(7)
    l = torch.full((256, E), -5.0)
    for t in range(256):
        at = torch.randperm(E, generator=g)[:6]
        l[t, at[0]] = 1.0
        l[t, at[1:]] = 2.0 ** -(36 + t % 27) * torch.randint(1, 9, (5,), generator=g).float()
    assert torch.equal(_ids(l, 6, groups)[:, :5], _ids(l, 5, groups))
