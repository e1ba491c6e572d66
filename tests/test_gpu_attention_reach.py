"""How far a query sees, as the C entries take it: any reach back and ahead, each or none of them bounded, beside the causal ones and the windows of the binding."""
import pytest
import torch

import attention_util
from attention_util import DEV, NAME, TYPES
from paper_2506_16235_amd import binding as nsml
from test_gpu_attention import check

pytestmark = pytest.mark.gpu
types = pytest.mark.parametrize("dt", TYPES, ids=NAME.get)
FAR = 2 ** 31 - 1


@types
@pytest.mark.parametrize("dim,heads,kv", [(64, 4, 2), (128, 2, 2)])
@pytest.mark.parametrize("left,right", [(0, 0), (0, -1), (-1, 5), (7, -1), (3, 40), (100, 1), (-1, FAR), (FAR, FAR), (FAR, 0), (70, FAR)])
def test_reach(monkeypatch, dt, dim, heads, kv, left, right):
    def mask(m, n, causal, window):
        ahead = torch.arange(n, device=DEV)[None] - torch.arange(n - m, n, device=DEV)[:, None]
        seen = torch.ones(m, n, dtype=torch.bool, device=DEV)
        if left >= 0:
            seen &= ahead >= -left
        if right >= 0:
            seen &= ahead <= right
        return seen
    monkeypatch.setattr(nsml, "_reach", lambda causal, window: (left, right))
    monkeypatch.setattr(attention_util, "mask_of", mask)
    check(dt, heads, kv, dim, [90, 1, 0, 200, 33], [90, 40, 7, 131, 300], k_rooms=[95, 40, 8, 140, 300], seed=left % 97 + right % 89)
    check(dt, heads, kv, dim, [1, 2], [900, 130], seed=3, backward=False)
