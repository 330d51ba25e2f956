"""GPU tests of the verification of drafted tokens that were chosen, not drawn, where the probabilities do not sum to 1."""

import pytest
import torch

import paper_2609_08131_gb300.api as api
from test_gpu_bytes import BF16, DEV, F32, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("u,taken,drawn", [
    ([0.999, 0.6, 0.0], 1, 3),   # 0.6 / 256 < 0.0025
    ([0.999, 0.64, 0.0], 1, 3),  # 0.00250 < 0.0025024
    ([0.999, 0.65, 0.0], 0, 1),  # 0.00254: rejected, and nothing is left: the target's own are drawn from
    ([0.999, 0.65, 0.998], 0, 2),
    ([0.99, 0.0, 0.0], 1, 3),
])
def test_rejected_probabilities_are_taken_from_one(u, taken, drawn):
    """Two siblings, of 0.99609375 and 0.0025024 = 0x1.48p-9 in bf16, which hold all of the row: after the first one is
    rejected Z is 1 - 0.99609375 = 2^-8, so that the second one is accepted below 0.64 (0x1.48p-9 / 2^-8 = 0.640625)."""
    p = torch.zeros(1, 3, 5, dtype=F32, device=DEV)
    p[0, 0, 1], p[0, 0, 2] = 0.99609375, 0.0025
    p[0, 1:, 3] = 1.0
    p = p.to(BF16)
    assert float(p[0, 0, 2]) == float.fromhex("0x1.48p-9")
    masks = api.tree_masks([[-1, -1]]).to(DEV)
    ver = api.DraftVerifier(1, 2, 5, device=DEV)
    path, got, token = ver.run(ints([[1, 2]]), p, torch.tensor([u], dtype=F32, device=DEV), None, masks)
    assert (got.tolist(), token.tolist()) == ([taken], [drawn])
    assert path.tolist() == [[-1, -1] if taken == 0 else ([0, -1] if u[0] < 0.99609375 else [1, -1])]
    ver.check()
