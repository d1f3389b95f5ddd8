"""decode_shared where its bounds are far from what a batch holds: bounds on an item's sequences that none comes near, heads of many
chunks beside heads of one, on the GPU against the float64 oracle with the tolerances of test_gpu_shared.py."""
import numpy as np
import pytest
import torch

from test_gpu_shared import A, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H_q,H_kv,d", [(28, 4, 128), (8, 2, 256), (8, 2, 64)])
@pytest.mark.parametrize("bound", ["tight", "all"])
def test_ragged_items_and_a_loose_bound(A, H_q, H_kv, d, bound):
    """Chunks that begin in the row blocks of other heads' ends, next to heads of one chunk and of none; sequences in different
    numbers; the workspace begins as NaN, so that a result that nobody wrote would be seen."""
    rng = np.random.default_rng(d + H_q)
    sharing = [1, 0, 7, 2, 30]
    budgets = [int(b) for b in rng.choice([0, 1, 127, 128, 129, 500, 1300, 2900], len(sharing) * H_kv)]
    budgets[0], budgets[-1] = 2900, 1300
    n = sum(sharing) + 3
    s = Step(rng, H_q, H_kv, d, budgets, sharing, rng.choice([0, 1, 64, 200], (sum(sharing), H_kv)), 210, spare=3)
    t = s.tensors(A)
    most = 30 if bound == "tight" else n
    ws = torch.full((A.decode_shared_workspace_bytes(t["p"], len(sharing), len(s.kp), n, most, s.max_own(True)),), 255, dtype=torch.uint8, device="cuda")
    s.call(A, t, max_seqs=most, workspace=ws)
    s.check(t)
