"""decode_shared where its bounds are far from what a batch holds: bounds on an item's sequences that none comes near, heads of many
chunks beside heads of one, on the GPU against the float64 oracle with the tolerances of test_gpu_shared.py."""
import numpy as np
import pytest
import torch

from oracle import audiokv_oracle as O
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


@pytest.mark.parametrize("stride_head,stride_tok", [((1 << 31) + 4096, 64), (64, 1 << 25)])
def test_eviction_moves_rows_beyond_32_bits(A, stride_head, stride_tok):
    """Rows further than 2^31 elements from the first, moved and left where they are: every slot against the oracle."""
    rng = np.random.default_rng(21)
    n, C, budget = [71, 67], 72, 40
    rows = torch.from_numpy(rng.integers(-30000, 30000, (2, 2, C, 64)).astype(np.int16)).cuda().view(torch.bfloat16)       # K, V
    weights = torch.from_numpy(rng.random((2, C)).astype(np.float32)).cuda()
    span = stride_head + (C - 1) * stride_tok + 64
    k, v = (torch.zeros(span, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    views = [x.as_strided((2, C, 64), (stride_head, stride_tok, 1)) for x in (k, v)]
    views[0].copy_(rows[0]); views[1].copy_(rows[1])
    slots = A.Slots(k, v, torch.tensor(n, dtype=torch.int32, device="cuda"), C, weights.clone())
    A.evict_accumulated(A.Params(4, 2, 64, 0, kv_stride_item=8, kv_stride_head=stride_head, kv_stride_tok=stride_tok), slots, 1, budget, 0, C)
    torch.cuda.synchronize()
    assert slots.lengths.tolist() == [budget] * 2
    for h in range(2):
        w = weights[h, :n[h]].cpu().numpy()
        src = torch.tensor(O.evict_accumulated(w, np.arange(n[h]), budget, 0) + list(range(budget, C)), device="cuda")
        assert src[:budget].tolist() != list(range(budget))
        assert torch.equal(slots.weights[h], weights[h, src])
        for x, was in zip(views, rows):
            assert torch.equal(x[h].view(torch.int16), was[h, src].view(torch.int16)), h
