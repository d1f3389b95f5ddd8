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


def test_a_captured_step_refilled_by_its_tables(A):
    """A graph of eleven sequences on four items, replayed with other numbers of sequences per item, and of rows per head, than it was
    captured with: results as of a call with those numbers."""
    rng = np.random.default_rng(31)
    p, n, capacity = A.Params(8, 2, 128, 0), 11, 70
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).bfloat16().cuda()
    q, kp, vp, k_new, v_new = draw(n, 8, 128), draw(3000, 128), draw(3000, 128), draw(n, 2, 128), draw(n, 2, 128)
    ko, vo = draw(n, 2, capacity, 128), draw(n, 2, capacity, 128)
    cu_s, cu_b, pos = (torch.zeros(m, dtype=torch.int32, device="cuda") for m in (5, 9, n))
    length = torch.tensor(rng.integers(0, 65, n * 2), dtype=torch.int32, device="cuda")
    state = [x.clone() for x in (ko, vo, length, torch.zeros(n * 2, capacity, device="cuda"), torch.full((n * 2, capacity), -1, dtype=torch.int32, device="cuda"))]
    slots = A.Slots(state[0], state[1], state[2], capacity, state[3], state[4])
    out = torch.empty_like(q)
    ws = torch.empty(A.decode_shared_workspace_bytes(p, 4, 3000, n, n, capacity), dtype=torch.uint8, device="cuda")

    def reset():
        for x, y in zip(state, (ko, vo, length)):
            x.copy_(y)
        state[3].zero_(); state[4].fill_(-1); out.fill_(7); ws.fill_(255)

    def call():
        A.decode_shared(p, q, kp, vp, cu_b, 3000, cu_s, n, slots=slots, max_own=capacity, k_new=k_new, v_new=v_new, pos_new=pos, out=out, workspace=ws)
    reset(); call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for sequences, budgets in (([2, 3, 1, 5], [100, 7, 0, 900, 300, 20, 1, 1000]), ([11, 0, 0, 0], [1500, 1500, 0, 0, 0, 0, 0, 0]),
                               ([0, 0, 1, 1], [1, 2, 3, 4, 500, 600, 700, 800]), ([0, 0, 0, 0], [375] * 8)):
        cu_s.copy_(torch.tensor(np.concatenate([[0], np.cumsum(sequences)]), dtype=torch.int32))
        cu_b.copy_(torch.tensor(np.concatenate([[0], np.cumsum(budgets)]), dtype=torch.int32))
        results = []
        for step in (call, graph.replay, graph.replay):
            reset(); step()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (out, *state)])
        for got in results[1:]:
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, results[0])), sequences
        active = sum(sequences)
        assert (out[active:] == 7).all() and torch.equal(state[2][2 * active:], length[2 * active:]) and (out[:active] != 7).any(2).all()
        assert torch.equal(state[2][:2 * active], length[:2 * active] + 1)


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
