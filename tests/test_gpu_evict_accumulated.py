"""Rows cut to a budget by recency and accumulated weight, on the GPU against the oracle: exact, since only comparisons decide
and rows move as they are. And the operators together, as a generating program uses them."""
import numpy as np
import pytest
import torch

from oracle import audiokv_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


class Rows:
    def __init__(self, rng, n_seqs, H_kv, d, lengths, capacity, layout="head", weights=None, positions=None):
        self.n, self.H, self.d, self.C, self.layout = n_seqs, H_kv, d, capacity, layout
        heads = n_seqs * H_kv
        self.lengths = np.resize(np.array(lengths, dtype=np.int32), heads)
        self.w = np.exp(2 * rng.standard_normal((heads, capacity))).astype(np.float32) if weights is None else weights(heads, capacity).astype(np.float32)
        self.pos = np.argsort(rng.random((heads, capacity)), axis=1).astype(np.int32) if positions is None else positions(heads, capacity).astype(np.int32)
        # every row says where it began: head, slot, K or V
        self.k = np.zeros((heads, capacity, d), dtype=np.int16)
        self.k[:, :, 0], self.k[:, :, 1] = np.arange(heads)[:, None], np.arange(capacity)
        self.k[:, :, 2:] = rng.integers(-30000, 30000, (heads, capacity, d - 2))
        self.v = self.k ^ 0x55

    def lay(self, x):
        x = x.reshape(self.n, self.H, self.C, self.d)
        if self.layout == "token":
            x = x.transpose(0, 2, 1, 3)
        elif self.layout == "strided":
            big = np.full((self.n, self.H, self.C + 1, 2 * self.d), 99, dtype=np.int16)
            big[:, :, :self.C, :self.d] = x
            x = big
        return torch.from_numpy(np.ascontiguousarray(x)).cuda().view(torch.bfloat16)

    def unlay(self, t):
        x = t.contiguous().view(torch.int16).cpu().numpy()
        if self.layout == "token":
            x = x.reshape(self.n, self.C, self.H, self.d).transpose(0, 2, 1, 3)
        elif self.layout == "strided":
            assert (x[:, :, self.C:] == 99).all() and (x[..., self.d:] == 99).all()
            x = x[:, :, :self.C, :self.d]
        return x.reshape(-1, self.C, self.d)

    def params(self, A):
        more = {}
        if self.layout == "strided":
            head = (self.C + 1) * 2 * self.d
            more = dict(kv_stride_item=self.H * head, kv_stride_head=head, kv_stride_tok=2 * self.d)
        return A.Params(self.H * 2, self.H, self.d, 0, kv_layout=1 if self.layout == "token" else 0, **more)

    def slots(self, A, positions=True):
        return A.Slots(self.lay(self.k), self.lay(self.v), torch.from_numpy(self.lengths.copy()).cuda(), self.C,
                       torch.from_numpy(self.w.copy()).cuda(), torch.from_numpy(self.pos.copy()).cuda() if positions else None)

    def check(self, s, budget, recent, max_own, budgets=None, positions=True):
        torch.cuda.synchronize()
        k, v, w, lengths = self.unlay(s.k), self.unlay(s.v), s.weights.cpu().numpy(), s.lengths.cpu().numpy()
        pos = s.positions.cpu().numpy() if positions else self.pos
        for g in range(self.n * self.H):
            n = int(self.lengths[g])
            b = budget if budgets is None else max(budget, int(budgets[g]))
            src = list(range(self.C))
            if b < n <= max_own:
                src[:b] = O.evict_accumulated(self.w[g, :n], self.pos[g, :n], b, recent)
                n = b
            assert lengths[g] == n, g
            assert np.array_equal(k[g], self.k[g, src]) and np.array_equal(v[g], self.v[g, src]), g
            assert np.array_equal(w[g], self.w[g, src], equal_nan=True), g
            assert not positions or np.array_equal(pos[g], self.pos[g, src]), g


def run(A, r, budget, recent, max_own=None, budgets=None, positions=True, **more):
    s = r.slots(A, positions)
    most = int(r.lengths.max()) if max_own is None else max_own
    A.evict_accumulated(r.params(A), s, r.n, budget, recent, most,
                        budgets=None if budgets is None else torch.tensor(budgets, dtype=torch.int32).cuda(), **more)
    r.check(s, budget, recent, most, budgets, positions)
    return s


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("layout", ["head", "token", "strided"])
def test_layouts(A, d, layout):
    run(A, Rows(np.random.default_rng(d), 3, 2, d, [40, 33, 7, 0, 25, 50], 50, layout), 24, 8)


@pytest.mark.parametrize("n,b", [(1, 0), (2, 1), (64, 63), (65, 64), (100, 92), (100, 91), (255, 1), (256, 128), (257, 250), (1025, 1024),
                                 (2048, 1024), (2049, 2045), (2049, 2000), (3000, 100), (8192, 8183), (8193, 8192), (8193, 5000),
                                 (20001, 20000), (20001, 11000), (600, 0)])
def test_sizes(A, n, b):
    """Either way to find what goes, ranks in LDS and not, either size of workgroup, moves in one launch and in two."""
    run(A, Rows(np.random.default_rng(n + b), 1, 3, 64, [n, max(0, n - 1), n // 2], n + 3), b, min(b, 16))


@pytest.mark.parametrize("recent", [0, 1, 5, 60, 1000, 2**31 - 1])
def test_recent(A, recent):
    run(A, Rows(np.random.default_rng(recent % 97), 2, 2, 64, [90, 61, 60, 30], 90), 60, recent)
    run(A, Rows(np.random.default_rng(recent % 89), 2, 2, 64, [90, 61, 60, 30], 90), 20, recent)


def test_extreme_positions(A):
    def ends(heads, C):
        p = np.resize(np.array([-2**31, 2**31 - 1, 0, -1, 5], dtype=np.int64), (heads, C))
        return p
    run(A, Rows(np.random.default_rng(1), 2, 1, 64, [30], 32, positions=ends), 20, 2)
    run(A, Rows(np.random.default_rng(2), 2, 1, 64, [30], 32, positions=lambda h, C: np.full((h, C), -2**31)), 20, 2**31 - 1)


@pytest.mark.parametrize("n,b", [(300, 296), (300, 150), (5000, 2500)])
def test_equal_weights_and_special_values(A, n, b):
    rng = np.random.default_rng(n)
    run(A, Rows(rng, 2, 1, 64, [n], n, weights=lambda h, C: np.zeros((h, C))), b, 10)
    run(A, Rows(rng, 2, 1, 64, [n], n, weights=lambda h, C: rng.integers(0, 3, (h, C))), b, 10)
    pool = np.array([0.0, -0.0, np.nan, np.inf, -np.inf, 1e-45, -1e-45, 3e38, -3e38, 1.0, -1.0], dtype=np.float32)
    run(A, Rows(rng, 2, 1, 64, [n], n, weights=lambda h, C: rng.choice(pool, (h, C))), b, 10)
    run(A, Rows(rng, 2, 1, 64, [n], n, weights=lambda h, C: np.full((h, C), np.nan)), b, 0)
    # close to one another: the last digits decide
    run(A, Rows(rng, 2, 1, 64, [n], n, weights=lambda h, C: 1 + rng.integers(0, 64, (h, C)) * 2.0 ** -23), b, 0)


def test_budgets_by_head_and_without_positions(A):
    r = Rows(np.random.default_rng(3), 2, 3, 64, [700, 400, 90, 700, 10, 0], 720)
    run(A, r, 50, 20, budgets=[600, 399, 0, 60, 500, 3])
    run(A, r, 50, 0, positions=False)


def test_heads_beyond_max_own_stay(A):
    run(A, Rows(np.random.default_rng(4), 2, 2, 64, [80, 70, 60, 50], 90), 40, 4, max_own=70)


def test_nobody_has_too_many(A):
    run(A, Rows(np.random.default_rng(5), 2, 2, 64, [8, 7, 3, 0], 9), 8, 2)
    run(A, Rows(np.random.default_rng(6), 2, 2, 64, [8, 7, 3, 0], 9), 8, 2, max_own=9)


def test_on_a_stream_and_in_a_graph(A):
    r = Rows(np.random.default_rng(7), 4, 2, 128, [1500, 900, 33, 1100], 1600)
    p, most, b = r.params(A), 1500, 700
    ws = torch.empty(A.evict_accumulated_workspace_bytes(p, 4, most, b), dtype=torch.uint8, device="cuda")
    s = r.slots(A)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        A.evict_accumulated(p, s, 4, b, 64, most, workspace=ws)
    r.check(s, b, 64, most)
    begin = r.slots(A)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.evict_accumulated(p, s, 4, b, 64, most, workspace=ws)
    for _ in range(3):
        for x, y in zip((s.k, s.v, s.lengths, s.weights, s.positions), (begin.k, begin.v, begin.lengths, begin.weights, begin.positions)):
            x.copy_(y)
        ws.fill_(255)
        graph.replay()
        r.check(s, b, 64, most)


def test_generation_on_an_evicted_prompt_with_a_bounded_cache(A):
    """All of it: a prompt is evicted, three sequences continue it, each step appends a row, attends, accounts and, once a
    head has more than its budget, evicts one. Every step against the oracle on the rows that the GPU kept."""
    rng = np.random.default_rng(8)
    H_q, H_kv, d, L, W, S, C, budget, recent = 8, 2, 64, 400, 16, 3, 24, 20, 6
    draw = lambda *s: bf16(rng.standard_normal(s))
    p = A.Params(H_q, H_kv, d, W)
    q_win, k, v = draw(1, H_q, W, d).cuda(), draw(H_kv, L, d).cuda(), draw(H_kv, L, d).cuda()
    got = A.evict(p, q_win, k, v, torch.tensor([1.0, 3.0], device="cuda"), [L], 0.3, 0.125, 1.0)
    rows, cu_b = got["total_rows"], got["cu_budgets"]
    slots = A.Slots(torch.zeros(S, H_kv, C, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(S, H_kv, C, d, dtype=torch.bfloat16, device="cuda"),
                    torch.zeros(S * H_kv, dtype=torch.int32, device="cuda"), C, torch.zeros(S * H_kv, C, device="cuda"),
                    torch.zeros(S * H_kv, C, dtype=torch.int32, device="cuda"))
    cu_s = torch.tensor([0, S], dtype=torch.int32, device="cuda")
    cu = cu_b.cpu().numpy()
    kp, vp = (got[x].float().cpu().numpy().astype(np.float64) for x in ("k_out", "v_out"))
    held = [[] for _ in range(S * H_kv)]            # (position, k, v, weight), in the order of the slots
    for step in range(40):
        q, k_new, v_new = draw(S, H_q, d), draw(S, H_kv, d), draw(S, H_kv, d)
        pos = torch.full((S,), L + step, dtype=torch.int32, device="cuda")
        out = A.decode_shared(p, q.cuda(), got["k_out"], got["v_out"], cu_b, rows, cu_s, S, slots=slots, max_own=C,
                              k_new=k_new.cuda(), v_new=v_new.cuda(), pos_new=pos)
        out, weights = out.float().cpu().numpy(), slots.weights.cpu().numpy()
        f = lambda t: t.float().numpy().astype(np.float64)
        for x in range(S):
            ks, vs = [], []
            for h in range(H_kv):
                held[x * H_kv + h].append((L + step, f(k_new)[x, h], f(v_new)[x, h], 0.0))
                own = held[x * H_kv + h]
                ks.append(np.concatenate([kp[cu[h]:cu[h + 1]], [r[1] for r in own]]))
                vs.append(np.concatenate([vp[cu[h]:cu[h + 1]], [r[2] for r in own]]))
            want, w = O.decode_weights(f(q)[x], ks, vs)
            assert np.abs(out[x] - want).max() <= 3 * 2.0 ** -8 * np.abs(np.concatenate(vs)).max()
            for h in range(H_kv):
                g = x * H_kv + h
                n = len(held[g])
                total = np.array([r[3] for r in held[g]]) + w[h][len(ks[h]) - n:]
                assert np.allclose(weights[g, :n], total, rtol=1e-4, atol=0)
                held[g] = [r[:3] + (float(weights[g, t]),) for t, r in enumerate(held[g])]      # (go on from what the GPU has)
        A.evict_accumulated(p, slots, S, budget, recent, C)
        for g in range(S * H_kv):
            src = O.evict_accumulated(np.array([r[3] for r in held[g]]), np.array([r[0] for r in held[g]]), budget, recent)
            held[g] = [held[g][t] for t in src]
        assert slots.lengths.tolist() == [min(step + 1, budget)] * (S * H_kv)
        where = slots.positions.cpu().numpy()
        for g in range(S * H_kv):
            assert where[g, :len(held[g])].tolist() == [r[0] for r in held[g]]
