"""One decoding step on shared prompts and own rows on the GPU against the float64 oracle, through the public entry point.

Tolerances, with u = 2^-24 (fp32) and b = 2^-8 (bf16), the relative error of one rounding. A weight p is off by e p: logits as
in test_gpu_accumulate.py (both numerator and denominator), n u for sums of n terms, 2^-21 for exp2 and log2. The output is
sum p v: each p rounded to bf16 once more, the result too, so it is off by (b + e + n u) sum p |v| + b |out|. Accumulated
weights are off by e times what was added, and the rounding of the sum."""
import numpy as np
import pytest
import torch

from oracle import audiokv_oracle as O

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


class Step:
    """budgets[g]: kept rows of head g = item * H_kv + h; sharing[i]: sequences of item i (None: no prompts); own[x][h]: own rows."""

    def __init__(self, rng, H_q, H_kv, d, budgets, sharing, own, capacity, layout="head", scale=None, spare=0, k_scale=1.0):
        self.H_q, self.H_kv, self.d, self.budgets, self.sharing, self.capacity = H_q, H_kv, d, budgets, sharing, capacity
        self.layout, self.scale = layout, scale
        self.active = sum(sharing) if sharing is not None else len(own)
        self.n = n = self.active + spare
        self.own = np.array([list(x) for x in own] + [[0] * H_kv] * (n - len(own)), dtype=np.int64).reshape(n, H_kv)
        draw = lambda *s, k=1.0: f64(bf16(k * rng.standard_normal(s)))
        self.q = draw(n, H_q, d)
        self.kp, self.vp = draw(sum(budgets or []), d, k=k_scale), draw(sum(budgets or []), d)
        self.ko, self.vo = draw(n, H_kv, capacity, d, k=k_scale), draw(n, H_kv, capacity, d)
        self.k_new, self.v_new = draw(n, H_kv, d, k=k_scale), draw(n, H_kv, d)
        self.w = rng.random((n, H_kv, capacity)).astype(np.float32)
        # slots that are not in use hold anything
        for x in range(n):
            for h in range(H_kv):
                self.ko[x, h, self.own[x, h]:] = np.nan
                self.vo[x, h, self.own[x, h]:] = np.inf
                self.w[x, h, self.own[x, h]:] = 7

    def lay(self, x):
        """[n, H_kv, capacity, d] as the asked layout."""
        if self.layout == "token":
            x = x.transpose(0, 2, 1, 3)
        elif self.layout == "strided":          # heads innermost but one, padded
            big = np.full((self.n, self.capacity + 2, self.H_kv + 1, self.d), np.nan)
            big[:, :self.capacity, :self.H_kv] = x.transpose(0, 2, 1, 3)
            x = big
        return bf16(x).cuda().contiguous()

    def unlay(self, t):
        x = f64(t)
        if self.layout == "token":
            return x.reshape(self.n, self.capacity, self.H_kv, self.d).transpose(0, 2, 1, 3)
        if self.layout == "strided":
            return x[:, :self.capacity, :self.H_kv].transpose(0, 2, 1, 3)
        return x.reshape(self.n, self.H_kv, self.capacity, self.d)

    def params(self, A):
        more = {}
        if self.layout == "strided":
            row = (self.H_kv + 1) * self.d
            more = dict(kv_stride_item=(self.capacity + 2) * row, kv_stride_head=self.d, kv_stride_tok=row)
        return A.Params(self.H_q, self.H_kv, self.d, 0, kv_layout=1 if self.layout == "token" else 0,
                        softmax_scale=self.scale or 0.0, **more)

    def tensors(self, A, weights=True, positions=True):
        t = dict(p=self.params(A), q=bf16(self.q).cuda(), k_new=bf16(self.k_new).cuda(), v_new=bf16(self.v_new).cuda())
        if self.sharing is not None:
            t["cu_b"] = torch.tensor(np.concatenate([[0], np.cumsum(self.budgets)]), dtype=torch.int32).cuda()
            t["cu_s"] = torch.tensor(np.concatenate([[0], np.cumsum(self.sharing)]), dtype=torch.int32).cuda()
            t["kp"], t["vp"] = bf16(self.kp).cuda(), bf16(self.vp).cuda()
        t["slots"] = A.Slots(self.lay(self.ko), self.lay(self.vo), torch.from_numpy(self.own.astype(np.int32).reshape(-1)).cuda(),
                             self.capacity, torch.from_numpy(self.w.copy()).cuda() if weights else None,
                             torch.full((self.n * self.H_kv, self.capacity), -5, dtype=torch.int32).cuda() if positions else None)
        t["pos"] = torch.arange(1000, 1000 + self.n, dtype=torch.int32).cuda()
        t["out"] = torch.full((self.n, self.H_q, self.d), 77.0, dtype=torch.bfloat16).cuda()
        return t

    def call(self, A, t, append=True, max_own=None, max_seqs=None, slots=True, workspace=None):
        rows = 0 if self.sharing is None else len(self.kp)
        got = A.decode_shared(t["p"], t["q"], t.get("kp"), t.get("vp"), t.get("cu_b"), rows, t.get("cu_s"),
                              max_seqs or max(1, max(self.sharing or [1])), slots=t["slots"] if slots else None,
                              max_own=self.max_own(append) if max_own is None else max_own,
                              k_new=t["k_new"] if append else None, v_new=t["v_new"] if append else None,
                              pos_new=t["pos"] if append else None, out=t["out"], workspace=workspace)
        assert got is t["out"]

    def max_own(self, append):
        return min(self.capacity, int(self.own.max()) + append)

    def check(self, t, append=True, max_own=None, slots=True, weights=True):
        torch.cuda.synchronize()
        out, s = f64(t["out"]), t["slots"]
        most = 0 if not slots else self.max_own(append) if max_own is None else max_own
        lengths = s.lengths.cpu().numpy().reshape(self.n, self.H_kv)
        ko, vo = self.unlay(s.k), self.unlay(s.v)
        w_got = s.weights.cpu().numpy().astype(np.float64).reshape(self.w.shape) if weights else None
        pos = s.positions.cpu().numpy().reshape(self.n, self.H_kv, -1) if s.positions is not None else None
        cu = np.concatenate([[0], np.cumsum(self.budgets or [])]).astype(int)
        G, c = self.H_q // self.H_kv, (self.scale or self.d ** -0.5) * 1.4426950408889634
        item_of = np.repeat(np.arange(len(self.sharing)), self.sharing) if self.sharing is not None else None
        for x in range(self.n):
            if x >= self.active:                                   # takes no part
                assert (out[x] == 77).all() and (lengths[x] == self.own[x]).all()
                assert weights is False or (w_got[x] == self.w[x]).all()
                continue
            k_rows, v_rows, added = [], [], []
            for h in range(self.H_kv):
                m = min(int(self.own[x, h]), most)
                new = bool(append) and m < most
                assert lengths[x, h] == (m + 1 if new else self.own[x, h]), (x, h)
                k, v = self.ko[x, h].copy(), self.vo[x, h].copy()
                if new:
                    k[m], v[m] = self.k_new[x, h], self.v_new[x, h]
                    assert pos is None or pos[x, h, m] == 1000 + x
                assert np.array_equal(ko[x, h], k, equal_nan=True) and np.array_equal(vo[x, h], v, equal_nan=True)
                assert pos is None or (np.delete(pos[x, h], m if new else []) == -5).all()
                k, v = k[:m + new], v[:m + new]
                if item_of is not None:
                    g = item_of[x] * self.H_kv + h
                    k, v = np.concatenate([self.kp[cu[g]:cu[g + 1]], k]), np.concatenate([self.vp[cu[g]:cu[g + 1]], v])
                k_rows.append(k); v_rows.append(v); added.append((m, new))
            want, ws = O.decode_weights(self.q[x], k_rows, v_rows, scale=self.scale)
            for h in range(self.H_kv):
                k, n = k_rows[h], len(k_rows[h])
                q = self.q[x, h * G:(h + 1) * G]
                keep = np.isfinite(k).all(1)
                if not keep.any():
                    assert (out[x, h * G:(h + 1) * G] == 0).all()
                    continue
                a = (np.abs(q) @ np.where(np.isfinite(k), np.abs(k), 0).T).max()
                z = c * (q @ np.where(np.isfinite(k), k, 0).T)
                e = 2 * 0.6932 * (c * self.d / 4 * U * a + 4 * U * (np.abs(z).max() + np.log2(n))) + (n / 8 + 64) * U + 2.0 ** -21
                p = np.where(keep, np.exp2(z - z[:, keep].max(1, keepdims=True)), 0)
                spread = (p / p.sum(1, keepdims=True)) @ np.abs(np.where(keep[:, None], v_rows[h], 0))
                w = want[h * G:(h + 1) * G]
                off = np.abs(out[x, h * G:(h + 1) * G] - w)
                assert (off <= (B + e + n * U) * 1.01 * spread + B * np.abs(w)).all(), (x, h, off.max(), spread.max())
                if weights and slots:
                    m, new = added[h]
                    before = self.w[x, h].astype(np.float64).copy()
                    after = before.copy()
                    if new:
                        before[m] = after[m] = 0
                    after[:m + new] += ws[h][n - m - new:]
                    off = np.abs(w_got[x, h] - after)
                    assert (off <= e * (after - before) + 2 * U * after).all(), (x, h, off.max(), e)
                    assert (w_got[x, h, m + new:] == self.w[x, h, m + new:]).all()
                elif weights:
                    assert (w_got[x, h] == self.w[x, h]).all()


def run(A, s, **how):
    t = s.tensors(A, weights=how.pop("weights", True))
    check = {k: how[k] for k in ("append", "max_own", "slots") if k in how}
    s.call(A, t, **how)
    s.check(t, weights=t["slots"].weights is not None, **check)
    return t


GEOMETRIES = [(28, 4, 128), (8, 2, 256), (8, 2, 64), (3, 3, 128), (32, 1, 64), (17, 1, 128)]


@pytest.mark.parametrize("H_q,H_kv,d", GEOMETRIES)
@pytest.mark.parametrize("layout", ["head", "token", "strided"])
def test_ragged_prompts_and_own_rows(A, H_q, H_kv, d, layout):
    rng = np.random.default_rng(H_q + d)
    sharing = [3, 0, 1, 2]
    budgets = [int(b) for b in rng.choice([1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 300], 4 * H_kv)]
    budgets[1 % len(budgets)] = 0
    own = rng.choice([0, 1, 15, 31, 32, 63, 64, 65, 130], (6, H_kv))
    run(A, Step(rng, H_q, H_kv, d, budgets, sharing, own, 140, layout))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 16, 31, 32, 33, 64, 65, 96, 128, 129, 300])
def test_numbers_of_query_rows(A, d, rows):
    """Every division of a workgroup's waves: rows = sequences of one query head each."""
    rng = np.random.default_rng(rows + d)
    run(A, Step(rng, 1, 1, d, [333], [rows], [[int(n)] for n in rng.integers(0, 5, rows)], 8))


@pytest.mark.parametrize("n", [1, 2, 31, 33, 64, 127, 128, 129, 191, 192, 193, 257, 1000, 2500])
def test_lengths_of_own_rows(A, n):
    rng = np.random.default_rng(n)
    run(A, Step(rng, 7, 1, 128, None, None, [[n], [n - 1], [0]], n + 1))
    run(A, Step(rng, 4, 2, 64, None, None, [[n, n // 2]], n), append=False)


def test_many_chunks(A):
    """Heads of many chunks, whose boundaries lie in the middle of others' slots."""
    rng = np.random.default_rng(3)
    run(A, Step(rng, 4, 2, 64, [9000, 4001], [5], [[3, 700]] * 5, 701))
    run(A, Step(rng, 2, 1, 64, [150_000], [2], [[3], [9]], 16))          # more chunks than the join keeps factors of: 1172


def test_nothing_but_a_new_row(A):
    """The first token of sequences that share nothing: its own row, with weight one a query."""
    t = run(A, Step(np.random.default_rng(4), 6, 2, 64, None, None, [[0, 0]] * 3, 1))
    assert torch.allclose(t["slots"].weights, torch.full_like(t["slots"].weights, 3.0))


def test_only_the_prompt(A):
    s = Step(np.random.default_rng(5), 8, 2, 128, [70, 0, 1, 500], [4, 2], [[0, 0]] * 6, 4)
    t = run(A, s, append=False, slots=False)
    assert (t["out"][:4, 4:] == 0).all()                                 # head 1 of item 0 kept nothing
    run(A, s, append=False, max_own=0)


def test_agrees_with_decode_attend(A):
    """One sequence a prompt and no own rows: the step after the eviction, as before."""
    s = Step(np.random.default_rng(6), 28, 4, 128, [300, 20, 1000, 5] * 2, [1, 1], [[0] * 4] * 2, 4)
    t = run(A, s, append=False, slots=False)
    ref = A.decode_attend(A.Params(28, 4, 128, 1), t["q"], t["kp"], t["vp"], t["cu_b"], 2, len(s.kp))
    assert (t["out"].float() - ref).abs().max() <= 3 * B * ref.abs().max()


def test_full_caches_and_bounds(A):
    """A head that has max_own rows appends none; rows beyond max_own are not read; sequences behind the last one, and
    beyond max_seqs, stay as they are."""
    rng = np.random.default_rng(7)
    s = Step(rng, 4, 2, 64, None, None, [[10, 4], [9, 10]], 10)
    run(A, s, max_own=10)
    run(A, s, max_own=6)
    run(A, s, append=False, weights=False)
    run(A, Step(rng, 4, 2, 64, [50, 60, 9, 70], [2, 3], [[3, 8]] * 5, 12, spare=4))


def test_sequences_beyond_max_seqs_take_no_part(A):
    s = Step(np.random.default_rng(8), 4, 2, 64, [50, 60], [5], [[3, 8]] * 5, 12)
    t = s.tensors(A)
    s.call(A, t, max_seqs=3)
    s.active = 3
    s.check(t)


def test_peaked_and_rising_logits(A):
    """Logits of tens of octaves, rising along the rows: the reference follows."""
    rng = np.random.default_rng(9)
    s = Step(rng, 8, 2, 128, [700, 400], [9], [[200, 10]] * 9, 220, k_scale=1.0)
    for k in (s.kp, s.ko.reshape(-1, s.d)):
        k *= np.linspace(0.05, 14, len(k))[:, None]
    s.kp, s.ko = f64(bf16(s.kp)), f64(bf16(s.ko))
    run(A, s)


def test_infinite_keys_and_values_in_unused_places(A):
    """Keys at -inf have no weight; a query that sees nothing else gives zeros, and its rows gain nothing. (Unused slots hold
    NaN and infinities in every test here.)"""
    s = Step(np.random.default_rng(10), 4, 2, 64, [40, 70], [3], [[20, 6]] * 3, 24)
    s.q[..., 0] = np.abs(s.q[..., 0]) + 1
    s.q = f64(bf16(s.q))
    s.kp[:40, 0] = -np.inf                       # all of head 0's rows
    s.kp[50:60, 0] = -np.inf
    s.ko[0, 0, :, 0] = s.k_new[0, 0, 0] = -np.inf
    t = s.tensors(A)
    s.call(A, t)
    torch.cuda.synchronize()
    assert (t["out"][0, :2] == 0).all() and torch.isfinite(t["out"].float()).all()
    got = t["slots"].weights.cpu().numpy()
    assert np.array_equal(got[0, 0, :20], s.w[0, 0, :20]) and got[0, 0, 20] == 0
    s.check(t)


def test_equal_calls_equal_bits_on_a_stream_and_in_a_graph(A):
    rng = np.random.default_rng(11)
    s = Step(rng, 28, 4, 128, [500, 100, 900, 40], [6], [[70, 3, 200, 0]] * 6, 210)
    t = s.tensors(A)
    s.call(A, t)
    torch.cuda.synchronize()
    first = [t["out"].clone(), t["slots"].weights.clone(), t["slots"].lengths.clone()]
    again = s.tensors(A)
    ws = torch.empty(A.decode_shared_workspace_bytes(t["p"], 1, len(s.kp), 6, 6, s.max_own(True)), dtype=torch.uint8, device="cuda")
    begin = [again["slots"].weights.clone(), again["slots"].lengths.clone()]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        s.call(A, again, workspace=ws)
    torch.cuda.synchronize()
    slots = again["slots"]
    assert all(torch.equal(x, y) for x, y in zip(first, [again["out"], slots.weights, slots.lengths]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call(A, again, workspace=ws)
    for _ in range(3):
        slots.weights.copy_(begin[0]); slots.lengths.copy_(begin[1]); again["out"].zero_(); ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, [again["out"], slots.weights, slots.lengths]))
    # replayed without going back: the caches grow, step by step, to max_own
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert slots.lengths.view(6, 4)[0].tolist() == [74, 7, 201, 4]


def test_steps_in_a_row_are_one_long_attention(A):
    """Twelve steps of two sequences: at each, the own rows are those appended so far, and the weights add up."""
    rng = np.random.default_rng(12)
    s = Step(rng, 4, 2, 64, [90, 33], [2], [[0, 0]] * 2, 16)
    t = s.tensors(A)
    t["slots"].weights.zero_()
    ks, vs, total = [], [], np.zeros((2, 2, 16))
    cu = [0, 90, 123]
    for step in range(12):
        kn, vn, q = (f64(bf16(rng.standard_normal(x.shape))) for x in (s.k_new, s.v_new, s.q))
        for name, x in (("k_new", kn), ("v_new", vn), ("q", q)):
            t[name].copy_(bf16(x))
        ks.append(kn); vs.append(vn)
        s.call(A, t, max_own=16)
        out = f64(t["out"])
        for x in range(2):
            rows = [[np.concatenate([p[cu[h]:cu[h + 1]], np.stack([r[x, h] for r in new])]) for h in range(2)]
                    for p, new in ((s.kp, ks), (s.vp, vs))]
            want, w = O.decode_weights(q[x], rows[0], rows[1])
            assert np.abs(out[x] - want).max() <= 3 * B * max(np.abs(r).max() for r in rows[1])
            for h in range(2):
                total[x, h, :step + 1] += w[h][cu[h + 1] - cu[h]:]
    assert t["slots"].lengths.tolist() == [12] * 4
    got = t["slots"].weights.cpu().numpy()
    assert (np.abs(got - total) <= 1e-4 * total + 1e-30).all()


def test_offsets_beyond_32_bits(A):
    """Prompts and own rows whose elements lie further than 2^31 from the first: strided heads far apart, a stride from row to
    row that passes it within the cache, and a capacity that does."""
    rng = np.random.default_rng(13)
    for stride_head, stride_tok in (((1 << 31) + 4096, 64), (64, 1 << 25)):
        s = Step(rng, 4, 2, 64, None, None, [[70, 66]], 72)
        t = s.tensors(A, positions=False)
        span = stride_head + 71 * stride_tok + 64
        k, v = (torch.zeros(span, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        views = [x.as_strided((2, 72, 64), (stride_head, stride_tok, 1)) for x in (k, v)]
        views[0].copy_(bf16(s.ko[0])); views[1].copy_(bf16(s.vo[0]))
        slots = A.Slots(k, v, t["slots"].lengths, 72, t["slots"].weights)
        p = A.Params(4, 2, 64, 0, kv_stride_item=8, kv_stride_head=stride_head, kv_stride_tok=stride_tok)
        A.decode_shared(p, t["q"], None, None, None, 0, None, 1, slots=slots, max_own=71, k_new=t["k_new"], v_new=t["v_new"], out=t["out"])
        t["slots"] = A.Slots(views[0].contiguous()[None], views[1].contiguous()[None], slots.lengths, 72, slots.weights)
        s.check(t)
        A.evict_accumulated(p, slots, 1, 40, 0, 71)
        w = t["slots"].weights.cpu().numpy()
        del k, v, views
    s = Step(rng, 2, 2, 256, None, None, [[33, 5]], 40)
    t = s.tensors(A)
    C = (1 << 23) + 8                                             # slots of a head: head 1 begins 2^31 elements on
    big = [torch.zeros(1, 2, C, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    big[0][:, :, :40], big[1][:, :, :40] = t["slots"].k, t["slots"].v
    weights = torch.zeros(2, C, device="cuda")
    weights[:, :40] = t["slots"].weights.view(2, 40)
    slots = A.Slots(big[0], big[1], t["slots"].lengths, C, weights)
    A.decode_shared(t["p"], t["q"], None, None, None, 0, None, 1, slots=slots, max_own=40, k_new=t["k_new"], v_new=t["v_new"], out=t["out"])
    t["slots"] = A.Slots(big[0][:, :, :40].contiguous(), big[1][:, :, :40].contiguous(), slots.lengths, 40, weights[:, :40].contiguous())
    s.check(t, max_own=40)


@pytest.mark.parametrize("n_items", [1, 40, 70, 130])
def test_many_items(A, n_items):
    """Tables of items and heads that a wave loads at once, and longer ones that it probes."""
    rng = np.random.default_rng(n_items)
    sharing = [int(x) for x in rng.integers(0, 3, n_items)]
    sharing[-1] = 2
    budgets = [int(x) for x in rng.integers(0, 9, 2 * n_items)]
    own = rng.integers(0, 4, (sum(sharing), 2))
    run(A, Step(rng, 4, 2, 64, budgets, sharing, own, 5, spare=2))


def test_what_the_binding_refuses(A):
    s = Step(np.random.default_rng(14), 4, 2, 64, [5, 6], [2], [[1, 2]] * 2, 8)
    t = s.tensors(A)

    def call(**change):
        u = {**t, **change}
        A.decode_shared(u["p"], u["q"], u["kp"], u["vp"], u["cu_b"], u.get("rows", 11), u["cu_s"], 2, slots=u["slots"], max_own=4,
                        k_new=u["k_new"], v_new=u["v_new"], pos_new=u["pos"], out=u["out"])
    short = A.Slots(t["slots"].k, t["slots"].v, t["slots"].lengths, 9, t["slots"].weights, t["slots"].positions)
    for change in (dict(q=t["q"].float()), dict(q=t["q"].cpu()), dict(q=t["q"].transpose(1, 2)), dict(kp=t["kp"][:10].contiguous()),
                   dict(rows=12), dict(cu_b=t["cu_b"][:2].contiguous()), dict(cu_b=t["cu_b"].long()), dict(k_new=t["k_new"][:1]),
                   dict(pos=t["pos"][:1]), dict(out=t["out"][:1]), dict(out=t["out"].float()), dict(slots=short)):
        with pytest.raises(ValueError):
            call(**change)
    call()
    s.check(t, max_own=4)
    slots = t["slots"]
    slots.lengths = slots.lengths[:3].contiguous()                # what was looked at before is looked at again
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("H_q,H_kv,d", [(28, 4, 128), (16, 2, 64), (8, 1, 128)])
def test_prompts_that_many_sequences_share(A, H_q, H_kv, d):
    """Several blocks of query rows on long prompts, ragged, and sequences in different numbers, own rows beside them."""
    rng = np.random.default_rng(d + H_q)
    G = H_q // H_kv
    sharing = [max(1, 130 // G), 300 // G + 1, 1]
    budgets = [int(x) for x in rng.integers(40000 // H_kv, 60000 // H_kv, 3 * H_kv)]
    budgets[0], budgets[-1] = 33, 0
    n = sum(sharing)
    s = Step(rng, H_q, H_kv, d, budgets, sharing, rng.integers(0, 70, (n, H_kv)), 72)
    t = s.tensors(A)
    s.call(A, t)
    # every seventh sequence, the rest by its being like them
    keep = list(range(0, n, 7))
    item_of = np.repeat(np.arange(3), sharing)
    for name in ("q", "own", "ko", "vo", "k_new", "v_new", "w"):
        setattr(s, name, getattr(s, name)[keep])
    s.sharing = [int((item_of[keep] == i).sum()) for i in range(3)]
    s.n = s.active = len(keep)
    heads = (np.array(keep)[:, None] * H_kv + np.arange(H_kv)).reshape(-1)
    at = torch.from_numpy(heads).cuda()
    sl = t["slots"]
    t["out"] = t["out"][keep]
    t["slots"] = A.Slots(sl.k[keep], sl.v[keep], sl.lengths[at], 72, sl.weights.view(n * H_kv, -1)[at], None)
    s.check(t)


def test_prompts_without_rows(A):
    """A compacted cache that kept nothing: sequences have their own rows, or nothing at all."""
    rng = np.random.default_rng(16)
    run(A, Step(rng, 4, 2, 64, [0] * 4, [1, 2], [[3, 0], [0, 70], [1, 5]], 80, spare=1))
