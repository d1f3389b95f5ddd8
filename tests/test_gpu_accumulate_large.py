"""The kernels that large calls of accumulate take (two stationary tiles a wave) with what the small ones are tested with: given
log-sum-exp, chunks of queries in a padded slab, no mask, logits that rise, tokens at -inf, a query of NaN. Against torch in 64 bits
on the device; tolerance as derived in test_gpu_accumulate.py, its largest logits and products found over all pairs."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LOG2E = 1.4426950408889634


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


class Call:
    """Items (L, Q); K padded to T tokens a head, q [H_q][Q][d] of item after item."""

    def __init__(self, seed, H_q, H_kv, d, items):
        self.H_q, self.H_kv, self.d, self.items, self.T = H_q, H_kv, d, items, max(L for L, _ in items) + 5
        gen = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
        self.k = draw(len(items), H_kv, self.T, d)
        self.q = [draw(H_q, Q, d) for _, Q in items]
        self.gone = torch.zeros(self.T, dtype=torch.bool, device="cuda")      # tokens at -inf

    def logits(self, i, j, causal):
        """[Q, L] of query head j, base e, in 64 bits; what a query does not see is -inf."""
        L, Q = self.items[i]
        k = torch.where(self.gone[:L, None], 0, self.k[i, j * self.H_kv // self.H_q, :L].double())
        z = self.q[i][j].double() @ k.T.contiguous() * self.d ** -0.5
        z.masked_fill_(self.gone[:L], -np.inf)
        if causal:
            z.masked_fill_(torch.arange(L, device="cuda") > L - Q + torch.arange(Q, device="cuda")[:, None], -np.inf)
        return z

    def lse(self, causal=True):
        return torch.cat([torch.cat([self.logits(i, j, causal).logsumexp(1) for j in range(self.H_q)]) for i in range(len(self.items))]).float()

    def run(self, A, lse=None, causal=True):
        lens, queries = [L for L, _ in self.items], [Q for _, Q in self.items]
        pairs = sum((Q * (L - Q) + Q * (Q + 1) / 2 if causal else Q * L) for L, Q in self.items) * self.H_q
        assert pairs / (2 * 7 * 32 * 64) >= 8 * 256                           # two tiles a wave: eight tiles of work for every CU
        k = self.k.clone()
        for i, (L, _) in enumerate(self.items):
            k[i, :, L:] = float("nan")                                        # rows past an item's end are never used
        k[:, :, self.gone, 0] = -float("inf")
        p = A.Params(self.H_q, self.H_kv, self.d, 0, causal=int(causal), kv_stride_item=self.H_kv * self.T * self.d,
                     kv_stride_head=self.T * self.d, kv_stride_tok=self.d)
        w = A.accumulate(p, torch.cat([q.reshape(-1) for q in self.q]), k.view(-1), lens, queries, pitch=self.T, lse=lse)
        w = w.view(len(lens), self.H_kv, self.T)
        for i, L in enumerate(lens):
            assert (w[i, :, L:] == 0).all()
        return w

    def check(self, w, causal=True):
        G, c = self.H_q // self.H_kv, self.d ** -0.5 * LOG2E
        for i, (L, Q) in enumerate(self.items):
            want, a, x = torch.zeros(self.H_kv, L, dtype=torch.float64, device="cuda"), 0.0, 0.0
            for j in range(self.H_q):
                z = self.logits(i, j, causal)
                x = max(x, z[z.isfinite()].abs().max().item() * LOG2E)
                want[j // G] += torch.softmax(z, dim=1).nan_to_num_(nan=0.0).sum(0)          # (a query that sees nothing)
                k = torch.where(self.gone[:L, None], 0, self.k[i, j // G, :L]).abs().float()
                a = max(a, (self.q[i][j].abs().float() @ k.T.contiguous()).max().item())
            tol = 2 * 0.6932 * (c * self.d / 4 * U * a + 4 * U * (x + np.log2(L))) + (L / 16 + G * Q / 16 + 64) * U + 2.0 ** -21
            off = (w[i, :, :L].double() - want).abs()
            assert (off <= tol * want + 1e-30).all(), (i, (off / (want + 1e-30)).max().item(), tol)


GEOMETRIES = [(8, 2, 64), (28, 4, 128), (8, 2, 256)]


def items_of(H_q):
    return [(4500, 2700), (700, 31), (1203, 1203)] if H_q == 8 else [(2600, 1500), (700, 31), (903, 903)]


@pytest.mark.parametrize("H_q,H_kv,d", GEOMETRIES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("given", [False, True])
def test_chunks_in_a_slab(A, H_q, H_kv, d, causal, given):
    c = Call(d, H_q, H_kv, d, items_of(H_q))
    c.check(c.run(A, lse=c.lse(causal) if given else None, causal=causal), causal)


@pytest.mark.parametrize("H_q,H_kv,d", GEOMETRIES)
@pytest.mark.parametrize("falling", [False, True])
def test_logits_far_from_the_first(A, H_q, H_kv, d, falling):
    """Rising by hundreds of octaves along the keys, or falling: the reference of a row has to follow, in either of a wave's tiles."""
    c = Call(d + 1, H_q, H_kv, d, items_of(H_q))
    for i, (L, _) in enumerate(c.items):
        rise = torch.linspace(0.1, 12, L, device="cuda")
        c.k[i, :, :L] *= (rise.flip(0) if falling else rise)[:, None].bfloat16()
        c.q[i] *= 4
    c.check(c.run(A))


@pytest.mark.parametrize("H_q,H_kv,d", GEOMETRIES)
def test_tokens_at_minus_infinity(A, H_q, H_kv, d):
    """They have no weight wherever they stand; the first queries of the last item see nothing else and give nothing."""
    c = Call(d + 2, H_q, H_kv, d, items_of(H_q))
    c.gone[:100] = c.gone[640:777] = True
    for q in c.q:
        q[..., 0] = q[..., 0].abs() + 1
    w = c.run(A)
    assert w.isfinite().all() and (w[:, :, c.gone] == 0).all()
    c.check(w)
    lse = c.lse()
    assert (lse == -np.inf).any()
    c.check(c.run(A, lse=lse))


@pytest.mark.parametrize("H_q,H_kv,d", GEOMETRIES)
@pytest.mark.parametrize("given", [False, True])
def test_nan_of_a_query_reaches_only_what_it_sees(A, H_q, H_kv, d, given):
    c = Call(d + 3, H_q, H_kv, d, items_of(H_q))
    L, Q = c.items[0]
    for at in (0, 900, Q - 300):
        q = c.q[0][0, at].clone()
        c.q[0][0, at] = float("nan")
        w = c.run(A, lse=c.lse() if given else None)
        seen = L - Q + at + 1
        assert w[0, 0, :seen].isnan().all() and w[0, 0, seen:].isfinite().all() and w[0, 1:].isfinite().all() and w[1:].isfinite().all()
        c.q[0][0, at] = 0                                     # (what it sees aside, that query changes nothing)
        clean = c.run(A, lse=c.lse() if given else None)
        assert torch.equal(w[0, 0, seen:], clean[0, 0, seen:]) and torch.equal(w[0, 1:], clean[0, 1:]) and torch.equal(w[1:], clean[1:])
        c.q[0][0, at] = q


@pytest.mark.parametrize("given", [False, True])
def test_few_queries_on_a_long_prompt(A, given):
    """One block of rows, or many of keys, cut between all workgroups: 256 parts of a row's statistics."""
    c = Call(77, 7, 1, 128, [(131072, 3), (90000, 120)])
    lens, queries = [131072, 90000], [3, 120]
    k = c.k.clone()
    k[1, :, 90000:] = float("nan")
    p = A.Params(7, 1, 128, 0, kv_stride_item=c.T * 128, kv_stride_head=c.T * 128, kv_stride_tok=128)
    w = A.accumulate(p, torch.cat([q.reshape(-1) for q in c.q]), k.view(-1), lens, queries, pitch=c.T, lse=c.lse() if given else None)
    c.check(w.view(2, 1, c.T))


@pytest.mark.parametrize("H_q,H_kv,d,L,Q", [(64, 1, 64, 300, 300), (100, 1, 128, 200, 170), (96, 2, 256, 500, 3)])
def test_many_query_heads_a_head(A, H_q, H_kv, d, L, Q):
    """More of them than a load's rows, and than a tile's."""
    c = Call(H_q, H_q, H_kv, d, [(L, Q), (40, 40)])
    p = A.Params(H_q, H_kv, d, 0, kv_stride_item=H_kv * c.T * d, kv_stride_head=c.T * d, kv_stride_tok=d)
    w = A.accumulate(p, torch.cat([q.reshape(-1) for q in c.q]), c.k.view(-1), [L, 40], [Q, 40], pitch=c.T)
    c.check(w.view(2, H_kv, c.T))


def test_given_lse_needs_no_workspace_where_no_block_is_shared(A):
    """No queries but of one item, one block of keys, one workgroup: the library takes a workspace of no bytes, and of no address."""
    import ctypes as C
    c = Call(5, 4, 2, 64, [(60, 8)])
    p = A.Params(4, 2, 64, 0, kv_stride_item=2 * c.T * 64, kv_stride_head=c.T * 64, kv_stride_tok=64)
    cu, cu_q = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (60, 8))
    w, lse, one = torch.zeros(2 * c.T, device="cuda"), c.lse(), lambda n: (C.c_int32 * 1)(n)
    rc = A.binding._lib.audiokv_accumulate(C.byref(p.c()), c.q[0].data_ptr(), c.k.data_ptr(), lse.data_ptr(), cu.data_ptr(), one(60), cu_q.data_ptr(),
                                           one(8), 1, w.data_ptr(), c.T, None, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == 0, A.binding._lib.audiokv_last_error()
    c.check(w.view(1, 2, c.T))
