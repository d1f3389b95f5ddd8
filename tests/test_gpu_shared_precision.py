"""How exact decode_shared's weights are when they meet V, against the float64 oracle. With u = 2^-24 and b = 2^-8 (bf16), the relative
error of one rounding: a weight p is the sum of two bf16 values, the upper half of its bits (or one step less) and the rest, which is
at most 2^-7 p and rounded once more: 2^-15 p. Its logit, sum and exponential add e p as in test_gpu_shared.py, the sum over n rows
n u, the output's rounding b |out|. So out is off by (2^-15 + e + n u) sum p |v| + b |out|: where a sum cancels, far less than one
rounding of each weight to bf16."""
import numpy as np
import pytest
import torch

from oracle import audiokv_oracle as O
from test_gpu_shared import A, B, Step, U, bf16, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H_q,H_kv,d", [(28, 4, 128), (8, 2, 256), (8, 2, 64), (32, 1, 64), (2, 2, 128)])
@pytest.mark.parametrize("sharing,rows,own", [([1], 700, 0), ([4, 2], 900, 40), ([40], 2000, 3), (None, 0, 333)])
def test_weights_keep_sixteen_bits(A, H_q, H_kv, d, sharing, rows, own):
    rng = np.random.default_rng(H_q + d + rows)
    n_items = len(sharing or [])
    n = sum(sharing or [5])
    s = Step(rng, H_q, H_kv, d, [rows + 7 * g for g in range(n_items * H_kv)] if sharing else None, sharing, [[own] * H_kv] * n, own + 1)
    t = s.tensors(A)
    s.call(A, t)
    torch.cuda.synchronize()
    out, cu = f64(t["out"]), np.concatenate([[0], np.cumsum(s.budgets or [])]).astype(int)
    item_of = np.repeat(np.arange(n_items), sharing) if sharing else None
    c, G = d ** -0.5 * 1.4426950408889634, H_q // H_kv
    for x in range(0, n, max(1, n // 5)):
        k_rows, v_rows = [], []
        for h in range(H_kv):
            k, v = np.concatenate([s.ko[x, h, :own], s.k_new[x, h][None]]), np.concatenate([s.vo[x, h, :own], s.v_new[x, h][None]])
            if sharing:
                g = item_of[x] * H_kv + h
                k, v = np.concatenate([s.kp[cu[g]:cu[g + 1]], k]), np.concatenate([s.vp[cu[g]:cu[g + 1]], v])
            k_rows.append(k); v_rows.append(v)
        want, _ = O.decode_weights(s.q[x], k_rows, v_rows)
        for h in range(H_kv):
            q, k, m = s.q[x, h * G:(h + 1) * G], k_rows[h], len(k_rows[h])
            z = c * (q @ k.T)
            e = 2 * 0.6932 * (c * d / 4 * U * (np.abs(q) @ np.abs(k).T).max() + 4 * U * (np.abs(z).max() + np.log2(m))) + (m / 8 + 64) * U + 2.0 ** -21
            p = np.exp2(z - z.max(1, keepdims=True))
            spread = (p / p.sum(1, keepdims=True)) @ np.abs(v_rows[h])
            w = want[h * G:(h + 1) * G]
            off = np.abs(out[x, h * G:(h + 1) * G] - w)
            assert (off <= (2.0 ** -15 + e + m * U) * 1.01 * spread + B * np.abs(w)).all(), (x, h, (off / spread).max(), e)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_infinite_values_that_have_weight(A, d):
    """A value of +inf or -inf makes its channel that; queries of zero, so that weights are powers of two, and others."""
    for zero in (True, False):
        s = Step(np.random.default_rng(d), 4, 2, d, [40, 64], [3], [[23, 0]] * 3, 24)
        s.vp[5, 3], s.vp[77, 9], s.vo[1, 0, 20, d - 1] = np.inf, -np.inf, np.inf
        if zero:
            s.q[:] = 0
        t = s.tensors(A)
        s.call(A, t)
        torch.cuda.synchronize()
        out = f64(t["out"])
        assert (out[:, :2, 3] == np.inf).all() and (out[:, 2:, 9] == -np.inf).all() and (out[1, :2, d - 1] == np.inf).all()
        out[:, :2, 3] = out[:, 2:, 9] = out[1, :2, d - 1] = 0
        assert np.isfinite(out).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_stays_where_it_is(A, d):
    """A query of NaN gives NaN, and NaN weights to the rows that its group owns; a value of NaN makes its channel that. Nothing else is."""
    s = Step(np.random.default_rng(d), 6, 2, d, [40, 64], [3], [[23, 5]] * 3, 24)
    s.q[1, 4], s.vp[70, 11] = np.nan, np.nan                  # query head 4 of sequence 1, in the group of KV head 1; a row of head 1
    t = s.tensors(A)
    s.call(A, t)
    torch.cuda.synchronize()
    out, w = f64(t["out"]), t["slots"].weights.cpu().numpy()
    assert np.isnan(out[1, 4]).all() and np.isnan(out[:, 3:, 11]).all() and np.isnan(w[1, 1, :6]).all()
    out[1, 4] = out[:, 3:, 11] = 0
    w[1, 1, :6] = 0
    assert np.isfinite(out).all() and np.isfinite(w).all()
