"""The paged-cache oracle against closed forms and the contiguous oracle (CPU only)."""
import numpy as np
import pytest

import oracle


def test_slots_by_hand():
    # pages of 4; request 0 has 3 tokens on page 9 and gets 3 more, request 1 is new with 5
    table, q_start, kv, slots, pos, used = oracle.paged_slots_reference([3, 0], [3, 5], [7, 5, 2, 8], 1, 4, [[9, -1], [-1, -1]], 9)
    assert table.tolist() == [[9, 5], [2, 8]] and q_start.tolist() == [0, 3, 8] and kv.tolist() == [6, 5] and used == 4
    assert slots.tolist() == [39, 20, 21, 8, 9, 10, 11, 32, -1] and pos.tolist() == [3, 4, 5, 0, 1, 2, 3, 4, 0]


def test_slots_run_out_and_rows_end():
    table, _, _, slots, _, used = oracle.paged_slots_reference([0, 0], [3, 9], [4], 0, 2, [[-1] * 3, [-1] * 3], 12)
    assert table.tolist() == [[4, -1, -1], [-1, -1, -1]] and used == 5
    assert slots.tolist() == [8, 9, -1] + [-1] * 9


def test_norm_and_rotation_agree_with_the_layer_steps():
    rng = np.random.default_rng(0)
    T, H, d = 5, 3, 64
    x = rng.standard_normal((T, H * d))
    gamma = rng.standard_normal(d)
    pos = np.arange(7, 7 + T)[None]
    ref, _ = oracle.qk_norm_rope_reference(x, H, d, gamma, 1e-6, pos, np.zeros(32, dtype=int), d, 1e4)
    rows, _ = oracle.rmsnorm_reference(x.reshape(-1, d), gamma, 1e-6)
    want, _ = oracle.rope_reference(rows.reshape(T, H * d), H, d, 7, 1e4)
    assert np.allclose(ref, want, atol=1e-12)


def test_axes_and_partial_rotation():
    x = np.ones((1, 8))
    ref, _ = oracle.qk_norm_rope_reference(x, 1, 8, None, 0.0, [[0], [1]], [0, 1], 4, 100.0)
    c, s = np.cos(0.1), np.sin(0.1)  # the second pair turns by 1 * 100^(-2/4)
    assert np.allclose(ref[0], [1, c - s, 1, c + s, 1, 1, 1, 1])


def _paged(rng, kv, page, Hk, d):
    need = [-(-n // page) for n in kv]
    perm = rng.permutation(sum(need) + 2)
    table = np.full((len(kv), max(need)), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = perm[at:at + n]
        at += n
    return table, rng.standard_normal((len(perm), page, Hk, d)), rng.standard_normal((len(perm), page, Hk, d))


def test_full_visibility_is_the_contiguous_attention():
    rng = np.random.default_rng(1)
    kv, H, Hk, d, page = [37], 4, 2, 16, 8
    table, K, V = _paged(rng, kv, page, Hk, d)
    Q = rng.standard_normal((5, H * d))
    ref, bound = oracle.paged_attention_reference(Q, K, V, table, [0, 5], kv, H, 0.25, prefix=[37])
    idx = np.arange(37)
    k, v = (c[table[0][idx // page], idx % page].reshape(37, -1) for c in (K, V))
    want, wbound = oracle.attention_reference(Q, k[:20], v[:20], k[20:], v[20:], H, Hk, d, 0.25)
    assert np.allclose(ref, want, atol=1e-12) and np.allclose(bound, wbound)


def test_causal_window_and_cap_one_by_one():
    rng = np.random.default_rng(2)
    kv, page, d = [9, 4], 4, 8
    table, K, V = _paged(rng, kv, page, 1, d)
    Q = rng.standard_normal((5, d))
    ref, _ = oracle.paged_attention_reference(Q, K, V, table, [0, 3, 5], kv, 1, 0.7, cap=1.5, window=3)
    for t, (r, p) in enumerate([(0, 6), (0, 7), (0, 8), (1, 2), (1, 3)]):
        js = range(max(0, p - 2), p + 1)
        k = np.array([K[table[r, j // page], j % page, 0] for j in js])
        v = np.array([V[table[r, j // page], j % page, 0] for j in js])
        w = np.exp(1.5 * np.tanh(0.7 * k @ Q[t] / 1.5))
        assert np.allclose(ref[t], w @ v / w.sum())


def test_rows_without_keys_and_missing_pages():
    rng = np.random.default_rng(3)
    table, K, V = _paged(rng, [6], 4, 1, 8)
    ref, bound = oracle.paged_attention_reference(rng.standard_normal((9, 8)), K, V, table, [0, 8], [6], 1, 1.0)
    assert (ref[:2] == 0).all() and (ref[2:8] != 0).any() and (ref[8] == 0).all() and (bound > 0).all()
    table[0, 0] = -1  # a page of zeros
    ref, _ = oracle.paged_attention_reference(np.zeros((1, 8)), K, V, table, [0, 1], [6], 1, 1.0)
    assert np.allclose(ref[0], V[table[0, 1], :2, 0].sum(0) / 6)


@pytest.mark.parametrize("weight_bits", [8, 16])
def test_bound_covers_rounded_weights(weight_bits):
    """fp32 scores, weights rounded to that many significant bits, fp32 sums and a bf16 store stay within the bound."""
    rng = np.random.default_rng(4)
    table, K, V = _paged(rng, [300], 16, 1, 64)
    K, V = oracle.bf16_round(K), oracle.bf16_round(V)
    Q = oracle.bf16_round(rng.standard_normal((4, 64)))
    ref, bound = oracle.paged_attention_reference(Q, K, V, table, [0, 4], [300], 1, 0.125, weight_error=2.0 ** -8 if weight_bits == 8 else 0.0)
    idx = np.arange(300)
    k, v = (c[table[0][idx // 16], idx % 16, 0].astype(np.float32) for c in (K, V))
    for i in range(4):
        n = 297 + i
        s = (k[:n] @ Q[i].astype(np.float32)) * np.float32(0.125)
        w = np.exp(s - s.max())
        m, e = np.frexp(w)
        wr = np.ldexp(np.round(m * 2 ** weight_bits) / 2 ** weight_bits, e)
        o = oracle.bf16_round((wr @ v[:n]) / w.sum())
        assert (np.abs(o - ref[i]) <= bound[i]).all()
