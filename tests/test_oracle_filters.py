"""CPU pins of the oracle's sampling filters, filtered consensus, page tables and packed store: hand-worked cases, closed
forms and invariants."""
import numpy as np
import pytest

import oracle

LOG = np.log


def test_hand_worked_row():
    x = LOG(np.array([0.1, 0.4, 0.2, 0.25, 0.05]))
    for args, want in [((1.0,), {0: .1, 1: .4, 2: .2, 3: .25, 4: .05}),
                       ((1.0, 3), {1: .4 / .85, 2: .2 / .85, 3: .25 / .85}),
                       ((1.0, 0, 0.6), {1: .4 / .65, 3: .25 / .65}),
                       ((1.0, 0, 0.66), {1: .4 / .85, 2: .2 / .85, 3: .25 / .85}),
                       ((1.0, 2, 0.6), {1: 1.0}),             # .4 of .65 is .615: top-p counts what top-k left
                       ((1.0, 0, 1.0, 0.45), {1: .4 / .85, 2: .2 / .85, 3: .25 / .85}),
                       ((0.5, 0, 1.0, 0.3), {1: .16 / .2225, 3: .0625 / .2225}),
                       ((0.0, 3, 0.2), {1: 1.0}), ((1.0, 0, 0.0), {1: 1.0}), ((1.0, 0, 1.0, 7.0), {1: 1.0})]:
        idx, p = oracle.filter_row(x, *args)
        assert idx.tolist() == sorted(want), args
        np.testing.assert_allclose(p, [want[i] for i in idx], rtol=1e-12)


def test_ties_go_to_the_lower_index_and_special_logits():
    assert oracle.filter_row(np.zeros(6), 1.0, 2)[0].tolist() == [0, 1]
    assert oracle.filter_row(np.zeros(6), 1.0, 0, 0.5)[0].tolist() == [0, 1, 2]
    assert oracle.filter_row(np.array([1.0, 3.0, 3.0, np.nan]), -1.0)[0].tolist() == [1]
    idx, p = oracle.filter_row(np.array([np.inf, 1.0, np.nan, np.inf, -np.inf]), 1.0)
    assert p[idx == 0] == p[idx == 3] == 0.5 and 2 not in idx and 4 not in idx
    assert oracle.filter_row(np.full(4, -np.inf), 1.0)[0].size == 0
    low = np.finfo(np.float32).min
    assert oracle.filter_row(np.array([low, 0.0, low]), 1.0)[1].tolist() == [0.0, 1.0, 0.0]
    np.testing.assert_array_equal(oracle.filter_row(np.full(3, low), 1.0)[1], 1 / 3)


def test_tokens_follow_the_distribution_over_a_grid_of_uniforms():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((1, 1, 23)).astype(np.float32) * 2
    f = (np.array([0.8]), np.array([15]), np.array([0.9]), np.array([0.02]))
    idx, p = oracle.filter_row(x[0, 0], 0.8, 15, 0.9, 0.02)
    n = 4000
    grid = (np.arange(n) + 0.5) / n
    got = np.array([oracle.sample_tokens(x, *f, np.array([[u]]))[0][0, 0] for u in grid])
    assert (np.diff(got) >= 0).all() and set(got) <= set(idx)      # inverse of a distribution function over the index
    for i, q in zip(idx, p):
        assert abs((got == i).mean() - q) <= 1.0 / n + 1e-12
    tokens, lp, _ = oracle.sample_tokens(x, *f, np.array([[0.3]]))
    assert abs(lp[0, 0] - LOG(p[idx == tokens[0, 0]])[0]) < 1e-12


def test_filtered_consensus_is_lossless():
    """First emitted token of a block, over draws of the draft and the uniforms: distributed as the filtered p."""
    rng = np.random.default_rng(5)
    V, n = 6, 20000
    ar, df = rng.standard_normal((1, 1, V)), rng.standard_normal((1, 1, V))
    f = (np.array([0.9]), np.array([4]), np.array([0.95]), np.array([0.05]))
    pi, p = oracle.filter_row(ar[0, 0], 0.9, 4, 0.95, 0.05)
    count = np.zeros(V)
    for _ in range(n):
        x = oracle.sample_tokens(df, *f, rng.random((1, 1)))[0]
        r = oracle.filtered_consensus_commit(ar, df, *f, x, rng.random((1, 1)), rng.gumbel(size=(1, V)))
        count[r["out_tokens"][0, 0]] += 1
    want = np.zeros(V)
    want[pi] = p
    assert np.all(np.abs(count / n - want) < 5 * np.sqrt(want * (1 - want) / n) + 1e-9)


def test_filtered_consensus_without_filters_is_the_sampling_consensus():
    from orthrus_inputs import Workload, make_sampling_case
    w = Workload(name="f", batch=3, num_q_heads=2, num_kv_heads=1, head_dim=64, block_k=5, vocab=301, context=5)
    c = make_sampling_case(w, seed=9, temperature=0.7, divergence=0.4)
    a = oracle.sampling_consensus_commit(c["ar_logits"], c["diff_logits"], c["draft_tokens"], c["accept_u"], c["gumbel"], 0.7)
    b = oracle.filtered_consensus_commit(c["ar_logits"], c["diff_logits"], np.full(3, 0.7), None, None, None,
                                         c["draft_tokens"], c["accept_u"], c["gumbel"])
    for k in ("accept_len", "num_committed", "out_tokens", "next_anchor"):
        np.testing.assert_array_equal(a[k], b[k])


def test_page_tables_by_hand():
    P, N = 4, 10
    table = np.array([[7, 2, -1, -1], [5, -1, -1, -1], [1, 3, 9, -1], [-1, -1, -1, -1]], np.int32)
    ring = np.array([0, 4, 6, 8, -1, -1, -1, -1, -1, -1], np.int32)
    state, slots = np.array([0, 4], np.int32), np.full(12, -9, np.int32)
    granted, starts, status = oracle.page_tables_update([6, 4, 9, 0], [5, 2, -1, 3], table, ring, state, P, 16, 12, slots)
    assert status == 0 and granted.tolist() == [5, 2, 0, 3] and starts.tolist() == [0, 5, 7, 7, 10]
    assert table.tolist() == [[7, 2, 0, -1], [5, 4, -1, -1], [-1] * 4, [6, -1, -1, -1]]
    assert slots.tolist() == [10, 11, 0, 1, 2, 16, 17, 24, 25, 26, -9, -9]
    assert state.tolist() == [3, 4] and ring[3:7].tolist() == [8, 1, 3, 9]


def test_page_tables_short_ring_bad_lengths_and_torn_pages():
    P, N = 4, 6
    table = np.full((4, 3), -1, np.int32)
    ring, state, slots = np.arange(N, dtype=np.int32), np.array([4, 3], np.int32), np.full(40, -9, np.int32)
    granted, starts, status = oracle.page_tables_update([0, 0, 0, 0], [8, 8, 0, 4], table, ring, state, P, 12, 40, slots)
    # two pages of three go to the first; the second lacks two more (four wanted), the last would make five
    assert status == -4 and granted.tolist() == [8, 0, 0, 0] and table[0].tolist() == [4, 5, -1] and (table[1:] == -1).all()
    assert state.tolist() == [0, 1]
    for L, n in ((-1, 2), (10, 3), (2, 1)):      # negative, too long, inside a page that is not there
        t = np.full((1, 3), -1, np.int32)
        g, _, st = oracle.page_tables_update([L], [n], t, ring, np.array([0, 6], np.int32), P, 12, 40, slots)
        assert st == -4 and g.tolist() == [0] and (t == -1).all()


def test_store_by_hand():
    k = np.arange(2 * 3 * 1 * 2, dtype=np.uint16).reshape(2, 3, 1, 2)
    kp, vp = np.zeros((2, 2, 1, 4, 2), np.uint16), np.zeros((2, 2, 1, 4, 2), np.uint16)
    assert oracle.kv_store(k, k + 100, [5, -1, 0], kp, vp) == 0
    np.testing.assert_array_equal(kp[:, 1, 0, 1], k[:, 0, 0])
    np.testing.assert_array_equal(vp[:, 0, 0, 0], k[:, 2, 0] + 100)
    assert np.count_nonzero(kp.any(-1)) == 4 - 0
    assert oracle.kv_store(k, k, [8], kp, vp) == -4


@pytest.mark.parametrize("seed", range(4))
def test_pages_are_conserved(seed):
    """Whatever is asked, every page is in exactly one place: an entry of the table or the ring."""
    rng = np.random.default_rng(seed)
    B, width, N, P = 7, 9, 40, 16
    table, ring, state = np.full((B, width), -1, np.int32), rng.permutation(N).astype(np.int32), np.array([11, N], np.int32)
    lens = np.zeros(B, np.int64)
    for _ in range(60):
        new = rng.integers(0, 40, B)
        new[rng.random(B) < 0.2] = -1
        granted, _, _ = oracle.page_tables_update(lens, new, table, ring, state, P, width * P, 1000, np.zeros(1000, np.int32))
        lens = np.where(new < 0, 0, lens + granted)
        free = [int(ring[(state[0] + i) % N]) for i in range(state[1])]
        assert sorted(free + table[table >= 0].tolist()) == list(range(N))
        assert all((table[b, :(lens[b] + P - 1) // P] >= 0).all() for b in range(B))
