"""CPU pins of the oracle's tree attention, tree consensus and logit rules: hand-worked cases and closed forms, and their agreement
with the chain's own oracle where a tree is a chain."""
import numpy as np

import oracle
from orthrus_inputs import bf16_bits_to_f32


def _bits(rng, *shape):
    return (rng.standard_normal(shape).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def test_paths():
    up = [-1, 0, 0, 1, 3, -1, 5, 9, 2, 2, 7, -1]
    want = {0: [0], 1: [0, 1], 2: [0, 2], 3: [0, 1, 3], 4: [0, 1, 3, 4], 8: [0, 2, 8], 9: [0, 2, 9]}
    for i in range(12):
        assert oracle.tree_path(up, i) == want.get(i, [0])   # 5, 6, 7 (follows a later node), 10 and 11 are unused


def test_a_chain_is_the_ar_view_and_siblings_do_not_see_one_another():
    rng = np.random.default_rng(1)
    B, K, Hq, H, d, P = 2, 5, 4, 2, 64, 16
    q, k, v = _bits(rng, B, K, Hq, d), _bits(rng, B, K, H, d), _bits(rng, B, K, H, d)
    kp, vp = _bits(rng, 9, H, P, d), _bits(rng, 9, H, P, d)
    table, lens = rng.permutation(9)[:8].reshape(2, 4).astype(np.int32), np.array([37, 0], np.int32)
    f = [bf16_bits_to_f32(x) for x in (q, k, v, kp, vp)]
    chain = np.tile(np.arange(-1, K - 1), (B, 1))
    got = oracle.tree_attn(0.125, chain, *f, table, lens)[0]
    np.testing.assert_allclose(got, oracle.dual_view_attn(1, 0.125, q, k, v, kp, vp, table, lens), rtol=1e-12, atol=1e-14)
    # every node on the root: what the chain gives for two rows, whatever the others hold
    star = np.tile([-1] + [0] * (K - 1), (B, 1))
    got, size, lse = oracle.tree_attn(0.125, star, *f, table, lens)
    for i in range(1, K):
        two = [x[:, [0, i]] for x in f[:3]]
        w = oracle.tree_attn(0.125, chain[:, :2], *two, *f[3:], table, lens)
        np.testing.assert_allclose(got[:, i], w[0][:, 1], rtol=1e-12)
        np.testing.assert_allclose(lse[:, :, i], w[2][:, :, 1], rtol=1e-12)
    assert (size >= np.abs(got) - 1e-12).all()


def test_a_chain_of_drafts_is_the_greedy_consensus():
    rng = np.random.default_rng(2)
    B, K, V = 40, 6, 9
    logits = rng.standard_normal((B, K, V)).astype(np.float32)
    draft = np.argmax(logits, 2).astype(np.int32)
    draft[rng.random((B, K)) < 0.2] = 3
    want = oracle.consensus_commit(logits, draft)
    tokens = np.concatenate([np.full((B, 1), 5, np.int32), draft[:, :-1]], 1)
    got = oracle.tree_consensus_commit(logits, np.tile(np.arange(-1, K - 1), (B, 1)), tokens, K)
    np.testing.assert_array_equal(got["num_committed"], want["num_committed"])
    np.testing.assert_array_equal(got["out_tokens"], want["out_tokens"])
    np.testing.assert_array_equal(got["next_anchor"], want["next_anchor"])
    np.testing.assert_array_equal(got["path_nodes"][:, 0], 0)


def test_hand_worked_walk():
    #        0 -> 1 (tok 4), 2 (tok 7), 3 (tok 7);   2 -> 4 (tok 1);  3 -> 5 (tok 1);  4 -> 6 (tok 0)
    up, tok = np.array([[-1, 0, 0, 0, 2, 3, 4, -1]]), np.array([[9, 4, 7, 7, 1, 1, 0, 7]], np.int32)
    x = np.zeros((1, 8, 10), np.float32)
    x[0, 0, 7] = x[0, 2, 1] = x[0, 4, 0] = 1.0
    x[0, 6, 5] = x[0, 6, 3] = 2.0
    r = oracle.tree_consensus_commit(x, up, tok, 8)
    assert r["path_nodes"].tolist() == [[0, 2, 4, 6, -1, -1, -1, -1]] and r["out_tokens"].tolist() == [[7, 1, 0, 3, -1, -1, -1, -1]]
    assert r["next_anchor"][0] == 3 and r["accept_len"][0] == 3
    assert oracle.tree_consensus_commit(x, up, tok, 2)["path_nodes"][0, :3].tolist() == [0, 2, -1]
    x[0, 2, 6] = np.nan
    assert oracle.tree_consensus_commit(x, up, tok, 8)["out_tokens"][0, :3].tolist() == [7, 6, -1]


def test_hand_worked_rules():
    x = np.array([[[2.0, -2.0, 1.0, 0.0, 3.0, 5.0]] * 2])
    rules = dict(history=np.array([[0, 1, 1, 9, 4]]), history_lens=np.array([4]), prompt_lens=np.array([1]), repetition=np.array([2.0]),
                 presence=np.array([0.5]), frequency=np.array([0.25]))
    out, _ = oracle.process_logits(x, tokens=np.array([[2, 1]]), parents=np.array([[-1, 0]]), **rules)
    # prompt {0}, written 1 twice; row 0 adds 2, row 1 adds 2 and 1
    np.testing.assert_allclose(out[0, 0], [1.0, -4 - .5 - .5, .5 - .25 - .5, 0, 3, 5])
    np.testing.assert_allclose(out[0, 1], [1.0, -4 - .75 - .5, .5 - .25 - .5, 0, 3, 5])
    out, _ = oracle.process_logits(x, bias_starts=np.array([1, 4]), bias_tokens=np.array([5, 3, 7, 3]), bias_values=np.array([9., 1, 1, -7]),
                                   masks=np.array([[0b011101]], np.int32), mask_rows=np.array([[-1, 0]]))
    np.testing.assert_allclose(out[0], [[2, -2, 1, -7, 3, 5], [2, -np.inf, 1, -7, 3, -np.inf]])
    same, size = oracle.process_logits(x, **dict(rules, repetition=np.array([np.nan]), presence=np.array([np.inf]), frequency=np.array([0.0])))
    np.testing.assert_array_equal(same, x)
    assert not size.any()


def test_a_row_of_nothing_ends_the_walk():
    #        0 -> 1 (tok 3) -> 2 (tok 0) -> 3 (tok 0);   row 1 has nothing left
    up, tok = np.array([[-1, 0, 1, 2]]), np.array([[9, 3, 0, 0]], np.int32)
    x = np.zeros((1, 4, 5), np.float32)
    x[0, 0, 3] = 1.0
    r = oracle.tree_consensus_commit(x, up, tok, 4)
    assert r["path_nodes"].tolist() == [[0, 1, 2, 3]] and r["next_anchor"][0] == 0
    x[0, 1] = -np.inf
    r = oracle.tree_consensus_commit(x, up, tok, 4)
    assert r["path_nodes"].tolist() == [[0, 1, -1, -1]] and r["out_tokens"].tolist() == [[3, 0, -1, -1]]
    assert r["next_anchor"][0] == -1 and r["accept_len"][0] == 1 and r["num_committed"][0] == 2
    x[0, 1, 4] = np.finfo(np.float32).min       # the lowest number is a token
    r = oracle.tree_consensus_commit(x, up, tok, 4)
    assert r["out_tokens"].tolist() == [[3, 4, -1, -1]] and r["next_anchor"][0] == 4
    x[0, 1, [2, 3]] = np.nan
    assert oracle.tree_consensus_commit(x, up, tok, 4)["next_anchor"][0] == 2
    x[0, 0] = -np.inf
    r = oracle.tree_consensus_commit(x, up, tok, 4)
    assert r["path_nodes"].tolist() == [[0, -1, -1, -1]] and r["next_anchor"][0] == -1 and r["num_committed"][0] == 1
