"""The tree operators together, as a serving loop uses them: cycles that map their pages, attend a tree of drafts in every layer, put its
logits through every request's rules and commit the greedy path, eager and as a replayed graph, each against the oracle; and the same
rules in front of drawing and of the filtered consensus."""
import numpy as np
import pytest
import torch

import oracle
from orthrus_inputs import bf16_bits_to_f32

pytestmark = pytest.mark.gpu

LAYERS, CYCLES, B, K, N, DEPTH, V, P, H, HQ, D, WIDTH = 2, 5, 6, 4, 40, 7, 3001, 16, 2, 8, 128, 12
U = 2.0 ** -8   # half a step of bf16


def _rt():
    from paper_2605_12825_amd import runtime
    return runtime


def _bits(rng, *shape):
    return (rng.standard_normal(shape).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _state(seed):
    rng = np.random.default_rng(seed)
    lens = np.array([0, 5, 37, 90, 64, 128], np.int32)
    pages = 70
    perm = rng.permutation(pages).astype(np.int32)
    table, at = np.full((B, WIDTH), -1, np.int32), 0
    for b in range(B):
        n = (lens[b] + P - 1) // P
        table[b, :n] = perm[at:at + n]
        at += n
    ring = np.full(pages, -1, np.int32)
    ring[(61 + np.arange(pages - at)) % pages] = perm[at:]
    history = np.zeros((B, 400), np.int32)
    history[:, :200] = rng.integers(0, 60, (B, 200))
    return dict(lens=lens, table=table, ring=ring, state=np.array([61, pages - at], np.int32), kp=_bits(rng, LAYERS, pages, H, P, D),
                vp=_bits(rng, LAYERS, pages, H, P, D), history=history, history_lens=np.array([0, 3, 40, 90, 64, 150], np.int32))


def _rules(rng, history, history_lens):
    """Of six requests: none, penalties, penalties and biases, a grammar for every node, one that allows nothing at some nodes, all."""
    masks = rng.integers(-2 ** 31, 2 ** 31, (N + 1, (V + 31) // 32)).astype(np.int32)
    masks[N] = 0
    rows = np.full((B, N), -1, np.int32)
    rows[3], rows[5] = np.arange(N), np.arange(N)[::-1]
    rows[4, ::3] = N
    return dict(history=history, history_lens=history_lens, prompt_lens=np.array([0, 2, 20, 50, 64, 100], np.int32),
                repetition=np.array([1, 1.2, 1.1, 1, 1, 0.9], np.float32), presence=np.array([0, 0.5, 0, 0, 0, 0.3], np.float32),
                frequency=np.array([0, 0.2, 0.1, 0, 0, 0.2], np.float32), bias_starts=np.array([0, 0, 0, 30, 30, 30, 40], np.int32),
                bias_tokens=rng.integers(0, V, 40).astype(np.int32), bias_values=(rng.standard_normal(40) * 4).astype(np.float32),
                masks=masks, mask_rows=rows)


def _inputs(c):
    rng = np.random.default_rng(200 + c)
    x = dict(q_diff=_bits(rng, LAYERS, B, K, HQ, D), q_ar=_bits(rng, LAYERS, B, N, HQ, D))
    for n, rows in (("k_blk_diff", K), ("v_blk_diff", K), ("k_blk_ar", N), ("v_blk_ar", N)):
        x[n] = _bits(rng, LAYERS, B, rows, H, D)
    parents, tokens = np.full((B, N), -1, np.int32), rng.integers(0, V, (B, N)).astype(np.int32)
    logits = rng.standard_normal((B, N, V)).astype(np.float32)
    for b in range(B):
        level = [0]
        for i in range(1, N - 5 * (b % 2)):
            k = int(rng.integers(max(0, i - 4), i))
            k = k if level[k] + 1 < DEPTH else 0
            parents[b, i] = k
            level.append(level[k] + 1)
        node = 0
        for _ in range(int(rng.integers(0, DEPTH))):    # a path that the logits ask for, before the rules
            below = np.flatnonzero(parents[b] == node)
            if not below.size:
                break
            child = int(rng.choice(below))
            logits[b, node, tokens[b, child]] = 11
            node = child
    return dict(x, parents=parents, node_tokens=tokens, ar_logits=logits)


def _close(got_bits, want, size):
    off = np.abs(bf16_bits_to_f32(got_bits).astype(np.float64) - want) - (1.06 * U * size + 1.01 * U * np.abs(want) + 1e-6)
    assert off.max() <= 0


def test_cycles_of_trees_under_rules_eager_and_replayed():
    rt = _rt()
    st, d = _state(1), _rt().to_device_bits
    rules = _rules(np.random.default_rng(3), st["history"], st["history_lens"])
    ref = {k: v.copy() for k, v in st.items()}
    stacks = []
    for _ in range(2):
        dev_rules = {k: d(v.copy()) for k, v in rules.items()}
        s = rt.DecodeStack(num_layers=LAYERS, batch=B, num_q_heads=HQ, num_kv_heads=H, head_dim=D, block_k=K, page_size=P, k_pool=d(st["kp"]),
                           v_pool=d(st["vp"]), page_table=d(st["table"]), seq_lens=d(st["lens"]), max_seq_len=WIDTH * P, vocab=V,
                           free_pages=d(st["ring"]), free_state=d(st["state"]), tree_nodes=N, tree_depth=DEPTH, rules=rt.LogitRules(**dev_rules))
        stacks.append((s, dev_rules))
    stacks[1][0].capture()
    committed = []
    for c in range(CYCLES):
        x = _inputs(c)
        slots = np.full(B * DEPTH, -9, np.int32)
        granted, _, status = oracle.page_tables_update(ref["lens"], np.full(B, DEPTH, np.int32), ref["table"], ref["ring"], ref["state"], P,
                                                       WIDTH * P, B * DEPTH, slots)
        assert status == 0 and (granted == DEPTH).all()
        want_d = [oracle.dual_view_attn(0, 1 / np.sqrt(D), x["q_diff"][l], x["k_blk_diff"][l], x["v_blk_diff"][l], ref["kp"][l], ref["vp"][l],
                                        ref["table"], ref["lens"]) for l in range(LAYERS)]
        want_a = [oracle.tree_attn(1 / np.sqrt(D), x["parents"], *[bf16_bits_to_f32(v) for v in (x["q_ar"][l], x["k_blk_ar"][l], x["v_blk_ar"][l],
                                   ref["kp"][l], ref["vp"][l])], ref["table"], ref["lens"]) for l in range(LAYERS)]
        now = dict(rules, history=ref["history"], history_lens=ref["history_lens"])
        logits, _ = oracle.process_logits(x["ar_logits"], x["node_tokens"], x["parents"], **now)
        # what the roundings could turn about (four of 2^-24, of values below 32) is not decided here: the two largest logits lie apart
        two = np.partition(logits, V - 2, axis=2)[..., V - 2:]
        assert np.all(np.isneginf(two[..., 0]) | (two[..., 1] > two[..., 0] + 8e-6))
        want = oracle.tree_consensus_commit(logits, x["parents"], x["node_tokens"], DEPTH, x["k_blk_ar"], x["v_blk_ar"], ref["kp"], ref["vp"],
                                            ref["table"], ref["lens"])
        assert want["status"] == 0
        committed.append(want["num_committed"])
        for (s, dev_rules), run in zip(stacks, (stacks[0][0].cycle, stacks[1][0].replay)):
            for k, v in x.items():
                getattr(s, k).copy_(d(v))
            dev_rules["history"].copy_(d(ref["history"]))
            dev_rules["history_lens"].copy_(d(ref["history_lens"]))
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            assert s.step.device_error() == 0
            for l in range(LAYERS):
                _close(rt.bits_to_numpy(s.out_ar[l]), want_a[l][0], want_a[l][1])
                assert np.abs(bf16_bits_to_f32(rt.bits_to_numpy(s.out_diff[l])).astype(np.float64) - want_d[l]).max() <= 2e-2
            for k in ("accept_len", "num_committed", "path_nodes", "out_tokens", "next_anchor"):
                np.testing.assert_array_equal(getattr(s, k).cpu().numpy(), want[k], err_msg=k)
            for k, v in (("k_pool", ref["kp"]), ("v_pool", ref["vp"]), ("seq_lens", ref["lens"]), ("page_table", ref["table"]), ("free_pages", ref["ring"]),
                         ("free_state", ref["state"])):
                np.testing.assert_array_equal(rt.bits_to_numpy(getattr(s, k)), v, err_msg=k)
        for b in range(B):   # the program extends the texts by what has been fed on the path
            m, n = int(want["num_committed"][b]), int(ref["history_lens"][b])
            ref["history"][b, n:n + m] = x["node_tokens"][b, want["path_nodes"][b, :m]]
            ref["history_lens"][b] = n + m
    assert np.max(committed) > 2 and np.min(committed) == 1
    for s, _ in stacks:
        s.close()


def test_a_chain_as_a_tree_is_the_plain_cycle():
    """The same block through both stacks: attention within the path's tolerance of one another, the same tokens, caches and lengths."""
    rt, d = _rt(), _rt().to_device_bits
    st = _state(5)
    rng = np.random.default_rng(6)
    common = dict(num_layers=LAYERS, batch=B, num_q_heads=HQ, num_kv_heads=H, head_dim=D, block_k=K, page_size=P, max_seq_len=WIDTH * P, vocab=V)
    for b in range(B):   # pages for the block
        n = (st["lens"][b] + P - 1) // P
        st["table"][b, n] = 69 - b
    make = lambda **kw: rt.DecodeStack(k_pool=d(st["kp"]), v_pool=d(st["vp"]), page_table=d(st["table"]), seq_lens=d(st["lens"]), **common, **kw)  # noqa: E731
    plain, tree = make(), make(tree_nodes=K)
    x = {k: _bits(rng, LAYERS, B, K, h, D) for k, h in (("q_ar", HQ), ("k_blk_ar", H), ("v_blk_ar", H))}
    logits = rng.standard_normal((B, K, V)).astype(np.float32)
    draft = np.argmax(logits, 2).astype(np.int32)
    draft[[1, 3], [0, 2]] += 1
    for s in (plain, tree):
        for k, v in x.items():
            getattr(s, k).copy_(d(v))
        s.ar_logits.copy_(torch.from_numpy(logits))
    plain.draft_tokens.copy_(torch.from_numpy(draft))
    tree.node_tokens.copy_(torch.from_numpy(np.concatenate([np.full((B, 1), 9, np.int32), draft[:, :-1]], 1)))
    plain.cycle()
    tree.cycle()
    torch.cuda.synchronize()
    for k in ("num_committed", "out_tokens", "next_anchor", "seq_lens", "k_pool", "v_pool"):
        assert torch.equal(getattr(plain, k), getattr(tree, k)), k
    diff = bf16_bits_to_f32(rt.bits_to_numpy(plain.out_ar)) - bf16_bits_to_f32(rt.bits_to_numpy(tree.out_ar))
    assert np.abs(diff).max() <= 4 * U * 4     # two roundings on either side, of values below four
    plain.close()
    tree.close()


def test_rules_in_front_of_drawing_and_of_the_filtered_consensus():
    rt = _rt()
    rng = np.random.default_rng(8)
    x = rng.standard_normal((B, K, V)).astype(np.float32) * 3
    rules = _rules(rng, np.random.default_rng(9).integers(0, V, (B, 300)).astype(np.int32), np.array([0, 3, 40, 90, 64, 150], np.int32))
    rules["mask_rows"] = np.ascontiguousarray(rules["mask_rows"][:, :K])
    fed = rng.integers(0, V, (B, K)).astype(np.int32)
    step = rt.DecodeStep(batch=B, num_q_heads=2, num_kv_heads=2, head_dim=64, block_k=K, page_size=16, max_pages_per_seq=1, max_seq_len=0, num_pages=1,
                         vocab=V)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    logits, r = dev(x), rt.LogitRules(**{k: dev(v) for k, v in rules.items()})
    step.process_logits(logits, r, dev(fed))
    y = logits.cpu().numpy()
    want, _ = oracle.process_logits(x, fed, None, **rules)
    np.testing.assert_allclose(np.where(np.isneginf(want), 0, y), np.where(np.isneginf(want), 0, want), rtol=2e-6, atol=2e-6)
    f = (np.array([0.8, 1, 0.7, 0, 1, 1.2], np.float32), np.array([0, 20, 0, 0, 5, 0], np.int32), np.array([0.95, 1, 0.9, 1, 1, 0.98], np.float32),
         np.array([0, 0, 0.02, 0, 0, 0], np.float32))
    u = rng.random((B, K), dtype=np.float32)
    tokens, lp = torch.zeros((B, K), dtype=torch.int32, device="cuda"), torch.zeros((B, K), device="cuda")
    step.sample_tokens(logits, *[dev(v) for v in f], dev(u), tokens, lp)
    got = tokens.cpu().numpy()
    t, _, margin = oracle.sample_tokens(y, *f, u)
    assert margin.min() > 1e-9
    np.testing.assert_array_equal(got, t)
    for b in range(B):
        for k in range(K):
            assert (got[b, k] == -1) == bool(np.isneginf(want[b, k]).all()) and (got[b, k] < 0 or np.isfinite(want[b, k, got[b, k]]))
    assert (got == -1).sum() == 2     # request 4's rows 0 and 3, which no token is allowed for
    diff = (y + 0.3 * rng.standard_normal(y.shape)).astype(np.float32)
    gumbel, accept = rng.gumbel(size=(B, V)).astype(np.float32), rng.random((B, K), dtype=np.float32)
    drafts, _, _ = oracle.sample_tokens(diff, *f, u)
    o = {n: torch.zeros(B, dtype=torch.int32, device="cuda") for n in ("accept_len", "num_committed", "next_anchor")}
    out = torch.zeros((B, K), dtype=torch.int32, device="cuda")
    step.filtered_consensus_commit(logits, dev(diff), *[dev(v) for v in f], dev(drafts), dev(accept), dev(gumbel), None, None, None, None, None, None,
                                   o["accept_len"], o["num_committed"], out, o["next_anchor"])
    w = oracle.filtered_consensus_commit(y, diff, *f, drafts, accept, gumbel)
    assert w["margin"] > 1e-8
    np.testing.assert_array_equal(out.cpu().numpy(), w["out_tokens"])
    for k, v in o.items():
        np.testing.assert_array_equal(v.cpu().numpy(), w[k])
    step.close()
