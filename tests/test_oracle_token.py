"""Pins of the oracle's functions for decoding one token at a time (CPU)."""
import numpy as np

from oracle import flowblock_oracle as O


def small(R=3, hq=4, hkv=2, d=8, pages=4, ps=4, seed=0):
    rng = np.random.default_rng(seed)
    cfg = O.Config(max_requests=R, wmax=1, block_len=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=ps,
                   num_pages=R * pages + 1, max_pages_per_req=pages)
    table = rng.permutation(R * pages + 1)[:R * pages].reshape(R, pages)
    shape = (R * pages + 1, hkv, ps, d)
    return cfg, table, rng.normal(size=shape), rng.normal(size=shape), rng


def test_append_is_the_scatter_of_a_window_of_one():
    cfg, table, kp, vp, rng = small()
    lens, pos = np.array([5, 0, 16]), np.array([4, 99, 15])
    k, v = rng.normal(size=(2, 3, 2, 8))
    ka, va, kb, vb = kp.copy(), vp.copy(), kp.copy(), vp.copy()
    rec, wt = np.full((3, 2, 16), -3), np.ones((3, 2, 16))
    for _ in range(2):                              # again is the same as once
        O.append_kv(cfg, lens, pos, table, k, v, ka, va, rec, wt, 100.0)
    st = O.State(np.array([1, 0, 1]), lens - 1, np.zeros(3, int), np.array([1, 0, 1]), np.zeros((3, 1), int),
                 np.zeros((3, 1), np.uint8), table)
    pk = O.pack_wavefronts(cfg, st)
    O.scatter_window_kv(cfg, pk, k[[0, 2]], v[[0, 2]], kb, vb, table, 100.0)
    np.testing.assert_array_equal(ka, kb)
    np.testing.assert_array_equal(va, vb)
    assert rec[0, 1, 4] == 4 and rec[2, 0, 15] == 15 and (rec != -3).sum() == 4 and (wt == 0).sum() == 4


def test_attention_of_a_token_is_a_window_of_one():
    cfg, table, kp, vp, rng = small()
    lens = np.array([5, 1, 16])
    q = rng.normal(size=(3, 4, 8))
    out, w = O.token_attn(cfg, lens, table, q, kp, vp)
    # the newest token in the window tensors, the others as the frozen prefix
    st = O.State(np.ones(3, int), lens - 1, np.zeros(3, int), np.ones(3, int), np.zeros((3, 1), int),
                 np.zeros((3, 1), np.uint8), table)
    pk = O.pack_wavefronts(cfg, st)
    last = lambda pool: np.stack([pool[table[r, (n - 1) // 4], :, (n - 1) % 4] for r, n in enumerate(lens)])
    ref = O.wavefront_attn(cfg, pk, q, last(kp), last(vp), kp, vp, table)
    np.testing.assert_allclose(out, ref, rtol=0, atol=1e-13)
    assert all(np.allclose(x.sum(1), 1) for x in w)
    # closed forms: a zero query gives the mean of the values; nothing stored gives 0
    out, w = O.token_attn(cfg, np.array([6, 0, -1]), table, q * 0, kp, vp)
    np.testing.assert_allclose(out[0, 3], O.stored_rows(cfg, [6], table, vp, 0, 1).mean(0), atol=1e-14)
    assert not out[1:].any() and w[1].shape == (4, 0) and np.allclose(w[0], 1 / 6)


def test_weights_add_up_over_the_heads_of_a_group():
    cfg, table, kp, vp, rng = small()
    lens = np.array([5, 0, 16])
    _, w = O.token_attn(cfg, lens, table, rng.normal(size=(3, 4, 8)), kp, vp)
    acc = np.ones((3, 2, 16))
    O.add_weights(cfg, lens, acc, w)
    np.testing.assert_allclose((acc - 1).sum(-1), [[2, 2], [0, 0], [2, 2]], atol=1e-13)
    assert (acc[0, :, 5:] == 1).all() and (acc[1] == 1).all()


def test_eviction_by_hand():
    cfg, table, kp, vp, _ = small(R=1, hkv=1, hq=1, pages=3)
    kp[:], vp[:] = 0, 0
    for j in range(10):                             # key j holds j, value j holds 100 + j
        kp[table[0, j // 4], 0, j % 4] = j
        vp[table[0, j // 4], 0, j % 4] = 100 + j
    pos = np.arange(12)[None, None] + 0
    wt = np.array([.1, 5, .2, .2, 9, .2, 3, .2, 0, 0, 7, 7])[None, None].copy()
    lens = np.array([10])
    # protected: position 0 (sink), 8 and 9 (last two); then 4, 1, and of 6 by weight 3: six places
    O.evict_kv(cfg, lens, np.array([9]), pos, wt, table, np.array([6]), 2, 1, kp, vp)
    assert lens[0] == 6
    kept = [float(x[0]) for x in O.stored_rows(cfg, lens, table, kp, 0, 0)]
    assert kept == [0, 1, 6, 8, 4, 9]               # holes 2, 3, 5 take 6, 8, 9
    assert list(pos[0, 0, :6]) == [0, 1, 6, 8, 4, 9] and list(wt[0, 0, :6]) == [.1, 5, 3, 0, 9, 0]
    assert list(pos[0, 0, 6:]) == [6, 7, 8, 9, 10, 11] and wt[0, 0, 10] == 7
    # ties go to the lower index; a NaN ranks last
    cfg, table, kp, vp, _ = small(R=1, hkv=1, hq=1, pages=3)
    pos, wt, lens = np.arange(12)[None, None] + 0, np.array([2., 1, 1, np.nan, 1, 0] + [9.] * 6)[None, None].copy(), np.array([6])
    O.evict_kv(cfg, lens, np.array([99]), pos, wt, table, np.array([3]), 0, 0, kp, vp)
    assert list(pos[0, 0, :3]) == [0, 1, 2]
    pos, wt, lens = np.arange(12)[None, None] + 0, np.array([np.nan, 1, 0, 0] + [9.] * 8)[None, None].copy(), np.array([4])
    O.evict_kv(cfg, lens, np.array([99]), pos, wt, table, np.array([3]), 0, 0, kp, vp)
    assert list(pos[0, 0, :3]) == [3, 1, 2]


def test_eviction_keeps_the_heaviest_and_attention_sees_just_them():
    cfg, table, kp, vp, rng = small(R=4, pages=5, seed=4)
    lens0 = np.array([20, 7, 0, 13])
    keep = np.array([6, 9, 3, -1])
    lens, pos = lens0.copy(), rng.integers(0, 50, (4, 2, 20))
    wt = rng.random((4, 2, 20))
    newest = np.array([49, 49, 49, 49])
    q = rng.normal(size=(4, 4, 8))
    k0, v0, p0, w0 = kp.copy(), vp.copy(), pos.copy(), wt.copy()
    O.evict_kv(cfg, lens, newest, pos, wt, table, keep, 5, 3, kp, vp)
    assert list(lens) == [6, 7, 0, 13]
    out, _ = O.token_attn(cfg, lens, table, q, kp, vp)
    for h in range(2):
        safe = (p0[0, h] < 3) | (p0[0, h] > 44)
        order = (list(np.flatnonzero(safe)) + [j for j in np.argsort(-w0[0, h], kind="stable") if not safe[j]])[:6]
        rows = lambda pool: O.stored_rows(cfg, lens0, table, pool, 0, h)[order]
        have = O.stored_rows(cfg, lens, table, kp, 0, h)
        np.testing.assert_array_equal(np.sort(have[:, 0]), np.sort(rows(k0)[:, 0]))
        assert sorted(zip(pos[0, h, :6], wt[0, h, :6])) == sorted((p0[0, h, j], w0[0, h, j]) for j in order)
        for g in (2 * h, 2 * h + 1):
            z = rows(k0) @ q[0, g] / np.sqrt(8)
            w = np.exp(z) / np.exp(z).sum()
            np.testing.assert_allclose(out[0, g], w @ rows(v0), atol=1e-13)
    np.testing.assert_array_equal(pos[1:], p0[1:])
