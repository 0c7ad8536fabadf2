"""fb_token_attn / fb_token_attn_fp8 against the oracle in 64 bits.

Bounds, element by element.  The softmax weights are rounded to bf16 (relative 2^-8; fp16 for 8-bit pages, 2^-11)
before they multiply V, so an output is off by at most that share of A = sum_j w_j |v_j|, and its own rounding to
bf16 adds 2^-8 of it.  A score is a sum of d <= 128 products in fp32, off by at most d 2^-23 of scale sum |q k|, which
is below 16 here: 2^-12 at most of each weight, and so of A and of the weight sums.  A weight of less than 2^-31 of the
largest may vanish (fp16 ends at 2^-24 and the weights are taken up to 2^7 above 1): 2^-31 |v| for every key."""
import numpy as np
import pytest
import torch

from oracle import flowblock_oracle as O
from paper_2607_17652_b200 import binding as B
from tests import harness as H
from tests.token_harness import Case, bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SENTINEL = 7.0


def call(case, ctx, cache, q, kp, vp, out, ws, status, accumulate=False, stream=None):
    if case.fp8:
        B.fb_token_attn_fp8(ctx, cache, q, kp, vp, *case.dev_scales(), out, ws, status, accumulate, stream)
    else:
        B.fb_token_attn(ctx, cache, q, kp, vp, out, ws, status, accumulate, stream)


def attend(case, accumulate=False, ctx=None, garbage=0xFF):
    """(out, kv_weight, status): the output starts as SENTINEL, the workspace as garbage."""
    ctx = ctx or case.context()
    cache, kp, vp = case.device()
    q = case.q.to(DEV)
    out = torch.full_like(q, SENTINEL)
    ws = B.alloc_token_workspace(ctx, DEV, accumulate).fill_(garbage)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call(case, ctx, cache, q, kp, vp, out, ws, status, accumulate)
    torch.cuda.synchronize()
    return out.cpu(), cache.kv_weight.cpu().numpy(), int(status)


def reference(case, q=None):
    cfg = case.oracle_cfg()
    k, v = case.pools64()
    q = H.f64(case.q) if q is None else q
    out, w = O.token_attn(cfg, case.lens, case.page_table, q, k, v)
    a, _ = O.token_attn(cfg, case.lens, case.page_table, q, k, np.abs(v))
    return out, a, w


def vanishing(case, r=None):
    """What the keys of least weight may lack together, per request."""
    v = np.nan_to_num(case.pools64()[1])
    per = np.array([max(1, n) for n in case.lens]) * 2.0 ** -31 * np.abs(v).max()
    return per[:, None, None] if r is None else per[r]


def check_out(case, got, ref, a):
    eps = 2.0 ** -11 if case.fp8 else 2.0 ** -8
    g = H.f64(got)
    live = case.lens >= 0
    assert (g[~live] == SENTINEL).all()
    err = np.abs(g - ref)[live]
    bound = (eps + 2.0 ** -12) * a[live] * 1.01 + 2.0 ** -8 * np.abs(ref[live]) + vanishing(case)[live]
    assert (err <= bound).all(), (err - bound).max()
    rel = np.linalg.norm(g[live] - ref[live]) / max(np.linalg.norm(ref[live]), 1e-30)
    assert rel <= 5e-3, rel                           # (the norm of the roundings, as for fb_wavefront_attn)


def check_weights(case, got, w):
    want = case.kv_weight.astype(np.float64)
    plain = np.zeros_like(want)
    O.add_weights(case.oracle_cfg(), case.lens, plain, w)
    untouched = np.arange(case.cap) >= case.lens[:, None, None]
    np.testing.assert_array_equal(got[np.broadcast_to(untouched, got.shape)], case.kv_weight[np.broadcast_to(untouched, got.shape)])
    want += plain
    assert (np.abs(got - want) <= 2.0 ** -12 * plain + 2.0 ** -23 * want).all()


LENS = [1, 64, 0, 65, -1, 300, 2, 63, 127, 128, 129, 17]
HEADS = [(4, 1, 64), (8, 8, 64), (128, 2, 64), (16, 4, 128), (32, 32, 128), (16, 2, 128), (16, 1, 128), (64, 2, 128), (128, 1, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
def test_lengths_and_head_layouts(heads, fp8):
    if fp8 and heads[2] == 64:
        pytest.skip("8-bit pages have head_dim 128")
    case = Case(LENS, heads, fp8, seed=1)
    ref, a, w = reference(case)
    got, weight, status = attend(case)
    assert status == 0
    check_out(case, got, ref, a)
    np.testing.assert_array_equal(weight, case.kv_weight)
    got2, weight, status = attend(case, accumulate=True, garbage=0)
    assert status == 0
    check_out(case, got2, ref, a)                     # (short caches in few rows: the two forms add the keys in other orders)
    check_weights(case, weight, w)
    again = [attend(case, accumulate=acc)[0] for acc in (False, True)]
    np.testing.assert_array_equal(bits(again[0]), bits(got))
    np.testing.assert_array_equal(bits(again[1]), bits(got2))


@pytest.mark.parametrize("lens,heads,fp8", [
    ([5000], (8, 2, 128), False), ([20011], (8, 2, 128), False), ([20011, 3], (8, 1, 64), False), ([20011], (8, 2, 128), True),
    ([1], (32, 8, 128), False), ([7, 4000, 0, 1500, 64, -1, 2999], (16, 2, 128), False),
    ([7, 4000, 0, 1500, 64, -1, 2999], (16, 2, 128), True), ([700] * 40, (8, 2, 128), False)])
def test_long_and_ragged_batches(lens, heads, fp8):
    case = Case(lens, heads, fp8, seed=2)
    ref, a, w = reference(case)
    got, weight, status = attend(case, accumulate=True)
    assert status == 0
    check_out(case, got, ref, a)
    check_weights(case, weight, w)


@pytest.mark.parametrize("heads,fp8", [((8, 1, 128), False), ((16, 1, 128), False), ((32, 1, 128), False), ((2, 1, 64), False),
                                       ((8, 1, 128), True), ((16, 1, 128), True)])
def test_one_long_row_in_many_pieces(heads, fp8):
    """A single KV head: its keys are cut into hundreds of pieces, more than the join reads in a turn."""
    case = Case([140001], heads, fp8, seed=140001)
    ref, a, w = reference(case)
    got, weight, status = attend(case, accumulate=True)
    assert status == 0
    check_out(case, got, ref, a)
    check_weights(case, weight, w)
    got, _, status = attend(case)
    assert status == 0
    check_out(case, got, ref, a)


@pytest.mark.parametrize("heads,fp8", [((32, 8, 128), False), ((32, 8, 128), True), ((4, 1, 64), False), ((16, 1, 128), False),
                                       ((32, 32, 128), False), ((16, 1, 128), True)])
@pytest.mark.parametrize("n", [1, 15, 16, 33, 95, 96, 97, 191, 193, 1000, 1536, 1537, 3001, 4031, 4096, 4097])
def test_one_request_around_the_steps_of_a_cluster(heads, fp8, n):
    """Short caches in few rows take a cluster of up to sixteen CTAs each, longer ones (the last) are dealt."""
    case = Case([n], heads, fp8, seed=n)
    ref, a, _ = reference(case)
    got, _, status = attend(case)
    assert status == 0
    check_out(case, got, ref, a)


@pytest.mark.parametrize("heads,fp8,n", [((8, 2, 128), False, 33), ((4, 1, 64), False, 300), ((8, 2, 128), True, 129), ((64, 2, 128), False, 40),
                                         ((16, 1, 128), False, 513)])
def test_many_requests(heads, fp8, n):
    """More requests than the deal looks at at once; some have nothing, some are none, one is long."""
    rng = np.random.default_rng(n)
    lens = rng.integers(-1, 150, n)
    lens[rng.random(n) < 0.2] = 0
    lens[n // 2] = 2000
    case = Case(lens, heads, fp8, seed=22)
    ref, a, w = reference(case)
    for acc in (False, True):
        got, weight, status = attend(case, accumulate=acc)
        assert status == 0
        check_out(case, got, ref, a)
    check_weights(case, weight, w)


def test_few_rows_with_room_to_spare():
    """Capacity far above the lengths, a page that is no page behind them, ragged rows, two calls in a row."""
    case = Case([3, 0, -1, 700, 64, 1], (8, 2, 128), seed=21, pages_per_req=40)
    case.page_table[0, 1:] = -1
    case.page_table[3, 11:] = 1 << 30
    ref, a, _ = reference(case)
    ctx = case.context()
    for _ in range(2):
        got, _, status = attend(case, ctx=ctx)
        assert status == 0
        check_out(case, got, ref, a)


@pytest.mark.parametrize("shape", ["rising", "falling", "dominant", "equal", "far"])
@pytest.mark.parametrize("fp8", [False, True])
def test_scores_that_move_the_reference(shape, fp8):
    """Scores that rise or fall over the whole range along the cache, one key that takes all, equal keys, and
    scores far from 0 on either side."""
    case = Case([1500, 200], (8, 2, 128), fp8, seed=4)
    ks = np.ones(2) if not fp8 else case.scales[0].numpy()
    j = np.arange(case.cap)
    level = {"rising": j * 0.05, "falling": -j * 0.05, "dominant": np.where(j == 777, 60.0, 0.0), "equal": 0.0 * j,
             "far": np.where(j % 2, -300.0, -320.0)}[shape]
    # q = (8, 0, 0, ...): the score of key j is 8 k_j[0] / sqrt(128)
    case.q.zero_()
    case.q[..., 0] = 8.0
    for r in range(case.R):
        for at in range(0, int(case.lens[r])):
            page, row = case.page_table[r, at // 64], at % 64
            for h in range(case.hkv):
                x = level[at] * 128 ** 0.5 / 8.0
                if fp8:
                    case.k_pool[page, h, row, 0] = int(O.e4m3_quantize(np.array([x]), ks[h])[0])
                else:
                    case.k_pool[page, h, row, 0] = x
    ref, a, w = reference(case)
    got, weight, status = attend(case, accumulate=True)
    assert status == 0
    check_out(case, got, ref, a)
    check_weights(case, weight, w)


def test_extreme_queries_keep_their_range_in_8_bits():
    """Rows of q that are tiny, huge or zero: scaled by a power of two each before they become fp16."""
    case = Case([300, 100, 130, 80], (8, 2, 128), True, seed=6)
    case.q[0] *= 2.0 ** -30
    case.q[1] *= 2.0 ** 20
    case.q[1, :, 1:] *= 2.0 ** -30
    case.q[2] = 0
    k, v = case.pools64()
    q = H.f64(case.q)
    cfg = case.oracle_cfg()
    ref, w = O.token_attn(cfg, case.lens, case.page_table, q, k, v)
    a, _ = O.token_attn(cfg, case.lens, case.page_table, q, k, np.abs(v))
    got, _, status = attend(case)
    assert status == 0
    g = H.f64(got)
    for r in range(case.R):
        # An fp32 sum of d products is off by at most d 2^-24 of S = scale sum |q k| (request 1: S is in the
        # thousands), a weight by a factor exp(2 of that) at most, for the score itself and for the sum.
        rows = [np.abs(O.stored_rows(cfg, case.lens, case.page_table, k, r, h)) for h in range(2)]
        s = max(float((rows[n // 4] @ np.abs(q[r, n])).max()) for n in range(8))
        delta = 128 * 2.0 ** -24 * s / np.sqrt(128)
        assert r == 1 or delta < 2.0 ** -13
        bound = (2.0 ** -11 + 2.0 ** -12 + np.expm1(2 * delta)) * 1.01 * a[r] + 2.0 ** -8 * np.abs(ref[r]) + vanishing(case, r)
        assert (np.abs(g - ref)[r] <= bound).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_bad_pages_are_left_out_and_bad_lengths_skipped(fp8):
    case = Case([300, 200, 100, 64], (8, 2, 128), fp8, seed=7)
    good = case.page_table.copy()
    case.page_table[0, 2] = case.num_pages
    case.page_table[1, 0] = -1
    case.page_table[3, 0] = 1 << 30
    case.lens[2] = case.cap + 1
    got, weight, status = attend(case, accumulate=True)
    assert status == B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE
    g = H.f64(got)
    assert (g[2] == SENTINEL).all() and not g[3].any()      # (every key of request 3 is left out)
    np.testing.assert_array_equal(weight[2:], case.kv_weight[2:])
    # the same without the keys of those pages
    k, v = case.pools64()
    for r, gone in ((0, 2), (1, 0)):
        stay = [j for j in range(int(case.lens[r])) if j // 64 != gone]
        for h in range(case.hkv):
            rows = lambda pool: np.stack([pool[good[r, j // 64], h, j % 64] for j in stay])
            for n in range(4 * h, 4 * h + 4):
                z = rows(k) @ H.f64(case.q)[r, n] / np.sqrt(128)
                w = np.exp(z - z.max())
                w /= w.sum()
                err = np.abs(g[r, n] - w @ rows(v))
                assert (err <= 2.0 ** -8 * 1.1 * (w @ np.abs(rows(v)) + np.abs(w @ rows(v)))).all()
            lost = slice(64 * gone, 64 * gone + 64)
            np.testing.assert_array_equal(weight[r, h, lost], case.kv_weight[r, h, lost])


def test_softmax_scale_of_the_context():
    case = Case([200], (8, 2, 128), seed=9)
    ctx = case.context(sm_scale=0.25)
    got, _, _ = attend(case, ctx=ctx)
    k, v = case.pools64()
    cfg = case.oracle_cfg(sm_scale=0.25)
    ref, _ = O.token_attn(cfg, case.lens, case.page_table, H.f64(case.q), k, v)
    a, _ = O.token_attn(cfg, case.lens, case.page_table, H.f64(case.q), k, np.abs(v))
    check_out(case, got, ref, a)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("accumulate", [False, True])
def test_a_captured_call_follows_lengths_pages_and_queries(fp8, accumulate):
    case = Case([300, 900, 64, 0], (16, 4, 128), fp8, seed=10)
    ctx = case.context()
    cache, kp, vp = case.device()
    q, status = case.q.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    out, ws = torch.zeros_like(q), B.alloc_token_workspace(ctx, DEV, True)
    call(case, ctx, cache, q, kp, vp, out, ws, status, accumulate)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(case, ctx, cache, q, kp, vp, out, ws, status, accumulate)
    rng = np.random.default_rng(3)
    for lens in ([300, 900, 64, 0], [1, 65, -1, 899], [0, 0, 0, 0], [120, 1, 500, 2]):
        cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.page_table.copy_(torch.from_numpy(rng.permutation(case.num_pages)[:case.page_table.size].reshape(case.page_table.shape).astype(np.int32)))
        q.copy_(torch.randn(q.shape, generator=case.gen).to(torch.bfloat16))
        # (the poison of the pools is somewhere else in these: fill it)
        for pool in (kp, vp):
            if fp8:
                pool[(pool & 0x7F) == 0x7F] = 0x21
            else:
                pool.nan_to_num_(0.5)
        cache.kv_weight.zero_()
        out.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        o1, w1 = out.clone(), cache.kv_weight.clone()
        cache.kv_weight.zero_()
        out.fill_(SENTINEL)
        call(case, ctx, cache, q, kp, vp, out, ws, status, accumulate)
        torch.cuda.synchronize()
        assert torch.equal(o1, out) and torch.equal(w1, cache.kv_weight)
    assert int(status) == 0


def test_calls_on_two_streams_with_workspaces_of_their_own():
    cases = [Case([3000, 50, 700], (8, 2, 128), seed=11), Case([900, 2500], (16, 2, 128), seed=12)]
    refs = [attend(c, True)[:2] for c in cases]
    torch.cuda.synchronize()
    made = []
    for c in cases:
        ctx = c.context()
        cache, kp, vp = c.device()
        q = c.q.to(DEV)
        made.append((c, ctx, cache, q, kp, vp, torch.zeros_like(q), B.alloc_token_workspace(ctx, DEV, True),
                     torch.zeros(1, dtype=torch.int32, device=DEV)))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for m, s in zip(made, streams):
            with torch.cuda.stream(s):
                m[2].kv_weight.copy_(torch.from_numpy(m[0].kv_weight), non_blocking=True)
            call(*m, accumulate=True, stream=s)
    torch.cuda.synchronize()
    for m, (out, weight) in zip(made, refs):
        np.testing.assert_array_equal(bits(m[6])[m[0].lens >= 0], bits(out)[m[0].lens >= 0])
        np.testing.assert_array_equal(m[2].kv_weight.cpu().numpy(), weight)


@pytest.mark.parametrize("heads,fp8", [((4, 1, 64), False), ((32, 8, 128), False), ((64, 2, 128), False), ((32, 8, 128), True)])
def test_guard_bands(heads, fp8):
    from tests.test_gpu_canary import Guarded
    case = Case([1, 700, 0, 64, 129], heads, fp8, seed=13)
    ctx = case.context()
    g = Guarded()
    cache, kp, vp = case.device()
    cache = B.CacheState(*(g.like(getattr(cache, n)) for n, _ in B.fb_cache._fields_))
    kp, vp, q = g.like(kp), g.like(vp), g.like(case.q)
    out, status = g.like(torch.zeros_like(case.q)), g.like(torch.zeros(1, dtype=torch.int32))
    for acc in (False, True):
        ws = g.like(torch.zeros_like(B.alloc_token_workspace(ctx, "cpu", acc)))
        for _ in range(2):
            call(case, ctx, cache, q, kp, vp, out, ws, status, acc)
    torch.cuda.synchronize()
    assert int(status) == 0
    g.check()


def test_offsets_past_32_bits():
    """Pages at the far end of a pool of 5.2 billion elements, records of 4.3 billion cells."""
    lens, heads, width, pages = [130, 100], (32, 32, 128), 1 << 20, 20000
    small = Case(lens, heads, seed=14)
    ctx = B.Context(**small.cfg(num_pages=pages, max_pages_per_req=width))
    kp, vp = (torch.empty(pages, 32, 64, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.zeros(2, width, dtype=torch.int32, device=DEV)
    for r in range(2):
        for i in range(3):
            to = pages - 1 - (3 * r + i)
            table[r, i] = to
            if i < small.width:
                kp[to], vp[to] = small.k_pool[small.page_table[r, i]].to(DEV), small.v_pool[small.page_table[r, i]].to(DEV)
    weight = torch.zeros(2, 32, width * 64, device=DEV)
    cache = B.CacheState(torch.tensor(lens, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), None,
                         weight, table)
    q = small.q.to(DEV)
    out, status = torch.zeros_like(q), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = B.alloc_token_workspace(ctx, DEV, True)
    B.fb_token_attn(ctx, cache, q, kp, vp, out, ws, status, True)
    torch.cuda.synchronize()
    assert int(status) == 0
    ref, a, w = reference(small)
    check_out(small, out.cpu(), ref, a)
    small.kv_weight[:] = 0
    check_weights(small, weight[..., :small.cap].cpu().numpy(), w)
    assert int(torch.count_nonzero(weight)) == int(torch.count_nonzero(weight[..., :130]))
    # the token's row there too
    k, v = small.k_new.to(DEV), small.v_new.to(DEV)
    B.fb_append_kv(ctx, cache, k, v, kp, vp, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for r, n in enumerate(lens):
        page = int(table[r, (n - 1) // 64])
        assert torch.equal(kp[page, :, (n - 1) % 64], k[r]) and torch.equal(vp[page, :, (n - 1) % 64], v[r])
        assert float(weight[r, :, n - 1].abs().max()) == 0.0
