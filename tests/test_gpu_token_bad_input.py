"""Page ids outside the pool and lengths above the capacity, in every form that fb_token_attn, fb_append_kv and fb_evict_kv take:
a cluster a row, dealt tiles, the join by lengths (up to 32 requests) and by what the CTAs have cut (more), heads in blocks of 8
and 16.  Reports, outputs over the keys that are left, their weights, and rows that stay as they were.  Bounds as derived
in test_gpu_token_attn.py, with the softmax over the keys that are left."""
import numpy as np
import pytest
import torch

from oracle import flowblock_oracle as O
from paper_2607_17652_b200 import binding as B
from tests import harness as H
from tests.test_gpu_token_attn import SENTINEL, attend, vanishing
from tests.test_gpu_token_evict import aged, evict, expected
from tests.token_harness import Case, bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BAD_IDS = [-1, -2 ** 31, 1 << 30, 2 ** 31 - 1, None]              # None: the number of pages


def spoil(case, rng, share):
    """Replaces page ids below the lengths (`share` of them, and all of the last request that has any); returns the page
    table as it was."""
    good = case.page_table.copy()
    some = [r for r in range(case.R) if case.lens[r] > 0]
    for r in some:
        pages = -(-int(case.lens[r]) // 64)
        hit = np.ones(pages, bool) if r == some[-1] else rng.random(pages) < share
        if r == some[0]:
            hit[0] = True
        for i in np.nonzero(hit)[0]:
            bad = BAD_IDS[rng.integers(len(BAD_IDS))]
            case.page_table[r, i] = case.num_pages if bad is None else bad
    return good


def over_what_is_left(case, good):
    """(out, sum of w |v|, weights added) over the keys of pages that are pages."""
    cfg = case.oracle_cfg()
    k, v = case.pools64()
    q = H.f64(case.q)
    g = case.hq // case.hkv
    out, a = np.zeros(q.shape), np.zeros(q.shape)
    added = np.zeros(case.kv_weight.shape)
    for r in range(case.R):
        if not 0 < case.lens[r] <= case.cap:
            continue
        page = case.page_table[r, np.arange(int(case.lens[r])) // 64]
        left = np.nonzero((page >= 0) & (page < case.num_pages))[0]
        if len(left) == 0:
            continue
        for h in range(case.hkv):
            rows = [x[good[r, left // 64], h, left % 64] for x in (k, v)]
            z = O._scale(cfg) * (q[r, h * g:(h + 1) * g] @ rows[0].T)
            w = np.exp(z - z.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out[r, h * g:(h + 1) * g], a[r, h * g:(h + 1) * g] = w @ rows[1], w @ np.abs(rows[1])
            added[r, h, left] = w.sum(0)
    return out, a, added


def check_attention(case, good, accumulate, want_status):
    lens = case.lens.copy()
    out, a, added = over_what_is_left(case, good)
    got, weight, status = attend(case, accumulate=accumulate)
    assert status == want_status
    g = H.f64(got)
    skipped = (lens < 0) | (lens > case.cap)
    assert (g[skipped] == SENTINEL).all()
    nothing = ~skipped & (a.sum((1, 2)) == 0)
    assert nothing.any() and not g[nothing].any()
    live = ~skipped & ~nothing
    eps = 2.0 ** -11 if case.fp8 else 2.0 ** -8
    case.lens = np.where(skipped, 0, lens).astype(np.int32)
    bound = (eps + 2.0 ** -12) * a * 1.01 + 2.0 ** -8 * np.abs(out) + vanishing(case)
    case.lens = lens
    assert (np.abs(g - out) <= bound)[live].all()
    want = case.kv_weight + (added if accumulate else 0.0)
    np.testing.assert_array_equal(weight[added == 0], case.kv_weight[added == 0])
    assert (np.abs(weight - want) <= 2.0 ** -12 * added + 2.0 ** -23 * want).all()


HEADS = [((8, 2, 128), False), ((8, 2, 128), True), ((16, 1, 128), False), ((16, 1, 128), True), ((32, 1, 128), False), ((4, 1, 64), False)]


@pytest.mark.parametrize("heads,fp8", HEADS)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("room", [None, 70])          # (70 pages: above what a cluster takes, so that the rows are dealt)
def test_few_requests(heads, fp8, accumulate, room):
    case = Case([300, 200, 100, 1, 0, -1, 700, 129], heads, fp8, seed=41, pages_per_req=room)
    good = spoil(case, np.random.default_rng(1), 0.3)
    case.lens[2], case.lens[3] = case.cap + 1, 2 ** 31 - 1
    check_attention(case, good, accumulate, B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE)


@pytest.mark.parametrize("heads,fp8", HEADS)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n", [33, 70, 500])          # (500: more empty and bad rows than the join has CTAs)
def test_many_requests(heads, fp8, accumulate, n):
    rng = np.random.default_rng(n)
    lens = rng.integers(-1, 300, n)
    lens[rng.random(n) < 0.2] = 0
    lens[n // 2], lens[0], lens[-1] = 1500 if n < 100 else 300, 130, 90
    case = Case(lens, heads, fp8, seed=42)
    good = spoil(case, rng, 0.15)
    over = 1 + rng.permutation(n - 2)[:n // 8]
    case.lens[over] = np.where(rng.random(len(over)) < 0.5, case.cap + 1, 2 ** 31 - 1)
    check_attention(case, good, accumulate, B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE)


@pytest.mark.parametrize("bad", ["page", "length"])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("accumulate", [False, True])
def test_each_report_alone(bad, n, accumulate):
    case = Case([100] * n, (8, 2, 128), seed=43)
    if bad == "page":
        case.page_table[n - 1, 1] = case.num_pages
    else:
        case.lens[n - 1] = case.cap + 1
    _, _, status = attend(case, accumulate=accumulate)
    assert status == (B.FB_ST_BAD_PAGE if bad == "page" else B.FB_ST_BAD_STATE)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("base", [0.0, 10000.0])
def test_append_skips_what_has_no_page(fp8, base):
    lens = [1, 64, 65, 200, 0, -1] * 7
    case = Case(lens, (8, 2, 128), fp8, seed=44)
    for r, bad in zip((0, 8, 15, 21), (-1, case.num_pages, 1 << 30, -2 ** 31)):
        case.page_table[r, (max(case.lens[r], 1) - 1) // 64] = bad
    case.lens[6], case.lens[13] = case.cap + 1, 2 ** 31 - 1
    skipped = [0, 8, 15, 21, 6, 13]
    ctx = case.context()
    cache, kp, vp = case.device()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    k, v = case.k_new.to(DEV), case.v_new.to(DEV)
    if fp8:
        B.fb_append_kv_fp8(ctx, cache, k, v, kp, vp, *case.dev_scales(), status, base)
    else:
        B.fb_append_kv(ctx, cache, k, v, kp, vp, status, base)
    torch.cuda.synchronize()
    assert int(status) == B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE
    # the same as a call in which those rows are no requests
    alone = Case(lens, (8, 2, 128), fp8, seed=44)
    alone.lens[skipped] = -1
    cache2, kp2, vp2 = alone.device()
    status.zero_()
    if fp8:
        B.fb_append_kv_fp8(ctx, cache2, k, v, kp2, vp2, *case.dev_scales(), status, base)
    else:
        B.fb_append_kv(ctx, cache2, k, v, kp2, vp2, status, base)
    torch.cuda.synchronize()
    assert int(status) == 0
    for x, y in ((kp, kp2), (vp, vp2)):
        np.testing.assert_array_equal(bits(x), bits(y))
    assert torch.equal(cache.kv_pos, cache2.kv_pos) and torch.equal(cache.kv_weight, cache2.kv_weight)


@pytest.mark.parametrize("fp8", [False, True])
def test_eviction_by_clusters_leaves_such_requests_alone(fp8):
    """Long caches take several CTAs a row, which have to leave together."""
    case = aged(Case([9000, 5000, 40000, 129, 20000], (8, 1, 128), fp8, seed=45))
    keep = [100, 100, 50, 64, 19000]
    want = expected(case, [-1, 100, -1, -1, 19000], 8, 1)
    case.lens[2] = case.cap + 1
    case.page_table[0, 140] = case.num_pages          # (the last page that request 0 has keys on)
    case.page_table[3, 0] = -7
    case.page_table[1, 80] = 1 << 30                  # (behind what request 1 has stored)
    got, kp, vp, status = evict(case, keep, 8, 1)
    assert status == B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE
    got = got.to_numpy()
    np.testing.assert_array_equal(got["kv_len"], [9000, 100, case.cap + 1, 129, 19000])
    np.testing.assert_array_equal(got["kv_pos"], want[1])
    np.testing.assert_array_equal(got["kv_weight"], want[2])
    np.testing.assert_array_equal(bits(kp), want[3][0].numpy())
    np.testing.assert_array_equal(bits(vp), want[3][1].numpy())
