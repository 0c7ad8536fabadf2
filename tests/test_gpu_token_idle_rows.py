"""Rows without a request (kv_len < 0): whatever their inputs and records hold, nothing of them is written, nothing is
reported, and the other rows' results are the same bits."""
import numpy as np
import pytest
import torch

from paper_2607_17652_b200 import binding as B
from tests.test_gpu_token_evict import aged
from tests.token_harness import Case, bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def step(case, idle, spoiled, accumulate):
    """A step of append, attention and eviction; `spoiled`: the rows in `idle` hold what no request could."""
    ctx = case.context()
    cache, kp, vp = case.device()
    k, v, q = case.k_new.to(DEV), case.v_new.to(DEV), case.q.to(DEV)
    out = torch.full_like(q, 7.0)
    keep = torch.full((case.R,), 50, dtype=torch.int32, device=DEV)
    if spoiled:
        for n, r in enumerate(idle):
            cache.kv_len[r] = (-1, -2 ** 31)[n % 2]
            cache.tok_pos[r] = (2 ** 31 - 1, -2 ** 31)[n % 2]
            cache.page_table[r] = (1 << 30, -7)[n % 2]
            cache.kv_pos[r], cache.kv_weight[r], keep[r] = -1, float("nan"), 0
            for x in (k, v, q):
                x[r] = (float("nan"), float("inf"))[n % 2]
    before = {n: getattr(cache, n)[idle].clone() for n in ("kv_len", "tok_pos", "kv_pos", "kv_weight", "page_table")}
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws, wse = B.alloc_token_workspace(ctx, DEV, accumulate).fill_(0xFF), B.alloc_evict_workspace(ctx, DEV).fill_(0xFF)
    if case.fp8:
        B.fb_append_kv_fp8(ctx, cache, k, v, kp, vp, *case.dev_scales(), status, 10000.0)
        B.fb_token_attn_fp8(ctx, cache, q, kp, vp, *case.dev_scales(), out, ws, status, accumulate)
    else:
        B.fb_append_kv(ctx, cache, k, v, kp, vp, status, 10000.0)
        B.fb_token_attn(ctx, cache, q, kp, vp, out, ws, status, accumulate)
    B.fb_evict_kv(ctx, cache, keep, 8, 2, kp, vp, wse, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for n, x in before.items():
        got = getattr(cache, n)[idle]
        assert torch.equal(got.view(torch.int32), x.view(torch.int32)), n
    assert (out[idle] == 7.0).all()
    live = [r for r in range(case.R) if r not in idle]
    return [bits(x) for x in (kp, vp, out[live])] + [getattr(cache, n)[live].cpu().numpy() for n in ("kv_len", "kv_pos", "kv_weight")]


@pytest.mark.parametrize("heads,fp8", [((8, 2, 128), False), ((16, 1, 128), False), ((8, 2, 128), True)])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n", [6, 40])
def test_what_rows_without_a_request_hold(heads, fp8, accumulate, n):
    lens = np.resize([-1, 300, 65, -1, 64, 130], n)
    idle = [r for r in range(n) if lens[r] < 0]
    plain, spoiled = (step(aged(Case(lens, heads, fp8, seed=51)), idle, s, accumulate) for s in (False, True))
    for x, y in zip(plain, spoiled):
        np.testing.assert_array_equal(x, y)
