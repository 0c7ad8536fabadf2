"""fb_append_kv / fb_append_kv_fp8 against the oracle: the row that is written, the records, and everything else bit
for bit as it was."""
import numpy as np
import pytest
import torch

from oracle import flowblock_oracle as O
from paper_2607_17652_b200 import binding as B
from tests import harness as H
from tests.token_harness import Case, bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BASE = 10000.0


def _append(case, ctx, cache, kp, vp, status, base):
    k, v = case.k_new.to(DEV), case.v_new.to(DEV)
    if case.fp8:
        B.fb_append_kv_fp8(ctx, cache, k, v, kp, vp, *case.dev_scales(), status, base)
    else:
        B.fb_append_kv(ctx, cache, k, v, kp, vp, status, base)


CASES = [
    ([1], (4, 1, 64), False), ([64], (4, 1, 64), False), ([65, 0, -1, 200, 1], (8, 2, 64), False),
    ([300, 1, 128, 0, 63, 64, 65], (8, 2, 128), False), ([17] * 9, (32, 32, 128), False), ([99, 2], (128, 1, 128), False),
    ([300, 1, 128, 0, -5, 64, 65], (8, 2, 128), True), ([5, 77], (32, 32, 128), True),
]


@pytest.mark.parametrize("lens,heads,fp8", CASES)
@pytest.mark.parametrize("base", [0.0, BASE])
def test_the_row_the_records_and_nothing_else(lens, heads, fp8, base):
    case = Case(lens, heads, fp8, seed=3)
    # lengths without the token first: every other byte of the pools is finite or NaN, and stays
    ctx = case.context()
    cache, kp, vp = case.device()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for _ in range(2):                                # again is the same as once
        _append(case, ctx, cache, kp, vp, status, base)
    torch.cuda.synchronize()
    assert int(status) == 0
    ref = [H.f64(p) if not fp8 else p.numpy().copy() for p in (case.k_pool, case.v_pool)]
    pos, weight = case.kv_pos.copy(), case.kv_weight.copy()
    O.append_kv(case.oracle_cfg(), case.lens, case.tok_pos, case.page_table, H.f64(case.k_new), H.f64(case.v_new), *ref,
                pos, weight, base, case.scales)
    got = cache.to_numpy()
    np.testing.assert_array_equal(got["kv_pos"], pos)
    np.testing.assert_array_equal(got["kv_weight"], weight)
    np.testing.assert_array_equal(got["kv_len"], case.lens)
    written = np.zeros(kp.shape[:3], bool)
    for r, n in enumerate(case.lens):
        if n > 0:
            written[case.page_table[r, (n - 1) // 64], :, (n - 1) % 64] = True
    for have, was, want in ((kp, case.k_pool, ref[0]), (vp, case.v_pool, ref[1])):
        np.testing.assert_array_equal(bits(have)[~written], bits(was)[~written])
        rotated = base > 0 and have is kp
        if fp8:
            a, b = bits(have)[written].astype(int), want[written].astype(int)
            if not rotated:
                np.testing.assert_array_equal(a, b)
            else:
                # fp32 against fp64 rotation: a value within rounding distance of a tie may fall on the next code
                # (codes of one sign count upwards with the magnitude)
                va, vb = O.e4m3_decode(a.astype(np.uint8)), O.e4m3_decode(b.astype(np.uint8))
                off = a != b
                assert off.mean() < 0.01
                step = np.maximum(np.abs(va), np.abs(vb))[off] * 2.0 ** -3
                assert (np.abs(va - vb)[off] <= np.maximum(step, 2.0 ** -9)).all()
        else:
            a, b = H.f64(have.cpu())[written], want[written]
            if not rotated:
                np.testing.assert_array_equal(a, b)
            else:
                # bf16 rounds by at most 2^-8 of the value; fp32: two products and a sum of |x| <= 5 or so, a
                # reduced angle and its sine and cosine, each 2^-23 or less: under 2^-18
                assert (np.abs(a - b) <= 2.0 ** -8 * np.abs(b) + 2.0 ** -18).all()


def test_same_bytes_as_the_scatter_of_a_block():
    """A block scattered at once and the same rows appended one by one give the same pages bit for bit."""
    lens, heads = [70 + 32, 3 + 32], (16, 4, 128)
    for fp8 in (False, True):
        case = Case(lens, heads, fp8, seed=8, fill=False)
        bl = 32
        over = dict(wmax=1, block_len=bl, window_in_pages=1, max_blocks=1, kv_fp8=int(fp8))
        ctx = B.Context(**case.cfg(**over))
        prefix = case.lens - bl
        R = case.R
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        st = B.DeviceState(z(R) + 1, torch.from_numpy(prefix).to(DEV), z(R), z(R) + 1, z(R, bl), torch.zeros(R, 1, dtype=torch.uint8, device=DEV),
                           torch.from_numpy(case.page_table).to(DEV))
        pk = B.PackBuffers.alloc(ctx, DEV)
        sb = B.StepBuffers(ctx, DEV)
        k, v = (torch.randn(R, bl, case.hkv, case.d, generator=case.gen).to(torch.bfloat16).to(DEV) for _ in range(2))
        cache, ka, va = case.device()
        kb, vb = ka.clone(), va.clone()
        B.fb_pack_wavefronts(ctx, st, pk, sb.ws, sb.status)
        flat = lambda x: x.reshape(R * bl, case.hkv, case.d).contiguous()
        args = (flat(k), flat(v), ka, va)
        if fp8:
            B.fb_scatter_window_kv_fp8(ctx, pk, st.page_table, *args, *case.dev_scales(), sb.status, rope_base=BASE)
        else:
            B.fb_scatter_window_kv(ctx, pk, st.page_table, *args, sb.status, rope_base=BASE)
        for t in range(bl):
            cache.kv_len.copy_(torch.from_numpy(prefix + t + 1))
            cache.tok_pos.copy_(cache.kv_len - 1)
            kt, vt = k[:, t].contiguous(), v[:, t].contiguous()
            if fp8:
                B.fb_append_kv_fp8(ctx, cache, kt, vt, kb, vb, *case.dev_scales(), sb.status, BASE)
            else:
                B.fb_append_kv(ctx, cache, kt, vt, kb, vb, sb.status, BASE)
        torch.cuda.synchronize()
        assert int(sb.status) == 0
        np.testing.assert_array_equal(bits(ka), bits(kb))
        np.testing.assert_array_equal(bits(va), bits(vb))


@pytest.mark.parametrize("fp8", [False, True])
def test_bad_pages_and_lengths_are_reported_and_skipped(fp8):
    case = Case([10, 130, 64, 20], (8, 2, 128), fp8, seed=5)
    ctx = case.context()
    cache, kp, vp = case.device()
    cache.page_table[1, 2] = case.num_pages           # the page of request 1's token
    cache.page_table[2, 0] = -1
    cache.kv_len[3] = case.cap + 1
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    _append(case, ctx, cache, kp, vp, status, BASE)
    torch.cuda.synchronize()
    assert int(status) == B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE
    got = cache.to_numpy()
    for r in (1, 2, 3):
        np.testing.assert_array_equal(got["kv_pos"][r], case.kv_pos[r])
        np.testing.assert_array_equal(got["kv_weight"][r], case.kv_weight[r])
    changed = (bits(kp) != bits(case.k_pool)).any((1, 3))
    assert set(map(tuple, np.argwhere(changed))) == {(case.page_table[0, 0], 9)}


def test_without_records():
    case = Case([10, 64], (8, 2, 128), seed=6)
    ctx = case.context()
    cache, kp, vp = case.device(records=False)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    _append(case, ctx, cache, kp, vp, status, 0.0)
    torch.cuda.synchronize()
    assert int(status) == 0
    np.testing.assert_array_equal(bits(kp[int(case.page_table[1, 0]), :, 63]), bits(case.k_new[1]))
