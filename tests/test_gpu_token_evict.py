"""fb_evict_kv against the oracle, everything bit for bit: which keys stay, where they go, records, lengths, and all
that does not move.  And the calls that decode one token at a time together, step by step."""
import numpy as np
import pytest
import torch

from oracle import flowblock_oracle as O
from paper_2607_17652_b200 import binding as B
from tests import harness as H
from tests.token_harness import Case, bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def evict(case, keep, recent, sinks, ctx=None, cache=None):
    """(cache, k_pool, v_pool, status) after the call on the case's state."""
    ctx = ctx or case.context()
    cache, kp, vp = case.device() if cache is None else cache
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = B.alloc_evict_workspace(ctx, DEV).fill_(0xFF)
    B.fb_evict_kv(ctx, cache, torch.tensor(keep, dtype=torch.int32, device=DEV), recent, sinks, kp, vp, ws, status)
    torch.cuda.synchronize()
    return cache, kp, vp, int(status)


def expected(case, keep, recent, sinks):
    pools = [torch.from_numpy(bits(p).copy()) for p in (case.k_pool, case.v_pool)]
    pos, weight, lens = case.kv_pos.copy(), case.kv_weight.copy(), case.lens.copy()
    O.evict_kv(case.oracle_cfg(), lens, case.tok_pos, pos, weight, case.page_table, keep, recent, sinks, *(p.numpy() for p in pools))
    return lens, pos, weight, pools


def check(case, keep, recent, sinks):
    want = expected(case, keep, recent, sinks)
    cache, kp, vp, status = evict(case, keep, recent, sinks)
    assert status == 0
    got = cache.to_numpy()
    np.testing.assert_array_equal(got["kv_len"], want[0])
    np.testing.assert_array_equal(got["kv_pos"], want[1])
    np.testing.assert_array_equal(got["kv_weight"].view(np.int32), want[2].view(np.int32))
    np.testing.assert_array_equal(bits(kp), want[3][0].numpy())
    np.testing.assert_array_equal(bits(vp), want[3][1].numpy())


def aged(case, seed=0):
    """Positions as a request has them: increasing, some gone already, the older half mixed."""
    rng = np.random.default_rng(seed)
    for r in range(case.R):
        n = max(0, int(case.lens[r]))
        for h in range(case.hkv):
            pos = np.sort(rng.permutation(int(1.3 * n) + 1)[:n])
            pos[:n // 2] = rng.permutation(pos[:n // 2])
            case.kv_pos[r, h, :n] = pos
        case.tok_pos[r] = case.kv_pos[r, :, :n].max() if n else 0
    return case


@pytest.mark.parametrize("heads,fp8", [((4, 1, 64), False), ((8, 8, 64), False), ((8, 2, 128), False), ((32, 8, 128), True)])
@pytest.mark.parametrize("recent,sinks", [(0, 0), (16, 4)])
def test_lengths_and_bounds(heads, fp8, recent, sinks):
    lens = [1, 2, 64, 65, 0, -1, 200, 200, 200, 200, 129, 128, 300, 300]
    keep = [0, 1, 63, 64, 5, 3, 1, 199, 200, 201, -1, 0, 100, 17]
    check(aged(Case(lens, heads, fp8, seed=1)), keep, recent, sinks)


@pytest.mark.parametrize("lens,keep,heads,fp8", [
    ([5000], [1234], (8, 2, 128), False), ([8192, 8191, 8193], [4000, 8190, 2], (4, 1, 64), False),      # a CTA's registers, and past them
    ([30000, 17], [29936, 3], (8, 2, 128), False), ([30000], [900], (8, 2, 128), True), ([70001, 65536], [3000, 65535], (4, 1, 64), False),
    ([2112] * 20, [2048] * 20, (16, 4, 128), False)])
def test_long_caches(lens, keep, heads, fp8):
    check(aged(Case(lens, heads, fp8, seed=2)), keep, 128, 4)


WEIGHTS = {
    "equal": lambda rng, s: np.ones(s), "zero": lambda rng, s: np.zeros(s), "few values": lambda rng, s: rng.integers(0, 4, s) * 0.25,
    "signed zeros": lambda rng, s: np.where(rng.random(s) < 0.5, -0.0, 0.0),
    "with nan and inf": lambda rng, s: rng.choice([np.nan, np.inf, -np.inf, 0.0, 1.0, -1.0, 3e38, 1e-45], s),
    "negative": lambda rng, s: -np.exp(rng.normal(size=s)), "one bit apart": lambda rng, s: (1.0 + rng.integers(0, 3, s) * 2.0 ** -23),
    "wide": lambda rng, s: np.exp(rng.normal(size=s) * 20), "nan alone": lambda rng, s: np.full(s, np.nan),
}


@pytest.mark.parametrize("kind", list(WEIGHTS))
def test_ties_and_weights_that_are_no_numbers(kind):
    case = aged(Case([700, 9000, 64, 300], (4, 2, 64), seed=3))
    with np.errstate(all="ignore"):
        case.kv_weight = WEIGHTS[kind](case.rng, case.kv_weight.shape).astype(np.float32)
    check(case, [350, 4000, 1, 299], 10, 2)


@pytest.mark.parametrize("recent,sinks", [(2 ** 31 - 1, 0), (0, 2 ** 31 - 1), (400, 0), (0, 400), (399, 1)])
def test_more_protected_than_kept(recent, sinks):
    """Then storage order decides among them."""
    case = aged(Case([500, 9000], (4, 2, 64), seed=4))
    check(case, [100, 400], recent, sinks)


def test_positions_at_the_ends_of_the_range():
    case = Case([300], (4, 2, 64), seed=5)
    case.kv_pos[:] = case.rng.choice([-2 ** 31, -1, 0, 1, 2 ** 31 - 1], case.kv_pos.shape)
    for tok in (-2 ** 31, 0, 2 ** 31 - 1):
        case.tok_pos[:] = tok
        check(case, [77], 2 ** 31 - 1, 1)


@pytest.mark.parametrize("fp8", [False, True])
def test_bad_pages_and_lengths_leave_the_request_alone(fp8):
    case = aged(Case([300, 200, 100, 129], (8, 2, 128), fp8, seed=6))
    keep = [100, 100, 50, 64]
    want = expected(case, [-1, 100, -1, -1], 8, 1)
    case.lens[2] = case.cap + 1
    cache = case.device()
    cache[0].page_table[0, 4] = case.num_pages
    cache[0].page_table[3, 0] = -7
    cache[0].page_table[1, 4] = 1 << 30               # (behind what request 1 has stored)
    got, kp, vp, status = evict(case, keep, 8, 1, cache=cache)
    assert status == B.FB_ST_BAD_PAGE | B.FB_ST_BAD_STATE
    got = got.to_numpy()
    np.testing.assert_array_equal(got["kv_len"], [300, 100, case.cap + 1, 129])
    np.testing.assert_array_equal(got["kv_pos"], want[1])
    np.testing.assert_array_equal(got["kv_weight"], want[2])
    np.testing.assert_array_equal(bits(kp), want[3][0].numpy())
    np.testing.assert_array_equal(bits(vp), want[3][1].numpy())


def test_again_is_nothing_and_a_captured_call_follows_the_bounds():
    case = aged(Case([900, 300, 64, 9000], (8, 2, 128), seed=7))
    ctx = case.context()
    cache, kp, vp = case.device()
    start = [x.clone() for x in (cache.kv_len, cache.kv_pos, cache.kv_weight, kp, vp)]
    keep, status = torch.full((4,), 1 << 20, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = B.alloc_evict_workspace(ctx, DEV)
    call = lambda: B.fb_evict_kv(ctx, cache, keep, 20, 2, kp, vp, ws, status)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for bound in ([500, 300, 10, 8000], [100, 299, -1, 64], [0, 0, 0, 0]):
        for x, y in zip((cache.kv_len, cache.kv_pos, cache.kv_weight, kp, vp), start):
            x.copy_(y)
        keep.copy_(torch.tensor(bound, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = expected(case, bound, 20, 2)
        after = [x.clone() for x in (cache.kv_len, cache.kv_pos, cache.kv_weight, kp, vp)]
        np.testing.assert_array_equal(after[0].cpu().numpy(), want[0])
        np.testing.assert_array_equal(after[1].cpu().numpy(), want[1])
        np.testing.assert_array_equal(bits(kp), want[3][0].numpy())
        graph.replay()                                # nothing is above its bound any more
        torch.cuda.synchronize()
        for x, y in zip((cache.kv_len, cache.kv_pos, cache.kv_weight), after):
            assert torch.equal(x, y)
        np.testing.assert_array_equal(bits(vp), want[3][1].numpy())
    assert int(status) == 0


@pytest.mark.parametrize("heads,fp8", [((4, 1, 64), False), ((32, 8, 128), True), ((8, 2, 128), False)])
def test_guard_bands(heads, fp8):
    from tests.test_gpu_canary import Guarded
    case = aged(Case([1, 700, 0, 64, 9000], heads, fp8, seed=8))
    ctx = case.context()
    g = Guarded()
    cache, kp, vp = case.device()
    cache = B.CacheState(*(g.like(getattr(cache, n)) for n, _ in B.fb_cache._fields_))
    kp, vp, keep = g.like(kp), g.like(vp), g.like(torch.tensor([1, 350, 2, 63, 4500], dtype=torch.int32))
    status, ws = g.like(torch.zeros(1, dtype=torch.int32)), g.like(torch.zeros_like(B.alloc_evict_workspace(ctx, "cpu")))
    B.fb_evict_kv(ctx, cache, keep, 10, 2, kp, vp, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    g.check()


def test_offsets_past_32_bits():
    """Pages at the far end of a pool of 5.2 billion elements, records of 4.3 billion cells."""
    lens, heads, width, pages = [130, 100], (32, 32, 128), 1 << 20, 20000
    case = aged(Case(lens, heads, seed=9))
    ctx = B.Context(**case.cfg(num_pages=pages, max_pages_per_req=width))
    kp, vp = (torch.empty(pages, 32, 64, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.zeros(2, width, dtype=torch.int32, device=DEV)
    for r in range(2):
        for i in range(case.width):
            to = pages - 1 - (3 * r + i)
            table[r, i] = to
            kp[to], vp[to] = case.k_pool[case.page_table[r, i]].to(DEV), case.v_pool[case.page_table[r, i]].to(DEV)
    weight = torch.zeros(2, 32, width * 64, device=DEV)
    pos = torch.zeros(2, 32, width * 64, dtype=torch.int32, device=DEV)
    weight[..., :case.cap] = torch.from_numpy(case.kv_weight).to(DEV)
    pos[..., :case.cap] = torch.from_numpy(case.kv_pos).to(DEV)
    cache = B.CacheState(torch.tensor(lens, dtype=torch.int32, device=DEV), torch.from_numpy(case.tok_pos).to(DEV), pos, weight, table)
    status, ws = torch.zeros(1, dtype=torch.int32, device=DEV), B.alloc_evict_workspace(ctx, DEV)
    keep = [70, 33]
    B.fb_evict_kv(ctx, cache, torch.tensor(keep, dtype=torch.int32, device=DEV), 8, 2, kp, vp, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    want = expected(case, keep, 8, 2)
    np.testing.assert_array_equal(cache.kv_len.cpu().numpy(), want[0])
    np.testing.assert_array_equal(pos[..., :case.cap].cpu().numpy(), want[1])
    np.testing.assert_array_equal(weight[..., :case.cap].cpu().numpy(), want[2])
    for r in range(2):
        for i in range(case.width):
            np.testing.assert_array_equal(bits(kp[int(table[r, i])]), want[3][0].numpy()[case.page_table[r, i]])
            np.testing.assert_array_equal(bits(vp[int(table[r, i])]), want[3][1].numpy()[case.page_table[r, i]])


@pytest.mark.parametrize("heads,fp8", [((8, 2, 128), False), ((4, 1, 64), False), ((16, 2, 128), True)])
def test_steps_of_append_attend_evict(heads, fp8):
    """Thirty tokens of three requests over caches of at most 80 keys, against the oracle doing the same.  The oracle goes
    by the kernel's own weights when it evicts (two keys may be nearly equal); those are compared step by step."""
    case = Case([70, 1, 130], heads, fp8, seed=10, pages_per_req=4)
    rng = np.random.default_rng(11)
    R, hkv, hq, d = case.R, case.hkv, case.hq, case.d
    case.kv_pos[:] = np.arange(case.cap)
    case.kv_weight[:] = 0
    case.tok_pos[:] = case.lens - 1
    cfg, ctx = case.oracle_cfg(), case.context()
    cache, kp, vp = case.device()
    status, keep = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((R,), 80, dtype=torch.int32, device=DEV)
    ws, wse = B.alloc_token_workspace(ctx, DEV, True), B.alloc_evict_workspace(ctx, DEV)
    out = torch.zeros(R, hq, d, dtype=torch.bfloat16, device=DEV)
    sc = case.dev_scales() if fp8 else None
    lens, tok, pos, weight = case.lens.copy(), case.tok_pos.copy(), case.kv_pos.copy(), case.kv_weight.copy()
    dec = lambda p, i: O.e4m3_decode(p.cpu().numpy()) * case.scales[i].double().numpy()[None, :, None, None] if fp8 else H.f64(p.cpu())
    for step in range(30):
        lens += 1
        tok += 1
        cache.kv_len += 1
        cache.tok_pos += 1
        new = [torch.from_numpy(rng.normal(size=(R, hkv, d))).to(torch.bfloat16) for _ in range(2)]
        q = torch.from_numpy(rng.normal(size=(R, hq, d))).to(torch.bfloat16)
        before = [p.clone() for p in (kp, vp)]
        if fp8:
            B.fb_append_kv_fp8(ctx, cache, new[0].to(DEV), new[1].to(DEV), kp, vp, *sc, status, 10000.0)
            B.fb_token_attn_fp8(ctx, cache, q.to(DEV), kp, vp, *sc, out, ws, status, accumulate=True)
        else:
            B.fb_append_kv(ctx, cache, new[0].to(DEV), new[1].to(DEV), kp, vp, status, 10000.0)
            B.fb_token_attn(ctx, cache, q.to(DEV), kp, vp, out, ws, status, accumulate=True)
        appended = [p.clone() for p in (kp, vp)]
        grown = cache.kv_weight.clone()
        B.fb_evict_kv(ctx, cache, keep, 16, 2, kp, vp, wse, status)
        torch.cuda.synchronize()
        assert int(status) == 0
        # append: the row (its rotation is compared elsewhere), and nothing else
        for r in range(R):
            page, row = case.page_table[r, (lens[r] - 1) // 64], (lens[r] - 1) % 64
            for i, (a, b) in enumerate(zip(before, appended)):
                np.testing.assert_array_equal(np.delete(bits(a[page]), row, 1), np.delete(bits(b[page]), row, 1))
            pos[r, :, lens[r] - 1] = tok[r]
            weight[r, :, lens[r] - 1] = 0
        # attend
        k64, v64 = dec(appended[0], 0), dec(appended[1], 1)
        ref, w = O.token_attn(cfg, lens, case.page_table, H.f64(q), k64, v64)
        a, _ = O.token_attn(cfg, lens, case.page_table, H.f64(q), k64, np.abs(v64))
        eps = 2.0 ** -11 if fp8 else 2.0 ** -8
        assert (np.abs(H.f64(out.cpu()) - ref) <= (eps + 2.0 ** -12) * 1.01 * a + 2.0 ** -8 * np.abs(ref) + 1e-6).all()
        plain = np.zeros(weight.shape)
        O.add_weights(cfg, lens, plain, w)
        got = grown.cpu().numpy()
        assert (np.abs(got - (weight + plain)) <= 2.0 ** -12 * plain + 2.0 ** -23 * (weight + plain)).all()
        # evict, by the weights that the kernel holds
        weight = got.copy()
        pools = [torch.from_numpy(bits(p).copy()) for p in appended]
        O.evict_kv(cfg, lens, tok, pos, weight, case.page_table, [80] * R, 16, 2, *(p.numpy() for p in pools))
        now = cache.to_numpy()
        np.testing.assert_array_equal(now["kv_len"], lens)
        np.testing.assert_array_equal(now["kv_pos"], pos)
        np.testing.assert_array_equal(now["kv_weight"], weight)
        np.testing.assert_array_equal(bits(kp), pools[0].numpy())
        np.testing.assert_array_equal(bits(vp), pools[1].numpy())
    assert list(lens) == [80, 31, 80]


@pytest.mark.parametrize("heads,fp8,accumulate,pages", [((8, 2, 128), False, True, 4), ((32, 8, 128), True, True, 4), ((32, 8, 128), False, False, 4),
                                                        ((8, 2, 128), False, False, 40)])
def test_a_captured_step_replayed_as_the_lengths_grow(heads, fp8, accumulate, pages):
    """Lengths advanced, token stored, attended to and the caches cut, captured as the context's first calls and
    replayed, against the same calls made directly."""
    case = aged(Case([70, 0, 130, -1], heads, fp8, seed=15, pages_per_req=pages), seed=16)
    case.kv_weight[:] = case.rng.random(case.kv_weight.shape)
    sides = []
    for _ in range(2):
        ctx = case.context()
        cache, kp, vp = case.device()
        R, hkv, hq, d = case.R, case.hkv, case.hq, case.d
        io = [torch.zeros(R, n, d, dtype=torch.bfloat16, device=DEV) for n in (hkv, hkv, hq)]
        out, status = torch.zeros(R, hq, d, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        keep = torch.full((R,), 100, dtype=torch.int32, device=DEV)
        ws, wse = B.alloc_token_workspace(ctx, DEV, accumulate), B.alloc_evict_workspace(ctx, DEV)
        live = torch.tensor([1, 1, 1, 0], dtype=torch.int32, device=DEV)
        sc = case.dev_scales() if fp8 else []

        def step(ctx=ctx, cache=cache, kp=kp, vp=vp, io=io, out=out, status=status, keep=keep, ws=ws, wse=wse, live=live, sc=sc):
            cache.kv_len.add_(live)
            cache.tok_pos.add_(live)
            append, attn = (B.fb_append_kv_fp8, B.fb_token_attn_fp8) if fp8 else (B.fb_append_kv, B.fb_token_attn)
            append(ctx, cache, io[0], io[1], kp, vp, *sc, status, 10000.0)
            attn(ctx, cache, io[2], kp, vp, *sc, out, ws, status, accumulate)
            B.fb_evict_kv(ctx, cache, keep, 8, 2, kp, vp, wse, status)
        sides.append((step, io, out, cache, kp, vp, status))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sides[0][0]()
    gen = torch.Generator().manual_seed(1)
    for _ in range(25):
        new = [torch.randn(x.shape, generator=gen).to(torch.bfloat16) for x in sides[0][1]]
        for _, io, *_ in sides:
            for x, y in zip(io, new):
                x.copy_(y)
        graph.replay()
        sides[1][0]()
        torch.cuda.synchronize()
        (_, _, o0, c0, k0, v0, s0), (_, _, o1, c1, k1, v1, s1) = sides
        assert int(s0) == int(s1) == 0
        for a, b in ((c0.kv_len, c1.kv_len), (c0.kv_pos, c1.kv_pos), (c0.kv_weight, c1.kv_weight), (o0, o1)):
            assert torch.equal(a, b)
        np.testing.assert_array_equal(bits(k0), bits(k1))
        np.testing.assert_array_equal(bits(v0), bits(v1))
    assert c0.kv_len.tolist() == [95, 25, 100, -1]


def test_block_decoding_goes_on_over_a_cut_prefix():
    """A prefix weighed by one query, cut, and read by the block attention: prefix_len is the cut length, and the block
    attends to what stays."""
    bl, heads = 32, (16, 4, 128)
    case = aged(Case([400, 150, 700], heads, seed=12, pages_per_req=12))
    case.kv_weight[:] = 0
    ctx = B.Context(**case.cfg(block_len=bl, wmax=2, max_blocks=4))
    # one query that weighs the stored keys
    cache, kp, vp = case.device()
    status, ws = torch.zeros(1, dtype=torch.int32, device=DEV), B.alloc_token_workspace(ctx, DEV, True)
    q1 = case.q.to(DEV)
    B.fb_token_attn(ctx, cache, q1, kp, vp, torch.empty_like(q1), ws, status, accumulate=True)
    keep = torch.tensor([128, 150, 101], dtype=torch.int32, device=DEV)
    B.fb_evict_kv(ctx, cache, keep, 32, 4, kp, vp, B.alloc_evict_workspace(ctx, DEV), status)
    # two live blocks a request
    R = case.R
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    st = B.DeviceState(z(R) + 1, cache.kv_len, z(R), z(R) + 2, z(R, 4 * bl), torch.zeros(R, 2, dtype=torch.uint8, device=DEV), cache.page_table)
    pk, sb = B.PackBuffers.alloc(ctx, DEV), B.StepBuffers(ctx, DEV)
    n = R * 2 * bl
    q, kw, vw = (torch.randn(n, h, 128, generator=case.gen).to(torch.bfloat16).to(DEV) for h in (16, 4, 4))
    # (the block attention wants finite memory under a page table)
    kp.nan_to_num_(0.25)
    vp.nan_to_num_(0.25)
    B.fb_pack_wavefronts(ctx, st, pk, sb.ws, sb.status)
    B.fb_wavefront_attn(ctx, pk, q, kw, vw, kp, vp, st.page_table, sb.out, sb.ws, sb.status)
    torch.cuda.synchronize()
    assert int(status) == 0 and int(sb.status) == 0
    assert cache.kv_len.tolist() == [128, 150, 101]
    ocfg = O.Config(**case.cfg(block_len=bl, wmax=2, max_blocks=4))
    ost = O.State(np.ones(R, int), cache.kv_len.cpu().numpy(), np.zeros(R, int), np.full(R, 2), np.zeros((R, 4 * bl), int),
                  np.zeros((R, 2), np.uint8), case.page_table)
    opk = O.pack_wavefronts(ocfg, ost)
    ref = O.wavefront_attn(ocfg, opk, H.f64(q.cpu()), H.f64(kw.cpu()), H.f64(vw.cpu()), H.f64(kp.cpu()), H.f64(vp.cpu()), case.page_table)
    max_abs, rel = H.attn_errors(sb.out, ref, H.live_rows(opk, bl))
    assert max_abs <= 1e-2 and rel <= 5e-3, (max_abs, rel)
