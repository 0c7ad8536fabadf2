"""What the calls that decode one token at a time refuse, on the host: no launch is made, no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2607_17652_b200 import binding as B

GOOD = dict(max_requests=4, wmax=1, block_len=32, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=64, num_pages=16,
            max_pages_per_req=4, vocab=1024, mask_id=1023, eos_id=-1, max_blocks=1, s_pe=0, tau_mask=0.9, tau_edit=0.95,
            theta_spawn=0.5, sm_scale=0.0)
FP8 = dict(GOOD, kv_fp8=1, window_in_pages=1)
P = 0x1000                         # a pointer that nothing may follow


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_17652_b200 import build
    build.build()


def full():
    return B.fb_cache(*([P] * 5))


def with_null(name):
    kv = full()
    setattr(kv, name, None)
    return kv


def refused(ctx, rc, code, text):
    assert rc == code
    assert text in B.lib().fb_last_error(ctx.handle)


def test_append_refuses():
    lib, ctx, ctx8 = B.lib(), B.Context(**GOOD), B.Context(**FP8)
    call = lambda c, kv, *a: lib.fb_append_kv(c.handle, kv and C.byref(kv), *a)
    ok = [P, P, P, P, 0.0, P, None]
    refused(ctx, call(ctx, None, *ok), B.FB_ERR_INVALID_ARG, b"cache is null")
    for name in ("kv_len", "page_table"):
        refused(ctx, call(ctx, with_null(name), *ok), B.FB_ERR_INVALID_ARG, b"cache.kv_len or cache.page_table")
    refused(ctx, call(ctx, with_null("tok_pos"), *ok), B.FB_ERR_INVALID_ARG, b"tok_pos")
    for i in (0, 1, 2, 3, 5):
        a = list(ok)
        a[i] = None
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_INVALID_ARG, b"null")
    for i in range(4):
        a = list(ok)
        a[i] = P + 8
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_ALIGNMENT, b"16-byte")
    for base in (-1.0, float("nan")):
        a = list(ok)
        a[4] = base
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_INVALID_ARG, b"rope_base")
    refused(ctx8, call(ctx8, full(), *ok), B.FB_ERR_UNSUPPORTED, b"_fp8")
    call8 = lambda c, *a: lib.fb_append_kv_fp8(c.handle, C.byref(full()), *a)
    refused(ctx, call8(ctx, P, P, P, P, P, P, 0.0, P, None), B.FB_ERR_UNSUPPORTED, b"kv_fp8 = 1")
    refused(ctx8, call8(ctx8, P, P, P, P, None, P, 0.0, P, None), B.FB_ERR_INVALID_ARG, b"null")
    assert lib.fb_append_kv(None, None, *ok) == B.FB_ERR_INVALID_ARG
    wide = B.Context(**dict(GOOD, max_pages_per_req=1 << 25))
    refused(wide, call(wide, full(), *ok), B.FB_ERR_UNSUPPORTED, b"2^30")


def cache_tensors(**over):
    c = dict(kv_len=torch.zeros(4, dtype=torch.int32), tok_pos=torch.zeros(4, dtype=torch.int32),
             kv_pos=torch.zeros(4, 2, 256, dtype=torch.int32), kv_weight=torch.zeros(4, 2, 256),
             page_table=torch.zeros(4, 4, dtype=torch.int32))
    c.update(over)
    return B.CacheState(**c)


def tensors():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    return dict(k=bf(4, 2, 128), v=bf(4, 2, 128), pool=bf(16, 2, 64, 128), status=torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("name,bad", [
    ("kv_len", torch.zeros(4, dtype=torch.int64)), ("kv_len", torch.zeros(5, dtype=torch.int32)),
    ("tok_pos", torch.zeros(8, dtype=torch.int32)[::2]), ("kv_pos", torch.zeros(4, 2, 192, dtype=torch.int32)),
    ("kv_weight", torch.zeros(4, 2, 256, dtype=torch.float64)), ("page_table", torch.zeros(4, 8, dtype=torch.int32)[:, :4])])
def test_records_of_another_type_size_or_stride_are_refused(name, bad, monkeypatch):
    ctx, t = B.Context(**GOOD), tensors()
    monkeypatch.setattr(B, "_device", lambda: -1)      # (tensors in host memory say -1: only the checks are meant)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    with pytest.raises(ValueError, match=name):
        B.fb_append_kv(ctx, cache_tensors(**{name: bad}), t["k"], t["v"], t["pool"], t["pool"], t["status"])


def test_tensors_of_another_type_size_stride_or_device_are_refused(monkeypatch):
    ctx, t = B.Context(**GOOD), tensors()
    monkeypatch.setattr(B, "_device", lambda: -1)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    bad = {"k": [t["k"].float(), t["k"][:3], torch.zeros(4, 2, 256, dtype=torch.bfloat16)[..., ::2], t["k"].transpose(0, 1)],
           "pool": [t["pool"][:15], t["pool"].to(torch.float16), torch.zeros(16, 2, 64, 128, dtype=torch.uint8)],
           "status": [torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)]}
    for name, values in bad.items():
        for x in values:
            u = dict(t, **{name: x})
            with pytest.raises(ValueError, match="contiguous"):
                B.fb_append_kv(ctx, cache_tensors(), u["k"], u["v"], u["pool"], u["pool"], u["status"])
    monkeypatch.setattr(B, "_device", lambda: 0)       # tensors elsewhere than on the current device
    with pytest.raises(ValueError, match="device 0"):
        B.fb_append_kv(ctx, cache_tensors(), t["k"], t["v"], t["pool"], t["pool"], t["status"])


def test_token_attn_refuses():
    lib, ctx, ctx8 = B.lib(), B.Context(**GOOD), B.Context(**FP8)
    call = lambda c, kv, *a: lib.fb_token_attn(c.handle, kv and C.byref(kv), *a)
    ok = [P, P, P, P, 0, P, P, None]               # q, k_pool, v_pool, out, accumulate, ws, status, stream
    refused(ctx, call(ctx, None, *ok), B.FB_ERR_INVALID_ARG, b"cache is null")
    for name in ("kv_len", "page_table"):
        refused(ctx, call(ctx, with_null(name), *ok), B.FB_ERR_INVALID_ARG, b"cache.kv_len or cache.page_table")
    for i in (0, 1, 2, 3, 6):
        a = list(ok)
        a[i] = None
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_INVALID_ARG, b"null")
    a = list(ok)
    a[5] = None
    refused(ctx, call(ctx, full(), *a), B.FB_ERR_WORKSPACE, b"workspace is null")
    for i in (0, 1, 2, 3, 5):
        a = list(ok)
        a[i] = P + 8
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_ALIGNMENT, b"aligned")
    for acc in (2, -1):
        a = list(ok)
        a[4] = acc
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_INVALID_ARG, b"accumulate")
    a[4] = 1
    refused(ctx, call(ctx, with_null("kv_weight"), *a), B.FB_ERR_INVALID_ARG, b"kv_weight")
    refused(ctx8, call(ctx8, full(), *ok), B.FB_ERR_UNSUPPORTED, b"_fp8")
    call8 = lambda c, *b: lib.fb_token_attn_fp8(c.handle, C.byref(full()), *b)
    ok8 = [P, P, P, P, P, P, 0, P, P, None]
    refused(ctx, call8(ctx, *ok8), B.FB_ERR_UNSUPPORTED, b"kv_fp8 = 1")
    refused(ctx8, call8(ctx8, P, P, P, P, None, P, 0, P, P, None), B.FB_ERR_INVALID_ARG, b"null")
    assert lib.fb_token_attn(None, None, *ok) == B.FB_ERR_INVALID_ARG
    assert lib.fb_token_workspace_bytes(None, 0) == 0
    assert lib.fb_token_workspace_bytes(ctx.handle, 1) >= lib.fb_token_workspace_bytes(ctx.handle, 0) > 0


def test_token_attn_refuses_tensors_that_do_not_fit(monkeypatch):
    ctx, t = B.Context(**GOOD), tensors()
    monkeypatch.setattr(B, "_device", lambda: -1)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    ws = [B.alloc_token_workspace(ctx, "cpu", a) for a in (False, True)]
    bad = [dict(q=q[:3]), dict(q=q.half()), dict(q=q.transpose(0, 1)), dict(out=q.float()), dict(out=q[:, ::2]),
           dict(ws=ws[0][:-1].clone()), dict(ws=ws[1][:-1].clone(), acc=True), dict(pool=t["pool"][:8]), dict(status=t["status"].long())]
    for b in bad:
        u = dict(dict(q=q, out=q.clone(), ws=ws[1], pool=t["pool"], status=t["status"], acc=False), **b)
        if "ws" in b and not u["acc"] and b["ws"].numel() >= B.lib().fb_token_workspace_bytes(ctx.handle, 0):
            u["ws"] = torch.zeros(8, dtype=torch.uint8)
        if "ws" in b and u["acc"] and b["ws"].numel() >= B.lib().fb_token_workspace_bytes(ctx.handle, 1):
            u["ws"] = torch.zeros(8, dtype=torch.uint8)
        with pytest.raises(ValueError, match="contiguous"):
            B.fb_token_attn(ctx, cache_tensors(), u["q"], u["pool"], u["pool"], u["out"], u["ws"], u["status"], u["acc"])


def test_evict_refuses():
    lib, ctx, ctx8 = B.lib(), B.Context(**GOOD), B.Context(**FP8)
    call = lambda c, kv, *a: lib.fb_evict_kv(c.handle, kv and C.byref(kv), *a)
    ok = [P, 16, 4, P, P, P, P, None]              # keep, recent, sinks, k_pool, v_pool, ws, status, stream
    refused(ctx, call(ctx, None, *ok), B.FB_ERR_INVALID_ARG, b"cache is null")
    for name in ("kv_len", "page_table"):
        refused(ctx, call(ctx, with_null(name), *ok), B.FB_ERR_INVALID_ARG, b"cache.kv_len or cache.page_table")
    for name in ("tok_pos", "kv_pos", "kv_weight"):
        refused(ctx, call(ctx, with_null(name), *ok), B.FB_ERR_INVALID_ARG, b"cache.tok_pos, cache.kv_pos or cache.kv_weight")
    for i in (0, 3, 4, 6):
        a = list(ok)
        a[i] = None
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_INVALID_ARG, b"null")
    for i in (1, 2):
        a = list(ok)
        a[i] = -1
        for c in (ctx, ctx8):
            refused(c, call(c, full(), *a), B.FB_ERR_INVALID_ARG, b"recent and sinks")
    a = list(ok)
    a[5] = None
    refused(ctx, call(ctx, full(), *a), B.FB_ERR_WORKSPACE, b"workspace is null")
    for i in (3, 4, 5):
        a = list(ok)
        a[i] = P + 8
        refused(ctx, call(ctx, full(), *a), B.FB_ERR_ALIGNMENT, b"aligned")
    for name in ("kv_pos", "kv_weight"):
        kv = full()
        setattr(kv, name, P + 4)
        refused(ctx, call(ctx, kv, *ok), B.FB_ERR_ALIGNMENT, b"16-byte")
    assert lib.fb_evict_kv(None, None, *ok) == B.FB_ERR_INVALID_ARG
    assert lib.fb_evict_workspace_bytes(None) == 0 and lib.fb_evict_workspace_bytes(ctx.handle) > 0
    wide = B.Context(**dict(GOOD, max_pages_per_req=1 << 25))
    refused(wide, call(wide, full(), *ok), B.FB_ERR_UNSUPPORTED, b"2^30")


def test_evict_refuses_tensors_that_do_not_fit(monkeypatch):
    ctx, t = B.Context(**GOOD), tensors()
    monkeypatch.setattr(B, "_device", lambda: -1)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    keep, ws = torch.zeros(4, dtype=torch.int32), torch.zeros(B.lib().fb_evict_workspace_bytes(ctx.handle), dtype=torch.uint8)
    for bad in (dict(keep=keep[:3]), dict(keep=keep.long()), dict(keep=torch.zeros(8, dtype=torch.int32)[::2]), dict(ws=ws[:-1].clone()),
                dict(ws=ws.view(torch.int32)), dict(pool=t["pool"].view(torch.int16)), dict(pool=torch.zeros(16, 2, 64, 128, dtype=torch.uint8)),
                dict(status=t["status"].float())):
        u = dict(dict(keep=keep, ws=ws, pool=t["pool"], status=t["status"]), **bad)
        with pytest.raises(ValueError, match="contiguous"):
            B.fb_evict_kv(ctx, cache_tensors(), u["keep"], 4, 2, u["pool"], u["pool"], u["ws"], u["status"])
    for name in ("tok_pos", "kv_pos", "kv_weight"):
        with pytest.raises(B.FlowBlockError, match="null"):
            B.fb_evict_kv(ctx, cache_tensors(**{name: None}), keep, 4, 2, t["pool"], t["pool"], ws, t["status"])
