"""Decoding one token at a time over the paged K/V cache: the operators, in their plain form and as
the library's calls.

A case is one pass through one operator:

  append  the new token's K and V of every request go to its pages (keys rotated by their absolute
          position on the way), with the records that eviction goes by
  attend  one query token per request over everything its pages hold; with ``weights`` the softmax
          weights are added to the running weight of every stored key
  evict   every request's cache is cut to ``keep`` keys per KV head: the last ``recent`` positions,
          the first ``sinks`` positions and the keys of greatest accumulated weight.  The engine writes
          the bookkeeping of its requests before the call (one copy), so every pass starts from the
          same state

Request counts (1 to 128), head layouts, cache lengths (tens to tens of thousands of keys) and the
64-key pages are those of the decode steps beside this file; ``draw`` spreads over the same ranges.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 64
ROPE_BASE = 10000.0
SMALL, MEDIUM, LARGE = (4, 1, 64), (16, 4, 128), (32, 8, 128)
FP8 = torch.float8_e4m3fn


def _case(name, op, requests, lens, heads, kv="bf16", **more):
    q_heads, kv_heads, head_dim = heads
    c = dict(name=name, op=op, requests=requests, len_lo=lens[0], len_hi=lens[1], q_heads=q_heads, kv_heads=kv_heads,
             head_dim=head_dim, kv=kv, weights=False, keep=0, recent=0, sinks=0)
    c.update(more)
    return c


def listed():
    return [
        # one user, a few thousand tokens in: pure latency, between two matrix products of a layer
        _case("append_chat", "append", 1, (3001, 3001), LARGE),
        # the widest batch, 8-bit pages
        _case("append_128_fp8", "append", 128, (64, 500), LARGE, "fp8"),
        # a toy model's request with one page of context
        _case("attend_tiny", "attend", 1, (64, 64), SMALL),
        # one user, one layer of a full-size model: the latency-critical call
        _case("attend_chat", "attend", 1, (3001, 3001), LARGE),
        # one user with a long document in the cache
        _case("attend_document", "attend", 1, (28123, 28123), LARGE),
        # a middling batch of ragged lengths, eight query heads a KV head, weights for eviction
        _case("attend_24_weights", "attend", 24, (700, 5000), (16, 2, 128), weights=True),
        # the serving batch
        _case("attend_64", "attend", 64, (1024, 8192), LARGE),
        # ... with the cache in 8 bits, weights kept
        _case("attend_64_fp8_weights", "attend", 64, (1024, 8192), LARGE, "fp8", weights=True),
        # long contexts
        _case("attend_long16", "attend", 16, (16384, 32768), LARGE),
        # a batch at its bound: a page's worth of keys over it in every cache
        _case("evict_64_page", "evict", 64, (2112, 2112), LARGE, keep=2048, recent=128, sinks=4),
        # one long document cut to a few thousand keys once its prompt has been read
        _case("evict_document", "evict", 1, (28123, 28123), LARGE, keep=4096, recent=256, sinks=4),
        # the serving batch in 8 bits, ragged: some caches are below the bound and stay as they are
        _case("evict_64_fp8", "evict", 64, (1024, 8192), LARGE, "fp8", keep=2000, recent=128, sinks=4),
    ]


def draw(rng):
    log = lambda lo, hi: math.exp(rng.uniform(math.log(lo), math.log(hi)))
    op = rng.choice(["append", "attend", "attend", "attend", "evict"])
    heads = rng.choice([SMALL, (8, 2, 64), MEDIUM, MEDIUM, LARGE, LARGE, LARGE, (12, 3, 128), (16, 2, 128), (4, 4, 128),
                        (16, 1, 128), (8, 8, 64)])
    hi = round(log(1, 32768))
    lens = (max(1, round(hi * rng.uniform(0.1, 1.0))), hi)
    c = _case("", op, round(log(1, 128)), lens, heads, rng.choice(["bf16", "fp8"]) if heads[2] == 128 else "bf16",
              weights=op == "attend" and rng.random() < 0.4)
    if op == "evict":
        c["keep"] = max(1, round(hi * rng.choice([rng.uniform(0.1, 0.6), rng.uniform(0.9, 1.0)])))
        c["recent"] = round(c["keep"] * rng.uniform(0.0, 0.3))
        c["sinks"] = rng.choice([0, 4])
    del c["name"]
    limit = max(work(k)["bytes"] for k in listed())
    while _pool_bytes(c) > limit and c["requests"] > 1:
        c["requests"] = max(1, c["requests"] * 3 // 4)
    return c


def _pool_bytes(case):
    return case["requests"] * (case["len_hi"] + PAGE) * 2 * case["kv_heads"] * case["head_dim"] * (1 if case["kv"] == "fp8" else 2)


def work(case):
    """What a pass cannot do without.  append: the rows in, as stored out.  attend: the stored keys and
    values once, queries, outputs; the running weights read and written; two products.  evict: weight
    and position of every stored key read, and the rows that survive above the bound moved (the
    survivors of weights drawn alike are spread evenly over the cache)."""
    n, hq, hkv, d = case["requests"], case["q_heads"], case["kv_heads"], case["head_dim"]
    row = 2 * d * (1 if case["kv"] == "fp8" else 2)
    lens = [case["len_lo"] + (i + 0.5) / n * (case["len_hi"] - case["len_lo"]) for i in range(n)]
    if case["op"] == "append":
        return {"bytes": n * hkv * (4 * d + row + 8) + n * 12, "flops": 6.0 * n * hkv * d}
    if case["op"] == "attend":
        keys = sum(lens) * hkv
        return {"bytes": keys * (row + (8 if case["weights"] else 0)) + n * hq * d * 4, "flops": 4.0 * d * hq * sum(lens)}
    moved = sum(case["keep"] * (m - case["keep"]) / m for m in lens if m > case["keep"]) * hkv
    return {"bytes": sum(lens) * hkv * 8 + moved * (2 * row + 16), "flops": sum(lens) * hkv}


# ------------------------------------------------------------------ inputs
def _lengths(case, rng):
    """One length from each of ``requests`` equal slices of the range, in an order of the seed's."""
    n = case["requests"]
    u = (np.arange(n) + rng.random(n)) / n
    lens = case["len_lo"] + np.floor(u * (case["len_hi"] - case["len_lo"] + 1)).astype(np.int64)
    return rng.permutation(np.minimum(lens, case["len_hi"]))


class _State:
    pass


def prepare(case, seed):
    rng = np.random.Generator(np.random.Philox(key=[seed & 0xFFFFFFFF, 37]))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, hq, hkv, d = case["requests"], case["q_heads"], case["kv_heads"], case["head_dim"]
    lens = _lengths(case, rng)
    width = -(-case["len_hi"] // PAGE)
    need = -(-lens // PAGE)
    slices = case["len_lo"] + np.floor(np.arange(1, n + 1) / n * (case["len_hi"] - case["len_lo"] + 1)).astype(np.int64)
    pages = int((-(-np.minimum(slices, case["len_hi"]) // PAGE)).sum())    # the same for every seed
    table = np.zeros((n, width), np.int32)
    perm, at = rng.permutation(pages), 0
    for r in range(n):
        table[r] = perm[at]
        table[r, :need[r]] = perm[at:at + need[r]]
        at += need[r]

    s = _State()
    s.case, cap = case, width * PAGE
    # bookkeeping of the requests in one buffer, so that the engine can write it with one copy: weights and
    # positions of every stored key, lengths, the position of the newest token
    cells = n * hkv * cap
    s.books = torch.zeros(2 * cells + 2 * n, dtype=torch.int32, device=DEV)
    s.kv_weight = s.books[:cells].view(torch.float32).view(n, hkv, cap)
    s.kv_pos = s.books[cells:2 * cells].view(n, hkv, cap)
    s.kv_len, s.tok_pos = s.books[2 * cells:2 * cells + n], s.books[2 * cells + n:]
    s.kv_len.copy_(torch.from_numpy(lens))
    s.tok_pos.copy_(s.kv_len + 700 - 1)               # an earlier cut has taken 700 keys out
    s.table = torch.from_numpy(table).to(DEV)
    j = torch.arange(cap, device=DEV)
    if case["op"] != "append" and (case["weights"] or case["op"] == "evict"):
        # weights gathered so far: a few keys carry most of it, the order of the older ones has been mixed by earlier cuts
        s.kv_weight.copy_(torch.randn(n, hkv, cap, device=DEV, generator=gen).mul_(1.5).exp_().mul_(0.05))
        s.kv_pos.copy_((j + 700).expand(n, hkv, cap))
        s.kv_pos[:, :, :4] = j[:4]
        old = (lens.min() - case["recent"]) // 2
        if old > 8:
            mixed = torch.rand(n, hkv, int(old) - 4, device=DEV, generator=gen).argsort(-1)
            s.kv_pos[:, :, 4:int(old)] = (mixed + 704).to(torch.int32)
        live = j < s.kv_len[:, None, None]
        s.kv_weight.mul_(live)
        s.kv_pos.mul_(live)
    s.books0 = s.books.clone()
    shape = (pages, hkv, PAGE, d)
    s.k_scale = s.v_scale = None
    if case["kv"] == "fp8":
        s.k_scale, s.v_scale = (6.0 / 448.0 * (0.5 + 1.5 * torch.rand(hkv, device=DEV, generator=gen)) for _ in range(2))
        s.k_pool, s.v_pool = (_quantised(torch.randn(shape, device=DEV, generator=gen), sc) for sc in (s.k_scale, s.v_scale))
    else:
        s.k_pool, s.v_pool = (torch.randn(shape, device=DEV, dtype=torch.bfloat16, generator=gen) for _ in range(2))
    if case["op"] == "append":
        s.k_new, s.v_new = (torch.randn(n, hkv, d, device=DEV, dtype=torch.bfloat16, generator=gen) for _ in range(2))
    if case["op"] == "attend":
        s.q = torch.randn(n, hq, d, device=DEV, dtype=torch.bfloat16, generator=gen)
    if case["op"] == "evict":
        s.keep = torch.full((n,), case["keep"], dtype=torch.int32, device=DEV)
    if own:
        _handle(s, cap, pages)
    return s


def _quantised(x, scale):
    return (x / scale[None, :, None, None]).clamp_(-448.0, 448.0).to(FP8).view(torch.uint8)


def _handle(s, cap, pages):
    from paper_2607_17652_b200 import binding as B
    c = s.case
    s.B = B
    s.ctx = B.Context(max_requests=c["requests"], wmax=1, block_len=128 * c["kv_heads"] // c["q_heads"],
                      n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], page_size=PAGE,
                      num_pages=pages, max_pages_per_req=cap // PAGE, vocab=1024, mask_id=1023, eos_id=-1, max_blocks=1,
                      s_pe=0, tau_mask=0.9, tau_edit=0.95, theta_spawn=0.5, sm_scale=0.0,
                      window_in_pages=int(c["kv"] == "fp8"), kv_fp8=int(c["kv"] == "fp8"))
    s.cache = B.CacheState(kv_len=s.kv_len, tok_pos=s.tok_pos, kv_pos=s.kv_pos, kv_weight=s.kv_weight, page_table=s.table)
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    if c["op"] == "attend":
        s.ws = B.alloc_token_workspace(s.ctx, DEV, accumulate=c["weights"])
        s.out = torch.zeros_like(s.q)
    elif c["op"] == "evict":
        s.ws = B.alloc_evict_workspace(s.ctx, DEV)


# ---------------------------------------------------------------- one pass
def _stored(s, pool):
    """A pool as run() returns it: 8-bit pages as the E4M3 values they hold."""
    return pool.view(FP8) if s.case["kv"] == "fp8" else pool


def run(s):
    op = s.case["op"]
    if op == "append":
        if own:
            _append_own(s)
        else:
            _append_plain(s)
        return {"k_pool": _stored(s, s.k_pool), "v_pool": _stored(s, s.v_pool), "kv_pos": s.kv_pos, "kv_weight": s.kv_weight}
    if op == "attend":
        out = _attend_own(s) if own else _attend_plain(s)
        return {"out": out, "kv_weight": s.kv_weight} if s.case["weights"] else {"out": out}
    s.books.copy_(s.books0)                          # the engine writes the bookkeeping of its requests
    if own:
        _evict_own(s)
    else:
        _evict_plain(s)
    return {"k_pool": _stored(s, s.k_pool), "v_pool": _stored(s, s.v_pool), "kv_pos": s.kv_pos, "kv_weight": s.kv_weight,
            "kv_len": s.kv_len}


# the library's calls
def _append_own(s):
    B = s.B
    if s.case["kv"] == "fp8":
        B.fb_append_kv_fp8(s.ctx, s.cache, s.k_new, s.v_new, s.k_pool, s.v_pool, s.k_scale, s.v_scale, s.status, ROPE_BASE)
    else:
        B.fb_append_kv(s.ctx, s.cache, s.k_new, s.v_new, s.k_pool, s.v_pool, s.status, ROPE_BASE)


def _attend_own(s):
    B, w = s.B, s.case["weights"]
    if s.case["kv"] == "fp8":
        B.fb_token_attn_fp8(s.ctx, s.cache, s.q, s.k_pool, s.v_pool, s.k_scale, s.v_scale, s.out, s.ws, s.status, accumulate=w)
    else:
        B.fb_token_attn(s.ctx, s.cache, s.q, s.k_pool, s.v_pool, s.out, s.ws, s.status, accumulate=w)
    return s.out


def _evict_own(s):
    s.B.fb_evict_kv(s.ctx, s.cache, s.keep, s.case["recent"], s.case["sinks"], s.k_pool, s.v_pool, s.ws, s.status)


# the plain forms
def _append_plain(s):
    n, hkv, d = s.k_new.shape
    rows = torch.arange(n, device=DEV)
    last = s.kv_len.long() - 1
    page = s.table[rows, last // PAGE].long()
    k, v = s.k_new.float(), s.v_new.float()
    half = d // 2
    inv = ROPE_BASE ** (-2.0 * torch.arange(half, device=DEV, dtype=torch.float64) / d)
    ang = s.tok_pos.double()[:, None] * inv                # far positions: angles in 64 bits
    cos, sin = ang.cos().float()[:, None, :], ang.sin().float()[:, None, :]
    lo, hi = k[..., :half], k[..., half:]
    k = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)
    if s.case["kv"] == "fp8":
        k = (k / s.k_scale[:, None]).clamp(-448.0, 448.0).to(FP8).view(torch.uint8)
        v = (v / s.v_scale[:, None]).clamp(-448.0, 448.0).to(FP8).view(torch.uint8)
    s.k_pool[page, :, last % PAGE] = k.to(s.k_pool.dtype)
    s.v_pool[page, :, last % PAGE] = v.to(s.v_pool.dtype)
    s.kv_pos[rows, :, last] = s.tok_pos[:, None].expand(n, hkv)
    s.kv_weight[rows, :, last] = 0.0


def _gathered(pool, table, scale):
    """[requests, KV heads, keys, d] in 32 bits."""
    x = pool[table.long()]
    n, p, hkv, page, d = x.shape
    x = (x.view(FP8).float() * scale[:, None, None] if scale is not None else x.float())
    return x.transpose(1, 2).reshape(n, hkv, p * page, d)


def _attend_plain(s):
    n, hq, d = s.q.shape
    hkv = s.k_pool.shape[1]
    k = _gathered(s.k_pool, s.table, s.k_scale)
    live = (torch.arange(k.shape[2], device=DEV) < s.kv_len[:, None])[:, None, None, :]
    z = torch.matmul(s.q.float().view(n, hkv, hq // hkv, d), k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    del k
    z = z.masked_fill(~live, -math.inf)
    w = (z - z.amax(-1, keepdim=True)).exp()
    w = w / w.sum(-1, keepdim=True)
    out = torch.matmul(w, _gathered(s.v_pool, s.table, s.v_scale))
    if s.case["weights"]:
        s.kv_weight += w.sum(2)
    return out.reshape(n, hq, d).to(torch.bfloat16)


def _evict_plain(s):
    n, hkv, cap = s.kv_pos.shape
    j = torch.arange(cap, device=DEV)
    size = s.kv_len[:, None, None]
    safe = (s.kv_pos < s.case["sinks"]) | (s.kv_pos > (s.tok_pos - s.case["recent"])[:, None, None])
    rank = torch.where(safe, math.inf, s.kv_weight).masked_fill(j >= size, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices        # ties: the lower index first
    new = torch.minimum(s.kv_len, s.keep)
    stays = torch.zeros(n, hkv, cap, dtype=torch.bool, device=DEV)
    stays.scatter_(2, order, (j < new[:, None, None]).expand(n, hkv, cap))
    below = j < new[:, None, None]
    r, h, to = torch.nonzero(below & ~stays, as_tuple=True)            # i-th hole and i-th survivor above the bound
    _, _, at = torch.nonzero(~below & stays, as_tuple=True)            # of the same request and head
    pt, pa = s.table[r, to // PAGE].long(), s.table[r, at // PAGE].long()
    for pool in (s.k_pool, s.v_pool):
        pool[pt, h, to % PAGE] = pool[pa, h, at % PAGE]
    s.kv_pos[r, h, to] = s.kv_pos[r, h, at]
    s.kv_weight[r, h, to] = s.kv_weight[r, h, at]
    s.kv_len.copy_(new)


# ---------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    lens, table = s.kv_len.tolist(), s.table.long()
    group, d = case["q_heads"] // case["kv_heads"], case["head_dim"]

    def values(pool, scale, r):
        """What request r's pages hold, [KV heads, keys, d]."""
        x = pool[table[r, :-(-lens[r] // PAGE)]]
        x = x.view(FP8).double() * scale.double()[None, :, None, None] if scale is not None else x.double()
        return x.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, d)[:, :lens[r]]

    if case["op"] == "attend":
        out = torch.empty(s.q.shape, dtype=torch.float64, device=DEV)
        weight = s.kv_weight.double()
        for r in range(case["requests"]):
            k, v = values(s.k_pool, s.k_scale, r), values(s.v_pool, s.v_scale, r)
            for h in range(case["kv_heads"]):
                w = torch.softmax(s.q[r, h * group:(h + 1) * group].double() @ k[h].T / d ** 0.5, -1)
                out[r, h * group:(h + 1) * group] = w @ v[h]
                weight[r, h, :lens[r]] += w.sum(0)
        return {"out": out, "kv_weight": weight} if case["weights"] else {"out": out}

    k_pool, v_pool = (_stored(s, p).double() for p in (s.k_pool, s.v_pool))
    if case["op"] == "append":
        at = [(int(table[r, (m - 1) // PAGE]), (m - 1) % PAGE) for r, m in enumerate(lens)]
        turn = np.exp(1j * np.outer(s.tok_pos.cpu().numpy().astype(np.float64), ROPE_BASE ** (-np.arange(0, d, 2) / d)))
        x = s.k_new.double().cpu().numpy()
        z = (x[..., :d // 2] + 1j * x[..., d // 2:]) * turn[:, None, :]
        k = torch.from_numpy(np.concatenate([z.real, z.imag], -1)).to(DEV)
        v = s.v_new.double()
        if case["kv"] == "fp8":
            k, v = (x.clamp(-448.0, 448.0) for x in (k / s.k_scale.double()[:, None], v / s.v_scale.double()[:, None]))
        for r, (page, t) in enumerate(at):
            k_pool[page, :, t], v_pool[page, :, t] = k[r], v[r]
            s.kv_pos[r, :, lens[r] - 1], s.kv_weight[r, :, lens[r] - 1] = s.tok_pos[r], 0.0
        return {"k_pool": k_pool, "v_pool": v_pool, "kv_pos": s.kv_pos, "kv_weight": s.kv_weight.double()}

    pos, weight = s.kv_pos.cpu().numpy(), s.kv_weight.cpu().numpy().astype(np.float64)
    newest = s.tok_pos.tolist()
    for r, m in enumerate(lens):
        if m <= case["keep"]:
            continue
        for h in range(case["kv_heads"]):
            p, w = pos[r, h], weight[r, h]
            free = ~((p[:m] < case["sinks"]) | (p[:m] > newest[r] - case["recent"]))
            kept = np.sort(np.lexsort((np.arange(m), -w[:m], free))[:case["keep"]])
            above = kept[kept >= case["keep"]]
            holes = np.setdiff1d(np.arange(case["keep"]), kept)
            p[holes], w[holes] = p[above], w[above]
            to, fr = torch.from_numpy(holes).to(DEV), torch.from_numpy(above).to(DEV)
            for pool in (k_pool, v_pool):
                pool[table[r, to // PAGE], h, to % PAGE] = pool[table[r, fr // PAGE], h, fr % PAGE]
        lens[r] = case["keep"]
    return {"k_pool": k_pool, "v_pool": v_pool, "kv_pos": torch.from_numpy(pos), "kv_weight": torch.from_numpy(weight),
            "kv_len": torch.tensor(lens, dtype=torch.int32)}
