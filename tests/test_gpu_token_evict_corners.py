"""fb_evict_kv where its order turns on one comparison: positions above the newest one, and ties in caches so long that a CTA
goes through its keys in chunks.  Against the oracle, everything bit for bit."""
import numpy as np
import pytest

from tests.test_gpu_token_evict import WEIGHTS, aged, check
from tests.token_harness import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("recent", [0, 1, 40, 2 ** 31 - 1])
@pytest.mark.parametrize("tok", [-2 ** 31, -1, 0, 1, 250, 2 ** 31 - 1])
def test_positions_above_the_newest_are_protected(recent, tok):
    """Protected is kv_pos > tok_pos - recent, so a caller that has taken tok_pos back keeps what lies above it, with
    recent = 0 too."""
    case = Case([600, 600], (4, 2, 64), seed=31)
    case.kv_pos[0] = case.rng.choice([-2 ** 31, -2, -1, 0, 1, 2, 249, 250, 251, 2 ** 31 - 1], case.kv_pos[0].shape)
    case.kv_pos[1] = case.rng.permutation(case.cap)[None]
    case.tok_pos[:] = tok
    check(case, [300, 77], recent, 0)


# one request on one KV head: eight CTAs have 17,500 keys each, of which 8,192 are in shared memory at a time
LONG, SPAN, CHUNK = 140000, 17500, 8192


def long_case(kind, seed):
    case = aged(Case([LONG], (4, 1, 64), seed=seed, fill=False))
    with np.errstate(all="ignore"):
        case.kv_weight = WEIGHTS[kind](case.rng, case.kv_weight.shape).astype(np.float32)
    return case


@pytest.mark.parametrize("kind", ["equal", "few values", "nan alone", "signed zeros", "one bit apart"])
@pytest.mark.parametrize("at", [SPAN * 3 + CHUNK + 3000, SPAN * 7 + 2 * CHUNK + 100, CHUNK])
def test_ties_across_chunks(kind, at):
    """The boundary among equal keys lies at index `at`: in a second chunk, in the last one of the last CTA, at a chunk's
    first key."""
    recent, sinks = 10, 2
    case = long_case(kind, seed=32)
    pos, w = case.kv_pos[0, 0, :LONG], case.kv_weight[0, 0, :LONG]
    safe = (pos < sinks) | (pos > int(case.tok_pos[0]) - recent)
    value = np.where(np.isnan(w), -np.inf, w).astype(np.float64) + 0.0
    at = int(np.nonzero(~safe[at:])[0][0]) + at
    keep = int(safe.sum() + (~safe & (value > value[at])).sum() + (~safe & (value == value[at]))[:at + 1].sum())
    assert (~safe & (value == value[at]))[at + 1:].any() or at > SPAN * 7
    check(case, [keep], recent, sinks)


@pytest.mark.parametrize("recent,sinks", [(2 ** 31 - 1, 0), (0, 2 ** 31 - 1), (90000, 4)])
def test_more_protected_than_kept_across_chunks(recent, sinks):
    case = long_case("few values", seed=33)
    pos = case.kv_pos[0, 0, :LONG]
    assert ((pos < sinks) | (pos > int(case.tok_pos[0]) - recent)).sum() > SPAN * 3 + CHUNK + 3000
    check(case, [SPAN * 3 + CHUNK + 3000], recent, sinks)
