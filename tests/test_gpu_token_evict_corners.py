"""fb_evict_kv where its order turns on one comparison: positions above the newest one.  Against the oracle, everything bit
for bit."""
import pytest

from tests.test_gpu_token_evict import check
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
