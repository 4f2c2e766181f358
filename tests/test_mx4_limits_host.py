"""The 4-bit calls at the ends of their ranges, on the host: plans, sizes and refusals (nothing here
launches a kernel)."""
import ctypes

import pytest

import paper_2606_08411_amd as al

INT32_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    return al.library()


# L, B, Hq, Hkv, refreshed rows: the token kernel, the unit kernel, the tile kernel, refreshed rows alone
LONGEST = [(1, 1, 4, 1, 0), (2, 16, 8, 2, 0), (64, 64, 4, 1, 0), (0, 1, 4, 1, 5000)]


@pytest.mark.parametrize("short_of", [0, 1, 30, 31, 62, 63, 64])
@pytest.mark.parametrize("case", LONGEST, ids=str)
def test_the_longest_prefixes_have_the_plan_of_long_ones(lib, case, short_of):
    """A prefix of up to INT32_MAX rows: counting its key tiles does not pass 32 bits."""
    L, B, Hq, Hkv, n_ref = case

    def plan(P):
        out = (ctypes.c_int32 * 4)()
        assert lib.al_internal_kv4_plan(L, B, P, Hq, Hkv, 64, n_ref, out) == 0
        return tuple(out), lib.lane_attn_kv4_workspace_size(L, B, P, Hq, Hkv, 64, n_ref)
    want = plan(INT32_MAX - 1000)
    assert max(want[0]) > 1 and want[1] > 0
    assert plan(INT32_MAX - short_of) == want
