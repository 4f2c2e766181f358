"""The 4-bit calls at the ends of their ranges, on the host: plans, sizes and refusals (nothing here
launches a kernel)."""
import ctypes

import numpy as np
import pytest
import torch

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


# ------------------------------------------------- whole numbers past 32 bits
FAKE = 1 << 20            # aligned non-null address, never dereferenced
PAST = [2 ** 32, 2 ** 32 + 100, 2 ** 31, -2 ** 31 - 1, 2 ** 64 + 1]


@pytest.mark.parametrize("n", PAST)
def test_library_arguments_are_not_cut_to_32_bits(lib, n):
    """(T = 0 rows to store: nothing is enqueued whatever becomes of the number.)"""
    for a in (dict(start=n), dict(T=n), dict(cap=n), dict(D=n)):
        a = dict(dict(start=0, T=0, cap=16, Hkv=2, D=64), **a)
        with pytest.raises(ctypes.ArgumentError, match="32-bit"):
            lib.kv4_store(FAKE, FAKE, None, a["start"], a["T"], a["cap"], a["Hkv"], a["D"], FAKE, FAKE, None)
    assert lib.kv4_store(FAKE, FAKE, None, INT32_MAX, 0, 16, 2, 64, FAKE, FAKE, None) == -2


@pytest.mark.parametrize("n", PAST)
def test_sizes_of_such_numbers_are_refused(n):
    for f, a in ((al.lmhead_packed_weight_mx4_size, (64, n)), (al.lmhead_packed_weight_mx4_size, (n, 64)),
                 (al.lmhead_confidence_mx4_workspace_size, (n, 64, 100)),
                 (al.lane_attn_kv4_workspace_size, (1, 1, n, 4, 4, 64)),
                 (al.lane_attn_workspace_size, (1, 16, n, 4, 4, 64)), (al.lmhead_packed_weight_size, (64, n)),
                 (al.lmhead_confidence_workspace_size, (1, 64, n))):
        with pytest.raises(al.AsyncLaneError, match="32-bit"):
            f(*a)


@pytest.mark.parametrize("V", PAST)
def test_lmhead_refuses_such_vocabularies(V):
    h = torch.zeros(8, 64, dtype=torch.bfloat16)
    with pytest.raises(al.AsyncLaneError, match="32-bit"):
        al.lmhead_confidence_mx4(h, torch.zeros(8704, dtype=torch.uint8), V)
    with pytest.raises(al.AsyncLaneError, match="32-bit"):
        al.lmhead_confidence_packed(h, torch.zeros(8192, dtype=torch.bfloat16), V)
    with pytest.raises(al.AsyncLaneError, match="32-bit"):   # (a weight of so many rows, without its memory)
        al.lmhead_pack_weight_mx4(torch.empty(2 ** 32 + 100, 32, dtype=torch.uint8, device="meta"),
                                  torch.empty(2 ** 32 + 100, 2, dtype=torch.uint8, device="meta"))


def test_numbers_of_other_types_are_still_taken():
    want = al.lane_attn_kv4_workspace_size(1, 1, 4096, 4, 2, 64)
    assert want > 0 and al.lane_attn_kv4_workspace_size(*np.array([1, 1, 4096, 4, 2, 64])) == want
    assert al.lane_attn_kv4_workspace_size(True, 1, 4096, 4, 2, 64) == want
