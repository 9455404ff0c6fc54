"""Which kernels hv_fp8_matmul takes (hv_fp8_matmul_launches), by the measures that its rule names."""
import ctypes

import pytest

from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

UNITS = 256
# launch kind -> fragments of 16 rows of B a workgroup has, for up to 16 rows of A
FRAGMENTS = {1: 1, 2: 2, 14: 3, 3: 4, 15: 5, 4: 7}


def kinds(m, n, k, type=hv.HV_BF16, aligned=1):
    count = ctypes.c_int(0)
    kind, splits = (ctypes.c_int * 3)(), (ctypes.c_uint32 * 3)()
    rows, cols = (ctypes.c_uint64 * 3)(), (ctypes.c_uint64 * 3)()
    assert hv.lib.hv_fp8_matmul_launches(type, aligned, m, n, k, ctypes.byref(count), kind, rows, cols,
                                         splits) == hv.HV_OK
    return list(kind[:count.value])


def busiest(m, n, fragments):
    """(rounds, rows) of the workgroups of the unit with the most, and what it loads of each group."""
    workgroups = -(-(-(-n // 16)) // fragments)
    rounds = -(-workgroups // UNITS)
    return rounds, rounds * (16 * fragments + m)


@pytest.mark.parametrize("m", [5, 8, 13, 16])
def test_few_rows_take_the_fragments_that_load_least(m):
    """Of one to five fragments a workgroup, and seven where each unit has one workgroup, the ones whose busiest
    unit loads least; no width is a case of its own."""
    taken = set()
    for n in [16 * UNITS * e - short for e in range(1, 12) for short in (0, 100, 2000)] + [1000, 5001, 18944, 57344, 128256]:
        kind, = kinds(m, n, 4096)
        loads = {e: busiest(m, n, e)[1] for e in (1, 2, 3, 4, 5, 7) if e < 7 or busiest(m, n, e)[0] == 1}
        assert loads[FRAGMENTS[kind]] == min(loads.values()), n
        taken.add(FRAGMENTS[kind])
    assert taken == {1, 2, 3, 4, 5, 7}


def test_up_to_four_rows_take_single_fragments():
    for m in (1, 4):
        for n in (16, 5000, 28672, 57344):
            assert kinds(m, n, 4096) == [1]


@pytest.mark.parametrize("m", [5, 16])
def test_few_rows_at_odd_addresses_take_the_fragments_that_load_least(m):
    """Seven fragments in any number of rounds: their units hold as many requests whatever else they hold."""
    taken = set()
    for n in [16 * UNITS * e - short for e in range(1, 17) for short in (0, 100, 2000)] + [1000, 5001, 57344]:
        kind, = kinds(m, n, 250, aligned=0)
        loads = {e: busiest(m, n, e)[1] for e in (1, 2, 3, 4, 5, 7)}
        assert loads[FRAGMENTS[kind]] == min(loads.values()), n
        taken.add(FRAGMENTS[kind])
    assert taken == {1, 2, 3, 4, 5, 7}


# (m, n, k, type, rows aligned): what is faster by a tenth or more, measured
STREAM, TILES = True, False
MEASURED = [(17, 16384, 4096, hv.HV_BF16, 1, STREAM), (24, 16384, 4096, hv.HV_BF16, 1, STREAM),
            (32, 16384, 8192, hv.HV_BF16, 1, STREAM), (17, 16384, 8192, hv.HV_BF16, 1, STREAM),
            (32, 8192, 1023, hv.HV_BF16, 0, STREAM), (24, 11008, 4096, hv.HV_F32, 1, STREAM),
            (17, 16384, 2047, hv.HV_BF16, 0, TILES), (24, 500, 8192, hv.HV_F32, 1, TILES),
            (17, 500, 4095, hv.HV_F32, 0, TILES), (24, 2000, 4095, hv.HV_F32, 0, TILES),
            (24, 4096, 4095, hv.HV_F32, 0, TILES), (32, 16384, 4095, hv.HV_BF16, 0, TILES)]


@pytest.mark.parametrize("m,n,k,type,aligned,stream", MEASURED)
def test_two_fragments_of_rows_only_where_they_are_faster(m, n, k, type, aligned, stream):
    assert (kinds(m, n, k, type, aligned)[0] in (11, 12, 13)) == stream
