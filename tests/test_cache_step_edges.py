"""Refusals of the calls around a paged cache at the ends of their ranges (no call here reaches a launch)."""
import paper_2604_17709_amd as dn
from test_cache_step import N, rope, step


def test_a_step_without_rows_needs_both_or_none_of_its_outputs():
    nothing = dict(T=0, slots=None, positions=None)
    assert step(row_start=None, counts=None, **nothing) == dn.OK
    for bad in (dict(row_start=None), dict(counts=None), dict(cached=None), dict(table=None), dict(first=N[7] + 12)):
        assert step(**{**nothing, **bad}) == dn.ERR_INVALID_ARG, bad
    assert step(row_start=N[4] + 2, **nothing) == dn.ERR_MISALIGNED


def test_a_rotary_store_without_rows_whatever_its_tensors_are():
    """A tensor without rows has no address, the pool beside it has one."""
    for nothing in (dict(q=None), dict(k=None), dict(v=None), dict(q=None, k=None, v=None, pos=None, slots=None), dict(qo=None), dict(q=None, qo=None)):
        assert rope(T=0, **nothing) == dn.OK, nothing
    assert rope(T=0, rot=31) == dn.ERR_INVALID_ARG and rope(T=0, dtype=7) == dn.ERR_UNSUPPORTED
