"""Refusals of the calls around a paged cache at the ends of their ranges (no call here reaches a launch)."""
import paper_2604_17709_amd as dn
from test_cache_step import N, step


def test_a_step_without_rows_needs_both_or_none_of_its_outputs():
    nothing = dict(T=0, slots=None, positions=None)
    assert step(row_start=None, counts=None, **nothing) == dn.OK
    for bad in (dict(row_start=None), dict(counts=None), dict(cached=None), dict(table=None), dict(first=N[7] + 12)):
        assert step(**{**nothing, **bad}) == dn.ERR_INVALID_ARG, bad
    assert step(row_start=N[4] + 2, **nothing) == dn.ERR_MISALIGNED
