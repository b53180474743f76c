"""The host code of the calls around a paged cache under AddressSanitizer and UndefinedBehaviorSanitizer: their refusals and
the rotary frequencies, in a child process with the sanitized library.  No GPU is involved."""
from paper_2604_17709_amd import build as b
from test_sanitizers import _run


def test_cache_step_host_code_under_asan_and_ubsan():
    _run(["tests/test_cache_step.py"], {"DEINFER_LIBRARY_PATH": b.build_host_sanitized()}, b.asan_runtime())
