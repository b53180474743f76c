"""The host code of the calls between the projections of a prompt under AddressSanitizer and UndefinedBehaviorSanitizer: their
refusals and the axes of rotary pairs, in a child process with the sanitized library.  No GPU is involved."""
from paper_2604_17709_amd import build as b
from test_sanitizers import _run


def test_prompt_host_code_under_asan_and_ubsan():
    _run(["tests/test_prompt.py"], {"DEINFER_LIBRARY_PATH": b.build_host_sanitized()}, b.asan_runtime())
