"""The serving entry points' host checks under AddressSanitizer and UndefinedBehaviorSanitizer: the sanitized build of the
C ABI's host side, with their refusals in place of the attention calls'."""
from tests import test_sanitizers as S


def test_host_code_under_asan_and_ubsan(tmp_path, monkeypatch):
    run = S._run
    monkeypatch.setattr(S, "_run", lambda tests, *rest: run(["tests/test_serving_abi_cpu.py",
                                                             "tests/test_serving_bounds_cpu.py"], *rest))
    S.test_abi_host_code_under_asan_and_ubsan(tmp_path)
