"""The boundary suite of the products, the recurrence and AdamW under the host sanitizers, as
tests/test_abi_sanitizers.py runs the others."""
import os

from tests.test_abi_sanitizers import ROOT, _child, sanitized  # noqa: F401


def test_training_boundary_suite_passes_under_asan_and_ubsan(sanitized):  # noqa: F811
    _, env = sanitized
    r = _child(env, ["-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu",
                     os.path.join(ROOT, "tests", "test_train_abi.py")])
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
    assert " passed" in r.stdout, tail


def test_training_refusals_pass_under_asan_and_ubsan(sanitized):  # noqa: F811
    """(Without the thread of 96 KB: instrumented frames are larger.)"""
    _, env = sanitized
    r = _child(env, ["-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu", "-k", "not small_stack",
                     os.path.join(ROOT, "tests", "test_train_refusals.py")])
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
    assert " passed" in r.stdout, tail
