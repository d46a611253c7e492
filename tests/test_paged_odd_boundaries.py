"""Boundaries of chunks and segments are values on the device, which the host does not see: whatever they are, the
kernels' look-ups stay inside the tensors and end (no GPU; tests/host_harness/paged_harness.cpp with "odd", under
AddressSanitizer and UndefinedBehaviorSanitizer)."""

from test_paged_host_sanitized import _run, harness  # noqa: F401


def test_boundaries_that_are_anything_lead_nowhere_outside(harness):  # noqa: F811
    r = _run(harness, "odd")
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert " 0 failures" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
