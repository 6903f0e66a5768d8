"""The host tests of the row operators' C entry points under AddressSanitizer and
UndefinedBehaviorSanitizer, as test_sanitizers.py runs those of the scratchpad."""
import subprocess
import sys

from tests.test_sanitizers import ROOT, sanitized  # noqa: F401  (a fixture)


def test_row_entry_points_under_the_sanitizers(sanitized):  # noqa: F811
    tests = ["tests/test_rowapi_host.py", "tests/test_product_forms.py"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", *tests], cwd=ROOT,
                       env=sanitized, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout
