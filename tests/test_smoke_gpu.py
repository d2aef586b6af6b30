"""The smoke entry point passes: one small calibration step against the oracle."""
import pytest

pytestmark = pytest.mark.gpu


def test_smoke(cuda_lib):
    import __graft_entry__ as entry
    entry.smoke()
