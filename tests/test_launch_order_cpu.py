"""Kernels of one stream run one after another: no launch is allowed to start beside its predecessor's end.

With such launches a bounded device wait once ran out for a cause that was not found, so the library has none;
and every launch goes through the check that counts it (omq_launch_count)."""
import os
import re

from paper_2308_13137_gb300 import build


def _sources():
    for f in sorted(os.listdir(build.CSRC)):
        if f.endswith((".cu", ".cuh", ".cpp")):
            with open(os.path.join(build.CSRC, f)) as s:
                yield f, s.read()


def test_no_programmatic_dependence():
    for f, text in _sources():
        assert "griddepcontrol" not in text and "rogrammaticStream" not in text, f


def test_every_launch_is_counted():
    """Launches are followed by OMQ_LAUNCH_CHECK before the function goes on to another or returns."""
    seen = 0
    for f, text in _sources():
        at = [m.start() for m in re.finditer(r"<<<|cudaLaunchKernelEx\(|cudaLaunchCooperativeKernel\(", text)]
        for i, a in enumerate(at):
            after = text[a:text.index("OMQ_LAUNCH_CHECK()", a)] if "OMQ_LAUNCH_CHECK()" in text[a:] else ""
            assert after and "OMQ_OK" not in after, f"{f}: {text[a - 60:a + 60]}"
            seen += 1
    assert seen > 20
