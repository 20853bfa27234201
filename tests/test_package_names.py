"""What importing the package needs."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code):
    p = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stderr
    return p.stdout.split()


def test_the_renderer_is_imported_without_torch():
    """All of its names too, where torch is not installed or not wanted."""
    assert "Renderer" in _run("import sys\nsys.modules['torch'] = None\nfrom paper_2103_07013_amd import *\nprint(*dir())")


def test_the_policy_operators_are_names_of_the_package():
    names = _run("import paper_2103_07013_amd as bps\nprint(*dir(bps))\nprint(bps.log_probs.__module__, bps.AdamW.__module__)")
    assert {"Renderer", "log_probs", "log_probs_backward", "LogProbs", "embedding", "embedding_backward", "AdamW"} <= set(names)
    assert names[-2:] == ["paper_2103_07013_amd.policy"] * 2
