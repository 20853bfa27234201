"""How many chunks the scans cut their time into, by what they launch on the stand-in for the HIP runtime."""
import pytest

from test_memory_launches import _calls, fake  # noqa: F401


@pytest.mark.parametrize("steps,chunks", [(1, 1), (64, 1), (127, 1), (128, 2), (129, 2), (191, 2), (192, 3), (193, 3), (256, 4), (1000, 13), (4096, 64)])
@pytest.mark.parametrize("states", [3, 16, 32])
def test_chunks_have_64_steps_or_more(fake, steps, chunks, states):  # noqa: F811
    """One sequence of few channels: only their shortest length limits them.  As many chunks as have 64 steps, of as many steps as that makes, rounded up to tiles
    of 16: 1000 steps are 15 times 67, so 80 each, 13 chunks."""
    (status, _, forward), (back, _, backward) = _calls(fake, f"scan(1, {steps}, 64, {states})")
    assert status == 0 and back == 0
    scans, grads = [g for n, g, _ in forward if n == "k_scan"], [g for n, g, _ in backward if n == "k_scan_grad_first"]
    assert scans[-1] == chunks and (chunks == 1) == (len(scans) == 1) == (not grads)
    if chunks > 1:
        assert scans[0] == chunks - 1 and grads == [chunks - 1]
