"""Host code of drafted trees on the CPU: refusals, scratch, lengths, against a stand-in for the HIP runtime."""
import subprocess

import pytest

from paper_2605_09490_amd import build


@pytest.mark.parametrize("scenario", ["refusals", "scratch", "refused_scratch", "lengths_and_gaps"])
def test_host_code_of_trees(scenario):
    r = subprocess.run([build.build_fake_check("tree_host_check"), scenario], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and f"{scenario}: ok" in r.stdout, r.stdout + r.stderr
