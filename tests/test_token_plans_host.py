"""The plans of the operators for token models (token_plans.hip): workspaces, places of states, shares of workgroups.  No GPU."""
import os
import subprocess

import pytest

from conftest import ROOT
from paper_2605_24584_amd import build


@pytest.mark.parametrize("source", ["attention", "logprob"])
def test_plans(source, tmp_path):
    program = str(tmp_path / source)
    flags = [f for f in build.FLAGS if f not in ("-O3", "-Wall")] + ["-O1", "-w"] + (["-DPLANS_OF_ATTENTION"] if source == "attention" else [])
    subprocess.run([build.HIPCC, *flags, os.path.join(ROOT, "tests", "token_plans.hip"), "-o", program], check=True, stderr=subprocess.DEVNULL)
    run = subprocess.run([program], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stdout
