"""The operators on rows of tokens, host side: what needs no GPU of their argument checks and workspaces."""
import os
import subprocess
import sys

import pytest

from paper_2205_12268_amd import wcc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NO_ROWS = """
from paper_2205_12268_amd import wcc
for t in (wcc.F32, wcc.BF16):
    for V in (1, 7, 1000, 4097, 100000, 2 ** 31 - 1):
        for k in (1, min(V, 64)):
            assert wcc.scores_workspace_bytes(wcc.make_scores_desc(0, V, k, t)) == 0
            assert wcc.distill_workspace_bytes(wcc.make_distill_desc(0, V, k, t)) == 0
        assert wcc.scores_workspace_bytes(wcc.make_scores_desc(0, V, 0, t)) == 0
    for n in (0, 3):
        wcc.adapter_workspace_bytes(wcc.make_adapter_desc(0, 1000, 77, n, 8 if n else 0, t))
print("fine")
"""


def test_workspaces_of_no_rows():
    """In a process of its own: a trap of the processor would end this one."""
    r = subprocess.run([sys.executable, "-c", NO_ROWS], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "fine", (r.returncode, r.stderr[-500:])


@pytest.mark.parametrize("t", [wcc.F32, wcc.BF16])
def test_workspaces_are_whole_blocks(t):
    for rows in (0, 1, 5, 64, 65, 511, 5000, 2 ** 31 - 1):
        for width in (1, 63, 640, 5003, 131072, 2 ** 20):
            descs = [(wcc.scores_workspace_bytes, wcc.make_scores_desc(rows, width, min(width, 20), t)),
                     (wcc.distill_workspace_bytes, wcc.make_distill_desc(rows, width, 33, t)),
                     (wcc.adapter_workspace_bytes, wcc.make_adapter_desc(rows, width, 1000, 4, 24, t)),
                     (wcc.adapter_workspace_bytes, wcc.make_adapter_desc(rows, 1000, width, 0, 0, t))]
            for call, d in descs:
                assert call(d) >= 0 and call(d) % 256 == 0


def test_temperatures_whose_factor_overflows_are_refused():
    """log2(e) / temperature is what a logit's difference is multiplied by: infinite, it made the largest logit's 0 NaN."""
    for tau in (1e-45, 2.9e-39, 3e-39, 3.5e-39, 4.2e-39):
        with pytest.raises(wcc.WccError) as e:
            wcc.distill_workspace_bytes(wcc.make_distill_desc(5, 100, 3, wcc.F32, temperature=tau))
        assert e.value.status == 2
    for tau in (4.3e-39, 1e-38, 1.0, 3e38):
        assert wcc.distill_workspace_bytes(wcc.make_distill_desc(5, 100, 3, wcc.F32, temperature=tau)) >= 0
