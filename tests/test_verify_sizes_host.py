"""Sizes that the verification operators' planning queries take without rows (CPU only)."""
from __future__ import annotations

import subprocess
import sys

import paper_2606_21848_gb300 as kl
from paper_2606_21848_gb300 import builder


def test_no_rows_of_logits():
    # (in a process of its own: a division by zero ends it)
    kl.build()
    code = ("import paper_2606_21848_gb300 as kl; kl.load(); "
            "print([kl.kl_logprobs_workspace_size(0, v, k) for v in (1, 1000, 100000) for k in (0, 5)])")
    r = subprocess.run([sys.executable, "-c", code], cwd=builder.ROOT,
                       capture_output=True, text=True)
    assert r.returncode == 0, r.returncode
    assert r.stdout.strip() == str([0] * 6)
