"""Sizes and scales that the verification operators take or refuse on the host (CPU only)."""
from __future__ import annotations

import subprocess
import sys

import pytest

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


@pytest.mark.parametrize("scale, fine", [(2.3e38, True), (2.358e38, True), (2.36e38, False), (3.4e38, False),
                                         (1e-45, True), (-1.0, True)])
def test_scales_whose_product_with_log2_e_is_finite(scale, fine):
    kl.build()
    call = lambda: kl.kl_token_logprobs(0, 10, 10, 16, kl.KL_FP32, scale, 16, 1, 0, 16, None, None, None,  # noqa: E731
                                        None, None, 0)
    if fine:
        call()                                        # no rows: nothing to do
    else:
        with pytest.raises(kl.KLError) as e:
            call()
        assert e.value.status == kl.KL_ERR_INVALID_ARG
