"""Latent calls: what the host refuses (no GPU)."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pask():
    subprocess.run([sys.executable, os.path.join(ROOT, "paper_2608_28276_b200", "build.py"), "--if-stale"], check=True, capture_output=True)
    import paper_2608_28276_b200 as P
    return P


def test_prompt_wait_limits(pask):
    for limit, surplus in ((0, 0), (-1, 0), (99_999, 0), (10 ** 12 + 1, 0), (10 ** 6, 8), (10 ** 6, 65552)):
        with pytest.raises(pask.PaskError) as e:
            pask.pask_debug_set_prompt_wait(limit, surplus)
        assert e.value.status == pask.ERR_INVALID_ARG
    pask.pask_debug_set_prompt_wait(100_000, 65536)
    pask.pask_debug_set_prompt_wait()
