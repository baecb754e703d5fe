"""What the compiler reports of the registers of the model side's kernels.  Attention keeps a row block's queries, outputs and the keys and values
under way in registers: one that went to memory would be read from there for every key.  Only the wavefronts of 48 rows over 128 columns
of 8 bits are wider than their registers (they are kept for what they convert once instead of twice)."""
import os

import pytest

from test_kernel_resources import HIPCC, _report

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="no compiler")


@pytest.mark.parametrize("source, kernels, wide", [
    ("attention.hip", 3, None), ("attention_bf16.hip", 14, None), ("attention_bf16_f8.hip", 18, "Li128ELi3E"), ("rope.hip", 5, None),
    ("kv_cache.hip", 12, None),
])
def test_nothing_is_spilled(source, kernels, wide, tmp_path):
    report = _report(source, tmp_path)
    assert len(report) == kernels
    spilled = [n for n, k in report.items() if k["VGPRs"] > 0]
    assert all(wide is not None and wide in n for n in spilled), spilled
