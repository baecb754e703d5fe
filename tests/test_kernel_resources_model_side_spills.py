"""What the kernels of all sources of the model side keep in memory for want of registers: these and no more.

Vector registers: attention's wavefronts of 48 rows over 128 columns of 8 bits (70 of them where pages hold whole tiles, 67 where not), its float32
wavefronts over float32 caches of 129 to 256 columns with pages or widths of other sizes (16), and the draw under warps from bfloat16
logits (10); nothing else.  Scalar registers are kept in lanes of vector registers: up to so many of a source's kernels."""
import os

import pytest

from test_kernel_resources import HIPCC, _report

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="no compiler")


@pytest.mark.parametrize("source, kernels, vector, scalar", [
    ("attention.hip", 3, {}, 0),
    ("attention_bf16.hip", 14, {}, 293),
    ("attention_bf16_f8.hip", 18, {"ILi1ELi2ELi128ELi3ELb1EE": 70, "ILi1ELi2ELi128ELi3ELb0EE": 67}, 611),
    ("attention_f32.hip", 6, {"ILi0ELi0ELi256ELi1ELb0EE": 16}, 789),
    ("attention_f32_f8.hip", 6, {}, 479),
    ("rope.hip", 5, {}, 0),
    ("kv_cache.hip", 12, {}, 2),
    ("sample.hip", 8, {"sample_kernelILi1EE": 10}, 88),
])
def test_what_is_spilled(source, kernels, vector, scalar, tmp_path):
    report = _report(source, tmp_path)
    assert len(report) == kernels
    for name, spilled in report.items():
        allowed = max([n for part, n in vector.items() if part in name], default=0)
        assert spilled["VGPRs"] <= allowed and spilled["SGPRs"] <= scalar, (name, spilled)
