"""What the compiler reports of the registers of the calls next to the step: 76 of the scoring gradient's hold a row between
its sums and its gradient, and one that went to memory would be read from there for every vector."""
import os

import pytest

from test_kernel_resources import HIPCC, _report

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="no compiler")


@pytest.mark.parametrize("source, kernels, scalars", [
    # scalar registers that are spilled, and no more: of the alternatives two, of the searches for a piece's tokens six
    ("token_logprobs.hip", 48, {"token_logprobs_kernel": 2}),
    ("embedding.hip", 25, {"embedding_grad_pieces_kernel": 6}),
    ("grad_norm.hip", 4, {}),
])
def test_nothing_is_spilled(source, kernels, scalars, tmp_path):
    report = _report(source, tmp_path)
    assert len(report) == kernels
    for n, k in report.items():
        assert k["VGPRs"] == 0, n
        assert k["SGPRs"] <= max([s for name, s in scalars.items() if name in n], default=0), (n, k)
