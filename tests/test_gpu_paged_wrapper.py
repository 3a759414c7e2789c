"""What paged.py and the calls behind it refuse, and what a refusal leaves behind."""
import pytest
import torch

from paper_2504_10724_amd import capi as ee
from paper_2504_10724_amd import paged as P

pytestmark = pytest.mark.gpu


def test_a_table_that_does_not_fit_leaves_no_error_behind():
    """2 TB are refused, and the next call is answered for itself"""
    print("[case] table too large", flush=True)
    rope = P.Rope(64, 100)
    with pytest.raises(ee.EEError):
        P.Rope(256, 2 ** 31 - 1)
    x = torch.zeros(1, 2, 64, device="cuda")
    assert torch.equal(rope.apply(x, torch.zeros(1, dtype=torch.int32, device="cuda")), x)
