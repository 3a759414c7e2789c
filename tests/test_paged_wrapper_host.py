"""paged.py's refusals that need no GPU: configurations come back as the library's own errors."""
import pytest

from paper_2504_10724_amd import capi as ee
from paper_2504_10724_amd import paged as P


@pytest.mark.parametrize("head_dim", [0, -64, 100, 2 ** 31 - 1])
def test_caches_of_no_such_width(head_dim):
    with pytest.raises(ee.EEError):
        P.PagedCache(1, 4, 2, head_dim, 32)


@pytest.mark.parametrize("kw", [dict(head_dim=0), dict(head_dim=64, rot_dim=63), dict(head_dim=64, theta=0.5), dict(head_dim=64, pairing="both")])
def test_tables_of_no_such_kind(kw):
    with pytest.raises(ee.EEError):
        P.Rope(max_pos=100, **kw)
