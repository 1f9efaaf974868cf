"""Sites of dropouts that do not fit the counter's word are refused, not cut off."""
import pytest


def test_sites():
    from paper_2607_19378_b200.build import build
    build()
    from paper_2607_19378_b200 import hyenand as hn
    for site in (1 << 31, (1 << 32) + 3, -(1 << 31) - 1):
        with pytest.raises(OverflowError):
            hn.Dropout(0.5, site=site)
        with pytest.raises(OverflowError):
            hn.Block((8,), 2, 3, p=0.5, site=site)
    for site in ((1 << 31) - 1, -(1 << 31), 0):
        assert hn.Dropout(0.5, site=site).site == hn.Block((8,), 2, 3, p=0.5, site=site).site == site
