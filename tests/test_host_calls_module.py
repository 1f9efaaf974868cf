"""The compiled side of the binding belongs to one interpreter and one torch: another's is neither taken for up to date nor loaded."""
import os
import sysconfig

import pytest
import torch


def test_module_of_another_torch(monkeypatch):
    from paper_2607_19378_b200 import build as bld
    bld.build()
    from paper_2607_19378_b200 import hyenand as hn
    here = bld.calls_path()
    assert os.path.exists(here) and sysconfig.get_config_var("SOABI") in here
    assert hn._calls.__wrapped__().make_recurrence and bld.build_calls() == here
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert bld.calls_path() != here
    with pytest.raises(OSError, match="build it with"):
        hn._calls.__wrapped__()
