"""What the binding of the paged cache repeats of include/sync.h."""
import os
import re

from tests.conftest import ROOT


def test_short_tables():
    import paper_2608_13757_gb300 as sg
    with open(os.path.join(ROOT, "include", "sync.h")) as f:
        assert int(re.search(r"^#define SYNC_CACHE_SHORT (\d+)$", f.read(), re.M).group(1)) == sg.cache.SHORT
