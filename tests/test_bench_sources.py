"""The bench line's measured traffic belongs to the sources of what it times: those of other operators do not unsettle it.  No GPU is needed."""
import glob
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2207_10741_amd", "csrc")


def _included(path, seen):
    for name in re.findall(r'#include "([^"]+)"', open(path).read()):
        for folder in (os.path.dirname(path), os.path.join(bench.ROOT, "include")):
            found = os.path.join(folder, name)
            if os.path.exists(found) and found not in seen:
                seen.add(found)
                _included(found, seen)
    return {os.path.basename(f) for f in seen}


def test_sources_that_count_are_the_convolutions():
    counted = bench.kernel_sources()
    names = {os.path.basename(f) for f in counted}
    assert {"fc_api.hip", "fc_conv_mfma.hip", "fc_mask.hip", "fc_dma_util.hpp"} <= names
    others = {os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.h*"))} - names
    for f in counted:
        included = _included(f, set())
        assert not included & {"focused_attention.h", "focused_layers.h", "focused_pages.h"}, f     # another operator's source
        assert not included & others, f                                                             # it would have to count


def test_the_traffic_is_of_these_sources():
    bytes_, note = bench.measured_traffic()
    assert bytes_ is not None and bytes_ > 0, note
