"""The sources that date bench.py's counter summaries: all that the layers' kernels are built
from, and none of the training calls' (CPU only)."""
import os
import re

import bench
from paper_1903_01521_amd import build


def _names():
    return {os.path.basename(f) for f in bench.layer_sources()}


def test_training_sources_do_not_date_the_layers_counters():
    mine = {os.path.basename(f) for f in build.SOURCES + build.HEADERS} - {"wino.h"}
    left = mine - _names()
    assert left and all(n.startswith(bench.TRAINING_SOURCES) for n in left)
    assert _names() < mine


def test_no_layer_source_includes_one_left_out():
    for f in bench.layer_sources():
        for inc in re.findall(r'#include "([^"]+)"', open(f).read()):
            assert os.path.basename(inc) in _names() | {"wino.h"}, (f, inc)
