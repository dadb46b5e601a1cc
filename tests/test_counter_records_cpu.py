"""The committed counter records stay valid when calls change that none of their
kernels belongs to."""
import glob
import json
import os
import re

import pytest

import bench

RECORDS = sorted(glob.glob(os.path.join(bench.PROFILES, "*_counters.json")))
LAYER = {"norm.hip", "dropout.hip", "rotate.hip", "project.hip", "philox.h", "lanes.h", "layer.h"}


def _text(fn):
    with open(os.path.join(bench.CSRC, fn)) as f:
        return f.read()


def _includes(fn):
    out = {fn}
    for inc in re.findall(r'#include "(\w+\.h)"', _text(fn)):
        out |= _includes(inc)
    return out


@pytest.mark.parametrize("path", RECORDS, ids=os.path.basename)
def test_records_do_not_depend_on_the_layer_calls(path):
    """Neither the shared header, which every record hashes, nor a source that a record hashes declares or includes
    what the norm, dropout, rotary positions and projections need."""
    with open(path) as f:
        kernels = json.load(f)["kernels"]
    files = bench._kernel_files()
    hashed = {files[bench._base_name(k)] for k in kernels if bench._base_name(k) in files} | {"snls_internal.h"}
    assert len(hashed) > 1
    for fn in hashed:
        assert not _includes(fn) & LAYER, fn
        assert not re.search(r"snls_(norm|rotate|project|dropout)|launch_(norm|rotate|project|dropout)|struct Drop\b", _text(fn)), fn
