"""Build ids (CPU only): every source's id covers the files that it includes, and the
attention's and the composition's ids, which profiled figures in the bench line are
tied to, cover no declaration of other operators."""
import os
import re

import pytest

from paper_2607_15650_amd import build

ALWAYS = {"internal.h", "per_device.h"}


def included(name, seen):
    for x in re.findall(r'^#include "([^"]+)"', open(os.path.join(build.CSRC, name)).read(), re.M):
        if x not in seen and os.path.exists(os.path.join(build.CSRC, x)):
            seen.add(x)
            included(x, seen)
    return seen


@pytest.mark.parametrize("name", build.SOURCES)
def test_ids_cover_what_is_included(name):
    assert included(name, set()) | ALWAYS == set(build.INCLUDES.get(name, [])) | ALWAYS


@pytest.mark.parametrize("name", ["attn_bf16.hip", "attn_bf16_any_q.hip", "merge.hip", "norms.hip"])
def test_other_operators_stay_out(name):
    files = included(name, set()) | ALWAYS
    assert not files & {"layer.h", "kernel_lds.h", "wide_range.h", "cross_tile.h"}
    text = "".join(open(os.path.join(build.CSRC, f)).read() for f in files if f.endswith(".h"))
    assert "CrossArgs" not in text and "RotaryArgs" not in text


def test_profiled_traffic_is_this_builds():
    """The bench line reports the profiled bytes only for the build that they were
    taken on: a change of these sources takes a new profile."""
    import bench
    assert build.source_id("attn_bf16.hip") == bench.ATTN_TRAFFIC["build_id"]
    assert build.source_id("merge.hip") == bench.MERGE_TRAFFIC["build_id"]
