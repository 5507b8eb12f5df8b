"""Rings that bulk copies refill: how their readers give a stage back, read from the sources (the fault itself shows in one
call of a million)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_04902_b200", "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as fh:
        return re.sub(r"//[^\n]*", "", fh.read())


def test_the_release_fences_first():
    body = re.search(r"void release_stage\(uint64_t\* empty\) \{(.*?)\n\}", _code("tma_pipeline.cuh"), re.S).group(1)
    steps = [body.index(s) for s in ("fence_async_smem();", "__syncwarp();", "mbar_arrive(empty);")]
    assert steps == sorted(steps)


@pytest.mark.parametrize("name", ["glu_few.cuh", "distill.cu", "vote_median_tma.cu", "vote_pairdist_kernel.cuh", "pairdist_i8_kernel.cuh", "probe.cu"])
def test_readers_release_through_it(name):
    code = _code(name)
    assert not re.search(r"mbar_arrive\(&(in_)?empty", code) and re.search(r"release_stage\(&(in_)?empty", code)
