"""What the compiler makes of the kernels of the paged cache's further calls, read from the assembly that it writes for them: no GPU is needed."""

import re

import pytest

import test_paged_resources as paged
from test_kernel_resources import _assembly

SOURCES = ("paged_norm.hip", "paged_evict.hip", "paged_weigh.hip", "paged_prefix.hip")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    return {s: _assembly(s, tmp_path_factory.mktemp(s)) for s in SOURCES}


def test_no_kernel_spills(assembly):
    kernels = {n: k for text in assembly.values() for n, k in paged._kernels(text).items()}
    assert len(kernels) == 8 + (3 + 1 + 2) + (48 + 2) + (24 + 8 + 5)
    assert not any(k["private_segment_fixed_size"] for k in kernels.values()), [n for n, k in kernels.items() if k["private_segment_fixed_size"]]


def _resident(k):
    """Workgroups on a compute unit by 512 registers per lane and SIMD, given out by the eight, and 160 KB of LDS; a workgroup has a wavefront on each SIMD."""
    lds = k["group_segment_fixed_size"]
    return min(512 // -(-k["next_free_vgpr"] // 8 * 8), 160 * 1024 // lds if lds else 8)


@pytest.mark.parametrize("source,count", [("paged_weigh.hip", 48), ("paged_prefix.hip", 32)])
def test_as_many_workgroups_reside_as_the_shared_runs_are_cut_for(assembly, source, count):
    # the same rule as in the source; the kernels with common prefixes plan for as many of both kinds, and fp32 heads of more than 160 elements for one
    seen = 0
    for name, k in paged._kernels(assembly[source]).items():
        m = re.search(r"decode_paged_kernelILb([01])ELi(\d+)ELi(\d+)ELb([01])E", name)
        if not m:
            continue
        bf16, dim, shared = m[1] == "1", 16 * int(m[2]), m[4] == "1"
        assert int(m[3]) == (32 if bf16 and dim <= (128 if shared else 64) else 16)
        planned = 3 if dim <= 64 or (bf16 and dim <= 128 and not shared) else 2 if bf16 or dim <= 160 else 1
        if source == "paged_prefix.hip":
            planned = min(planned, 2)
        assert _resident(k) >= planned, (name, k["next_free_vgpr"], k["group_segment_fixed_size"])
        seen += 1
    assert seen == count


@pytest.mark.parametrize("source", ["paged_weigh.hip", "paged_prefix.hip"])
def test_matrix_results_are_waited_for_on_every_path(assembly, source):
    paged.test_matrix_results_are_waited_for_on_every_path(assembly, source, "decode_paged_kernel", 1000)


def test_vector_pipe_has_no_packed_fp32(assembly):
    for source, text in assembly.items():
        assert not re.search(r"\tv_pk_(add|mul|fma)_f32", text), source
