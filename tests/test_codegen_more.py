"""Generated code of the 4-bit cache, rotary positions and a step's rows and pages (no GPU needed): no scratch memory, no packed fp32 instruction."""
import os
import re
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2604_24432_amd import build as B
from tests.test_codegen import _assembly, _kernels

# source: kernel -> instantiations
KERNELS = {"ksa_paged_fp4.hip": {"ksa_paged_few_fp4_kernel": 6, "ksa_paged_many_kernel": 6},
           "ksa_paged_cache_fp4.hip": {"ksa_paged_append_kernel": 2, "ksa_paged_read_kernel": 2},
           "ksa_rotary.hip": {"ksa_rotary_kernel": 12}, "ksa_paged_rotary.hip": {"ksa_paged_rotary_kernel": 18},
           "ksa_paged_advance.hip": {"ksa_advance_count_kernel": 1, "ksa_advance_free_kernel": 1, "ksa_advance_take_kernel": 1, "ksa_advance_rows_kernel": 1}}


@pytest.fixture(scope="module")
def assembly():
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    with tempfile.TemporaryDirectory() as d, ThreadPoolExecutor(3) as pool:
        return dict(zip(KERNELS, pool.map(lambda s: _assembly(s, d), KERNELS)))


@pytest.mark.parametrize("source", KERNELS)
def test_no_scratch_memory(assembly, source):
    seen = dict.fromkeys(KERNELS[source], 0)
    for name, blocks in _kernels(assembly[source]).items():
        kernel = next((k for k in seen if k in name), None)
        assert kernel, name
        seen[kernel] += 1
        assert not [i for ins in blocks.values() for i in ins if i.startswith(("scratch_", "buffer_"))], name
    assert seen == KERNELS[source]
    sizes = re.findall(r"\.private_segment_fixed_size:\s*(\d+)", assembly[source])
    assert len(sizes) == sum(KERNELS[source].values()) and set(sizes) == {"0"}


@pytest.mark.parametrize("source", KERNELS)
def test_no_packed_fp32_instructions(assembly, source):
    assert not re.findall(r"\bv_pk_(?:add|mul|fma)_f32\b", assembly[source])


def test_the_conversions_are_the_hardware_s(assembly):
    assert "v_cvt_scalef32_pk_bf16_fp4" in assembly["ksa_paged_fp4.hip"] and "v_cvt_scalef32_pk_fp4_bf16" in assembly["ksa_paged_cache_fp4.hip"]
