"""Generated code of the paged cache's kernels (no GPU needed): no scratch memory, which a spill of vector registers into the tile loops would take, and
no packed fp32 instruction."""
import os
import re
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2604_24432_amd import build as B
from tests.test_codegen import _assembly, _kernels

# source: kernel -> instantiations
KERNELS = {"ksa_paged.hip": {"ksa_paged_few_kernel": 4, "ksa_paged_many_kernel": 12, "ksa_paged_join_few_kernel": 6, "ksa_paged_join_kernel": 2},
           "ksa_paged_cache.hip": {"ksa_paged_append_kernel": 4, "ksa_paged_read_kernel": 4}}


@pytest.fixture(scope="module")
def assembly():
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    with tempfile.TemporaryDirectory() as d, ThreadPoolExecutor(2) as pool:
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


def test_the_products_are_where_the_check_looks(assembly):
    for name, blocks in _kernels(assembly["ksa_paged.hip"]).items():
        n = sum("v_mfma_f32_32x32x16_bf16" in i for ins in blocks.values() for i in ins)
        assert (n > 0) == ("join" not in name), name
