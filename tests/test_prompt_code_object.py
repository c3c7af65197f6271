"""Properties of the compiled kernels of prompts and chunks that results do not show."""
import re

from paper_2508_08256_amd import binding as B
from test_code_object import _code_objects, _kernels


def _prompt_kernels():
    return [k for o in _code_objects(B.LIB_PATH) for k in _kernels(o) if "prompt_attn_kernel" in k[".name"]]


def test_three_workgroups_of_the_attention_fit_a_cu():
    """The rows of K and V are cut into as many parts as 256 CUs hold workgroups of four wavefronts three at a time: 512
    registers per SIMD lane, given out in eights, and 160 KiB of LDS."""
    found = _prompt_kernels()
    assert len({re.search(r"ILi(\d)ELb(\d)E", k[".name"]).groups() for k in found}) == 4  # type, cache
    for k in found:
        registers = -(-(k[".vgpr_count"]) // 8) * 8
        assert 512 // registers >= 3 and 160 * 1024 // k[".group_segment_fixed_size"] >= 3, k
        assert not k.get(".agpr_count"), k  # accumulators stay in the registers that the softmax works on
        assert k[".private_segment_fixed_size"] == 0, k


def test_block_tables_of_the_largest_batch_fit_the_lds():
    found = [k for o in _code_objects(B.LIB_PATH) for k in _kernels(o) if "block_table_kernel" in k[".name"]]
    assert len(found) == 1 and found[0][".group_segment_fixed_size"] + 4 * 16384 <= 160 * 1024
