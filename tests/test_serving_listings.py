"""What the listings of the packed and cache kernels show: products in inline assembly are waited for, no row address
sits in a scalar offset, matrix kernels keep their registers (fp32 ones of head_dim 128 apart), and two workgroups of the
decoding kernel fit a CU."""
import re

import pytest

from tests.asm_listing import BF16, F64, functions, kernel_resources, listing, product_hazards, scalar_offset_accesses

SOURCES = ["packed_fwd_bf16.hip", "packed_q_sums.hip", "packed_bwd_dq.hip", "packed_bwd_dkdv.hip", "packed_fwd_f32.hip", "packed_bwd_f32.hip",
           "prefix_bf16.hip", "prefix_f32.hip"]


def text_of(src):
    text = listing(src)
    if text is None:
        pytest.skip("hipcc not available")
    return text


@pytest.mark.parametrize("src,product,file,n", [("packed_fwd_f32.hip", F64, "v", 2), ("packed_bwd_f32.hip", F64, "v", 4),
                                                ("prefix_f32.hip", F64, "v", 2), ("packed_bwd_dkdv.hip", BF16, "a", 4)])
def test_products_are_waited_for(src, product, file, n):
    kernels = {name: b for name, b in functions(text_of(src)).items()
               if any(op == product and ops[0].startswith(file) for _, _, op, ops in b)}
    assert len(kernels) == n, sorted(kernels)
    bad = {name: product_hazards(b, product, file) for name, b in kernels.items()}
    assert not any(bad.values()), bad


@pytest.mark.parametrize("src", ["packed_fwd_f32.hip", "packed_bwd_f32.hip"])
def test_no_row_address_in_a_scalar_offset(src):
    found = {n: scalar_offset_accesses(b) for n, b in functions(text_of(src)).items()}
    assert sum(n for n, _ in found.values()) > 0
    assert not any(lines for _, lines in found.values()), {n: x[1] for n, x in found.items() if x[1]}


@pytest.mark.parametrize("src", [s for s in SOURCES if "f32" not in s])
def test_nothing_is_spilled(src):
    for name, r in kernel_resources(text_of(src)).items():
        assert r["vgpr_spill_count"] == 0 and r["sgpr_spill_count"] == 0 and r["private_segment_fixed_size"] == 0, (name, r)


def test_two_workgroups_of_the_decoding_kernel_fit_a_cu():
    seen = 0
    for name, r in kernel_resources(text_of("prefix_bf16.hip")).items():
        if re.search("prefix_bf16_kernel", name):
            assert 2 * r["group_segment_fixed_size"] <= 160 * 1024 and r["vgpr_count"] <= 256, (name, r)
            seen += 1
    assert seen == 4
