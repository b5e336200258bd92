"""Static checks of the assembly of the kernels around the paged cache and of the attention with forms (no GPU needed), as in
test_paged_asm.py."""

import re

import pytest

import test_kernel_asm
from test_kernel_asm import _asm, _have_hipcc, _in_flight_violations, _kernels
from test_paged_asm import test_buffer_descriptors_in_scalar_registers as descriptors

pytestmark = pytest.mark.skipif(not _have_hipcc(), reason="hipcc not installed")

FORMS = ["fa_paged_forms_few_kernel.hip", "fa_paged_masked_kernel.hip", "fa_paged_capped_kernel.hip", "fa_paged_biased_kernel.hip"]


@pytest.fixture(scope="module", params=FORMS + ["fa_paged_moves_kernel.hip", "fa_rotate_kernel.hip"])
def text(request):
    return request.param, _asm(request.param)


def test_generated_code(text):
    name, asm = text
    assert not re.findall(r"\bv_pk_(?:add|mul|fma)_f32\b", asm)
    assert not re.findall(r"\bs_(?:store|atomic|buffer_store|dcache_wb|dcache_discard)\w*", asm)
    sizes = [int(x) for x in re.findall(r"\.amdhsa_private_segment_fixed_size\s+(\d+)", asm)]
    assert sizes
    if name != "fa_paged_biased_kernel.hip":
        assert all(x == 0 for x in sizes), sizes
    else:
        # Beside the step, slopes leave a few registers too few for what lies around the loop; the steps use none of it: a
        # scratch access there would wait for the tiles that are on their way.
        assert all(x <= 64 for x in sizes), sizes
        steps = [b for b in re.split(r"^\.LBB\d+_\d+:", asm, flags=re.M)
                 if all(x in b for x in ("v_mfma_", "ds_read_b64_tr", "ds_read_b128", "buffer_load_dwordx4"))]
        assert len(steps) >= 2 * len(sizes) and not any("scratch_" in b for b in steps)
    if name not in FORMS:
        return
    descriptors(asm)
    kernels = _kernels(asm)
    n = sum(1 for code in kernels.values() for k, t, a in code if a and k == "ins" and re.match(r"global_load", t))
    assert n > 0, "no inline-asm load found: the check would be vacuous"
    report = {name: bad[:5] for name, code in kernels.items() if (bad := _in_flight_violations(code))}
    assert not report, report
    if name != FORMS[0]:
        test_kernel_asm.test_inline_asm_mfma_operands_settled(asm)
