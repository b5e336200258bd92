"""Static checks of the assembly of the paged-cache kernels (no GPU needed), as in test_kernel_asm.py."""

import re

import pytest

import test_kernel_asm
from test_kernel_asm import _asm, _have_hipcc, _in_flight_violations, _kernels

pytestmark = pytest.mark.skipif(not _have_hipcc(), reason="hipcc not installed")


@pytest.fixture(scope="module", params=["fa_paged_kernel.hip", "fa_paged_fwd_kernel.hip"])
def text(request):
    return _asm(request.param)


def test_no_packed_fp32_no_scratch_no_scalar_writes(text):
    assert not re.findall(r"\bv_pk_(?:add|mul|fma)_f32\b", text)
    sizes = re.findall(r"\.amdhsa_private_segment_fixed_size\s+(\d+)", text)
    assert sizes and all(int(x) == 0 for x in sizes), sizes
    assert not re.findall(r"\bs_(?:store|atomic|buffer_store|dcache_wb|dcache_discard)\w*", text)


def test_buffer_descriptors_in_scalar_registers(text):
    loads = re.findall(r"^\s*(buffer_\w+\s+[^\n]*)$", text, re.M)
    assert loads
    bad = [ln for ln in loads if not re.search(r",\s*s\[\d+:\d+\],\s*[^,]+$", ln)]
    assert not bad, bad[:5]


def test_no_access_to_registers_of_in_flight_loads(text):
    kernels = _kernels(text)
    n = sum(1 for code in kernels.values() for k, t, a in code if a and k == "ins" and re.match(r"global_load", t))
    assert n > 0, "no inline-asm load found: the check would be vacuous"
    report = {name: bad[:5] for name, code in kernels.items() if (bad := _in_flight_violations(code))}
    assert not report, report


def test_inline_asm_mfma_operands_settled():
    test_kernel_asm.test_inline_asm_mfma_operands_settled(_asm("fa_paged_fwd_kernel.hip"))
