"""Machine-code checks of the int8 product kernels, whose global->LDS requests are
inline assembly like those of the bf16 kernels (host only: compiled to gfx950
assembly with the library's options, nothing runs): the requests are there, no SCC
value of compiler code lives across one, M0 is theirs alone and read a wait state
after its write, nothing spills."""
import os
import re
import shutil

import pytest

import test_isa_inline_asm as base

# source, kernel name, instantiations, requests of the smallest one (the prologue's and the loop's tiles)
KERNELS = {"gemm_int8_wide": ("gemm_int8_wide.hip", "gemm_int8_wide_kernel", 2, 32),
           "gemm_int8_ring": ("gemm_int8_ring.hip", "gemm_int8_ring_kernel", 6, 6),
           "gemm_int8": ("gemm_int8.hip", "gemm_int8_kernel", 14, 12)}


@pytest.fixture(scope="module", params=sorted(KERNELS))
def kernels(request, tmp_path_factory):
    """Assembly lines of every instantiation of a kernel, as the library is compiled."""
    if not shutil.which(base.HIPCC) and not os.path.exists(base.HIPCC):
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("isa") / (request.param + ".s")
    patch = pytest.MonkeyPatch()
    patch.setattr(base, "KERNELS", KERNELS)
    try:
        found = base._instantiations(request.param, out)
    finally:
        patch.undo()
    assert len(found) == KERNELS[request.param][2], sorted(found)
    spills = re.findall(r"\.vgpr_spill_count:\s+(\d+)", out.read_text())
    assert len(spills) == len(found) and not any(map(int, spills))
    return found, KERNELS[request.param][3]


def test_requests_present(kernels):
    base.test_requests_present(kernels)


def test_no_compiler_scc_value_across_a_request(kernels):
    base.test_no_compiler_scc_value_across_a_request(kernels)


def test_wait_state_between_m0_write_and_lds_load(kernels):
    base.test_wait_state_between_m0_write_and_lds_load(kernels)


def test_m0_is_written_by_the_requests_alone(kernels):
    base.test_m0_is_written_by_the_requests_alone(kernels)


def test_products_are_the_i8_instruction(kernels):
    for name, asm in kernels[0].items():
        assert sum(ln.startswith("v_mfma_i32_16x16x64_i8") for ln in asm) >= 2, name
        assert not any("f32_16x16" in ln for ln in asm), name
