"""The build's static checks of the kernels whose stages differ from the level kernel's (host logic, no GPU)."""
import pytest

from paper_1904_07421_amd import build as B

MFMA = "\tv_mfma_f32_32x32x16_bf16 v[20:35], v[10:13], v[10:13], v[20:35]\n"


def _walk(loads: int, wait: int, extra: str = "", barriers: int = 1) -> str:
    tile = "\tglobal_load_lds_dwordx4 v1, s[2:3]\n" * (loads - 1) + "\tglobal_load_lds_dword v1, s[2:3]\n" + MFMA
    return ("_ZN5jitdb15resident_kernelILi1ELi8ELi0EEEvNS_7ResArgsE:\n"
            "\tglobal_load_dwordx4 v[40:43], v[2:3], off\n"
            ".LBB0_1:\n" + (tile + extra + f"\ts_waitcnt vmcnt({wait}) lgkmcnt(0)\n\ts_barrier\n") * barriers +
            "\ts_cbranch_scc1 .LBB0_1\n\ts_endpgm\n")


def test_a_wait_for_as_many_loads_as_a_tile_has_passes():
    assert B.check_walk_loads(_walk(5, 5), "resident_kernel") == 1
    assert B.check_walk_loads(_walk(5, 5, barriers=2), "resident_kernel") == 1
    assert B.check_walk_loads(_walk(5, 5, extra="\tglobal_store_dwordx4 v[0:1], v[20:23], off\n"), "resident_kernel") == 1
    assert B.check_walk_loads(_walk(5, 5), "wide_kernel") == 0


@pytest.mark.parametrize("code", [_walk(5, 6), _walk(6, 5, barriers=2)])
def test_another_number_of_loads_is_refused(code):
    with pytest.raises(RuntimeError, match="in flight"):
        B.check_walk_loads(code, "resident_kernel")


def test_another_load_in_the_walk_is_refused():
    with pytest.raises(RuntimeError, match="besides the tiles"):
        B.check_walk_loads(_walk(5, 5, extra="\tglobal_load_dword v40, v[2:3], off\n"), "resident_kernel")


def test_the_number_of_stage_loads_may_be_given():
    loop = ("_ZN5jitdb19grad_product_kernelILi4EEEv:\n.LBB0_1:\n" + ("\tglobal_load_lds_dwordx4 v1, s[2:3]\n" + MFMA) * 4 +
            "\ts_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier\n\ts_cbranch_scc1 .LBB0_1\n\ts_endpgm\n")
    assert B.check_stage_loads(loop, "grad_product_kernel", 4) == 1
    with pytest.raises(RuntimeError, match="assume 6 per stage"):
        B.check_stage_loads(loop, "grad_product_kernel", 6)
