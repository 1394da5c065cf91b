"""Generated-code checks of the training losses' kernels (CPU: hipcc
cross-compiles), as of the GEMM cores: their slice loops do not
spill, the large-group kernels' accumulators are not touched before the MFMAs
that write them (inline asm, whose latency the compiler does not see) have
finished, LDS reads land before their registers are used, and no copy into LDS
sits in a loop over distinct lane values (a wave-uniform operand that the
compiler took for a lane's own)."""
import re

import pytest

from test_gemm_codegen import (_compile, _function, _hazards, _lds_races, _loops_with_mfma,
                               _mfma_lds_hazards, _part_races, pytestmark)  # noqa: F401

SOURCES = {
    "head_loss.hip": ["k_dz_big", "k_prod_big", "k_dz_mid", "k_dz_few", "k_few_grad", "k_loss_f32", "k_dz_f32"],
    "products.hip": ["k_prod_f32"],
    "gemm.hip": ["k_loss_big", "k_loss_mma"],
    "skinny.hip": ["k_loss_skinny", "k_dz_skinny"],
    "balance.hip": ["k_balance_forward", "k_balance_grad", "k_balance_grad_f32"],
}
LARGE = ("k_dz_big", "k_prod_big", "k_loss_big")  # MFMAs in inline asm


@pytest.fixture(scope="module", params=list(SOURCES))
def kernels(request, tmp_path_factory):
    text = _compile(tmp_path_factory, request.param)
    found = {}
    for kernel in SOURCES[request.param]:
        names = re.findall(r"^(_ZN7trimmoe\w*?\d%s(?:I\w*|E\w*)):" % kernel, text, re.M)
        assert names, kernel
        found.update({n: (kernel, _function(text, n, remarks="skinny" in kernel)) for n in names})
    return found


def test_slice_loops_do_not_spill(kernels):
    for name, (_, body) in kernels.items():
        loops = _loops_with_mfma(body)
        assert any(b.startswith("v_mfma") for b in body), name
        for s, e in loops:
            assert not [b for b in body[s:e] if b.startswith("scratch_")], name


def test_accumulators_are_not_touched_early(kernels):
    for name, (kernel, body) in kernels.items():
        if kernel in LARGE:
            assert not _hazards(body), (name, _hazards(body)[:2])


def test_lds_reads_land_before_their_registers_are_used(kernels):
    for name, (kernel, body) in kernels.items():
        assert not _lds_races(body), (name, _lds_races(body)[:2])


def test_streams_of_w_keep_their_sums_areas_apart(kernels):
    for name, (kernel, body) in kernels.items():
        if "skinny" in kernel:
            assert not _mfma_lds_hazards(body), name
            assert not _part_races(body), name


def test_no_copy_into_lds_waits_for_one_lane_at_a_time(kernels):
    for name, (kernel, body) in kernels.items():
        for i, b in enumerate(body):
            if b.startswith("buffer_load") and b.endswith("lds"):
                assert not any(x.startswith("s_cbranch_execnz") for x in body[i:i + 4]), (name, b)
