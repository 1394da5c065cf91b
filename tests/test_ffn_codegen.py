"""Generated-code checks of the expert feed-forward kernels (CPU: hipcc
cross-compiles), as of the training losses' kernels: slice loops do not spill,
the inline LDS reads land before their registers are used, the large tiles'
accumulators are not touched before their MFMAs have finished, and no copy into
LDS sits in a loop over distinct lane values."""
import re

import pytest

from test_gemm_codegen import (_compile, _function, _hazards, _lds_races, _loops_with_mfma,
                               pytestmark)  # noqa: F401

SOURCES = {
    "expert_ffn.hip": ["k_expert_up", "k_expert_rows", "k_expert_dact", "k_expert_weights"],
    "expert_ffn_f32.hip": ["k_expert_up_f32", "k_expert_rows_f32", "k_expert_dact_f32",
                           "k_expert_weights_f32"],
}


@pytest.fixture(scope="module", params=list(SOURCES))
def kernels(request, tmp_path_factory):
    text = _compile(tmp_path_factory, request.param)
    found = {}
    for kernel in SOURCES[request.param]:
        names = re.findall(r"^(_ZN7trimmoe\w*?\d%s(?:I\w*|E\w*)):" % kernel, text, re.M)
        assert names, kernel
        found.update({n: (kernel, _function(text, n, remarks=False)) for n in names})
    return found


def test_slice_loops_do_not_spill(kernels):
    for name, (_, body) in kernels.items():
        loops = _loops_with_mfma(body)
        assert loops and any(b.startswith("v_mfma") for b in body), name
        for s, e in loops:
            assert not [b for b in body[s:e] if b.startswith("scratch_")], name


def test_accumulators_are_not_touched_early(kernels):
    for name, (kernel, body) in kernels.items():
        if "BigCore" in name:  # (MFMAs in inline asm)
            assert not _hazards(body), (name, _hazards(body)[:2])


def test_lds_reads_land_before_their_registers_are_used(kernels):
    for name, (kernel, body) in kernels.items():
        assert not _lds_races(body), (name, _lds_races(body)[:2])


def test_no_copy_into_lds_waits_for_one_lane_at_a_time(kernels):
    for name, (kernel, body) in kernels.items():
        for i, b in enumerate(body):
            if b.startswith("buffer_load") and b.endswith("lds"):
                assert not any(x.startswith("s_cbranch_execnz") for x in body[i:i + 4]), (name, b)


def _registers(operand):
    m = re.match(r"v\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.match(r"v(\d+)$", operand)
    return {int(m.group(1))} if m else set()


def _store_hazards(body):
    """16-byte buffer stores with a scalar offset register whose data registers the next
    instruction writes: the compiler takes such a pair as safe, and it is not."""
    bad = []
    for store, after in zip(body, body[1:]):
        m = re.match(r"buffer_store_dwordx[34] (\S+), \S+, s\[\S+\], s\d+", store)
        if not m or not after.startswith("v_"):
            continue
        operands = [x.strip() for x in after.split(None, 1)[1].split(",")]
        written = _registers(operands[0]) | (_registers(operands[1]) if "swap" in after else set())
        if written & _registers(m.group(1)):
            bad.append((store, after))
    return bad


def test_the_hazard_check_finds_one():
    pair = ["buffer_store_dwordx4 v[76:79], v60, s[8:11], s13 offen", "v_add_u32_e32 v76, s6, v156"]
    assert _store_hazards(pair)
    assert not _store_hazards([pair[0], "s_nop 0", pair[1]])
    assert not _store_hazards([pair[0], "v_add_u32_e32 v75, s6, v76"])
    assert not _store_hazards([pair[0].replace("s13", "0"), pair[1]])


@pytest.mark.parametrize("source", ["expert_ffn.hip", "head_loss.hip", "gemm.hip"])
def test_stored_registers_are_not_written_at_once(source, tmp_path_factory):
    text = _compile(tmp_path_factory, source)
    body = [x.split(";")[0].strip() for x in text.splitlines()]
    assert any(x.startswith("buffer_store") for x in body)
    assert not _store_hazards([x for x in body if x])
