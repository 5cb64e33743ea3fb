"""What the build looks at in the compiled kernels, on assembly of a few lines."""
import pytest

from paper_2412_08521_amd import build

RING = "_ZN3ems13prompt_kernelILi128ELb0ELb0ELi1ELi1ELi2EEEvNS_10PromptArgsE"
BARRIER = RING.replace("ELi2EEE", "ELi1EEE")
FILL = "\tglobal_load_lds_dwordx4 v3, s[2:3] offset:1024"
READ = "\tds_read_b64_tr_b16 v[8:9], v2 offset:64"


def _kernel(*lines, name=RING):
    return "\n".join([f"{name}:                ; @kernel", *lines, "\ts_endpgm", ".Lfunc_end0:", ""])


@pytest.mark.parametrize("lines", [
    (FILL, READ),
    (READ, "\ts_waitcnt lgkmcnt(0)", FILL),
    (READ, "\ts_waitcnt vmcnt(0) lgkmcnt(0)", FILL),
    (READ, "\tds_read_b32 v1, v2", "\ts_waitcnt lgkmcnt(1)", FILL),
    (READ, "\tglobal_load_lds_dword v3, off"),                                    # (of a table, to a place of its own)
    (FILL, ".LBB0_1:", READ, "\ts_waitcnt lgkmcnt(0)", FILL, "\ts_cbranch_scc1 .LBB0_1"),
    (READ, "\ts_branch .LBB0_2", ".LBB0_1:", FILL, "\ts_endpgm", ".LBB0_2:", "\ts_nop 0"),
])
def test_dma_after_reads_is_taken(lines):
    build._check_reads_before_dma("prompt.hip", _kernel(*lines))


@pytest.mark.parametrize("lines", [
    (READ, FILL),
    (READ, "\ts_waitcnt vmcnt(0)", FILL),
    (READ, "\ts_waitcnt lgkmcnt(1)", FILL),
    (READ, "\tds_read_b32 v1, v2", "\ts_waitcnt lgkmcnt(2)", FILL),
    ("\ts_waitcnt lgkmcnt(0)", ".LBB0_1:", FILL, READ, "\ts_cbranch_scc1 .LBB0_1"),        # the next turn's
    (READ, "\ts_cbranch_scc1 .LBB0_2", "\ts_waitcnt lgkmcnt(0)", ".LBB0_2:", FILL),        # one way of two
    (READ, "\ts_branch .LBB0_2", ".LBB0_1:", "\ts_endpgm", ".LBB0_2:", FILL),
])
def test_dma_beside_reads_is_refused(lines):
    with pytest.raises(RuntimeError, match="while a read of it may be under way"):
        build._check_reads_before_dma("prompt.hip", _kernel(*lines))
    with pytest.raises(RuntimeError, match="no kernel with rings"):                # kernels whose waves share one have barriers
        build._check_reads_before_dma("prompt.hip", _kernel(*lines, name=BARRIER))
