"""The build's check of the kernels over the 4-bit cache: the whole of a loop that holds matrix instructions counts, from its label to
its branch back."""
import pytest

SCRATCH, ASM = "\tscratch_load_dword v1, off, off", "\t;;#ASMSTART\n\tv_and_or_b32 v1, v2, s0, v3\n\t;;#ASMEND"
KERNEL = """_ZN4sage18cache4_attn_kernelILi{n}E:
{before}
.LBB{n}_1:
{head}
\ts_cbranch_vccnz .LBB{n}_3
\tv_mfma_f32_16x16x32_f16 a
\tv_add_f32 v0, v1, v2
\tv_mfma_f32_16x16x32_f16 b
.LBB{n}_3:
{tail}
\ts_cbranch_scc1 .LBB{n}_1
{behind}
.LBB{n}_4:
\tds_read_b32 v0, v1
{other}
\ts_branch .LBB{n}_4
\ts_endpgm
.Lfunc_end{n}:
"""


def kernel(n, **parts):
    return KERNEL.format(n=n, **{name: parts.get(name, "\ts_nop 0") for name in ("before", "head", "tail", "behind", "other")})


@pytest.mark.parametrize("what", [SCRATCH, ASM])
def test_a_loops_head_and_tail_count(what):
    from paper_2410_02367_amd.build import check_cache4_attn_asm
    assert check_cache4_attn_asm(kernel(0)) == []
    for place in ("head", "tail"):
        problems = check_cache4_attn_asm(kernel(0) + kernel(1, **{place: what}))
        assert len(problems) == 1 and "ILi1E" in problems[0], place


@pytest.mark.parametrize("what", [SCRATCH, ASM])
def test_what_stands_outside_of_the_loop_does_not(what):
    from paper_2410_02367_amd.build import check_cache4_attn_asm
    for place in ("before", "behind", "other"):
        assert check_cache4_attn_asm(kernel(0, **{place: what})) == [], place


def test_nested_loops_and_loops_with_several_ways_back():
    from paper_2410_02367_amd.build import _loops, check_cache4_attn_asm
    lines = [".LBB0_1:", ".LBB0_2:", "\tv_mfma a", "\ts_cbranch_scc1 .LBB0_2", "\ts_cbranch_vccz .LBB0_1", SCRATCH, "\ts_branch .LBB0_1", "\ts_branch .LBB0_9"]
    assert _loops(lines) == [(0, 6), (1, 3)]
    assert len(check_cache4_attn_asm("_ZN4sage1kE:\n" + "\n".join(lines) + "\n.Lfunc_end0:\n")) == 1
