"""Loads in inline asm must not read a scalar register right after a vector instruction wrote it (paper_2410_12513_amd/asm_check.py): the part asks for
five wait states, which the compiler keeps for its own instructions only.  A check of the library's own assembly, on the CPU."""
from paper_2410_12513_amd import asm_check


def test_scan_finds_a_descriptor_that_is_read_too_early():
    text = """
_ZN5first11k_lora_tileINS_4bf16ELi256EEEvNS_8LoraArgsE:
	v_readlane_b32 s11, v221, 12
	s_mov_b32 m0, s20
	;;#ASMSTART
	s_nop 0
	buffer_load_dwordx4 v2, s[8:11], s7 offen lds
	;;#ASMEND
	s_endpgm
"""
    hits = asm_check.scalars_read_too_early(text)
    assert len(hits) == 1 and "v_readlane" in hits[0][3]
    assert not asm_check.scalars_read_too_early(text.replace("s_nop 0", "s_nop 4"))
    assert not asm_check.scalars_read_too_early(text.replace("s11, v221", "s12, v221"))                   # another register
    offset = text.replace("v_readlane_b32 s11, v221, 12", "v_readfirstlane_b32 s7, v3")
    assert len(asm_check.scalars_read_too_early(offset)) == 1
    managed = text.replace("\t;;#ASMSTART\n", "").replace("\t;;#ASMEND\n", "")
    assert not asm_check.scalars_read_too_early(managed)                                                  # the compiler's own


def test_no_load_of_the_library_reads_a_scalar_too_early():
    asm = asm_check.assembly()
    assert all(n >= 1 for n in asm_check.kernels_seen(asm).values())
    hits = asm_check.scalars_read_too_early(asm)
    assert not hits, hits[:5]
