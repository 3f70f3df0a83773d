"""The build's checks on assembly statements (no GPU, no compiler)."""
import pytest

from paper_1712_01537_amd import build

LOAD = ('asm volatile("s_mov_b32 m0, %%0\\n\\ts_nop 0\\n\\tbuffer_load_dwordx4 %%1, %%2, 0 offen lds" '
        '::"s"(lds), "v"(off),\n               "s"(f(rsrc))\n               : "memory"%s);')


@pytest.mark.parametrize("text,word", [
    ("", ""),
    (LOAD % ', "m0"', ""),
    (LOAD % "", "m0"),
    (LOAD % ', "m0"' + LOAD % "", "m0"),
    ('asm volatile("s_waitcnt vmcnt(0)" ::: "memory");', ""),
    ('// m0 is written here\nconst int64_t m0 = 3;', ""),
])
def test_m0_is_declared(text, word):
    why = build.asm_fault(text)
    assert bool(why) == bool(word) and word in why


@pytest.mark.parametrize("load", ["buffer_load_dwordx4 %1, %2, 0 offen lds",
                                  "global_load_lds_dword %1, off"])
def test_a_wait_state_behind_m0(load):
    text = 'asm volatile("s_mov_b32 m0, %0\\n\\t" "' + load + '" ::"s"(a), "v"(b) : "m0");'
    assert "right behind" in build.asm_fault(text)
    assert build.asm_fault(text.replace('\\n\\t" "', '\\n\\ts_nop 0\\n\\t"\n"')) == ""
    assert build.asm_fault('asm("s_mov_b32 m0, %0\\n\\tv_mov_b32 %1, 0" ::"s"(a) : "m0");') == ""


def test_every_source():
    assert len(build._sources()) > 10
    build.check_asm()
