"""The build's checks on assembly statements (no GPU, no compiler)."""
import pytest

from paper_1712_01537_amd import build

LOAD = ('asm volatile("s_mov_b32 m0, %%0\\n\\tbuffer_load_dwordx4 %%1, %%2, 0 offen lds" ::"s"(lds), '
        '"v"(off),\n               "s"(f(rsrc))\n               : "memory"%s);')


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


def test_every_source():
    assert len(build._sources()) > 10
    build.check_asm()
