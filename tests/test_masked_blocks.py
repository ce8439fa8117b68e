"""Elements of matrix results that are written under several conditions: the compiler has made branches of them, wrote the value ahead of these,
took it back, and left the block empty that should have written it again (see window_device.hpp).  Such a block switches lanes off and
on again with nothing between; this reads the built library, in which there is none."""
import re

from test_mfma_waits import listings  # noqa: F401  (the fixture)


def empty_blocks(listing):
    """(kernel, line) of places where lanes are switched off and on again with nothing between."""
    out, name, before = [], None, ""
    for n, line in enumerate(listing.splitlines()):
        m = re.match(r"^[0-9a-f]+ <(.+)>:$", line)
        if m:
            name, before = m.group(1), ""
        elif line.startswith("\t"):
            code = line.split("//")[0].strip()
            if "saveexec" in before and re.match(r"s_or_b64\s+exec, exec", code):
                out.append((name, n))
            before = code
    return out


def test_no_block_of_masked_lanes_is_empty(listings):  # noqa: F811
    assert sum(t.count("saveexec") for t in listings) > 100
    found = [b for t in listings for b in empty_blocks(t)]
    assert not found, "%d: %s" % (len(found), found[:5])


def test_the_check_sees_an_empty_block():
    code = ("0000000000001000 <kernel>:\n"
            "\ts_and_saveexec_b64 s[0:1], s[8:9] // 000000001000: BE80200A\n"
            "%s"
            "\ts_or_b64 exec, exec, s[0:1] // 000000001004: 87FE007E\n"
            "\ts_endpgm // 000000001008: BF810000\n")
    assert empty_blocks(code % "") == [("kernel", 2)]
    assert not empty_blocks(code % "\tv_mov_b32_e32 v3, s73 // 000000001004: 7E060249\n")
