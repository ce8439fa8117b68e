"""What the compiler does not see of the kernels of fewer bits, read in the built library: that no result of a matrix instruction of their kinds is
touched early, and that no lane's register is read by another within two wait
states of its writing (additions across lanes are inline assembly)."""
import re

import test_mfma_waits as waits
from test_mfma_waits import listings  # noqa: F401  (the fixture)

KINDS = {"v_mfma_i32_16x16x64_i8": 4}


def early_reads(listing):
    """(kernel, text) of additions across lanes whose source was written by one of the two instructions before."""
    out, name, before = [], None, []
    for line in listing.splitlines():
        m = re.match(r"^[0-9a-f]+ <(.+)>:$", line)
        if m:
            name, before = m.group(1), []
        if not line.startswith("\t"):
            continue
        code = line.split("//")[0].strip()
        op, _, args = code.partition(" ")
        args = [a.strip() for a in args.split(",")]
        if op == "v_fmac_f32_dpp":
            source = waits.regs(args[1])
            if any(source & written for written in before):
                out.append((name, code))
        # (a wait of n counts for n + 1; labels are not instructions, a branch is one)
        n = 1 + int(args[0], 0) if op == "s_nop" else 1
        written = waits.regs(args[0]) if op.startswith("v_") else frozenset()
        before = ([written] + [frozenset()] * (n - 1) + before)[:2] if n == 1 else [frozenset()] * 2
    return out


def test_no_matrix_result_is_touched_early(listings, monkeypatch):  # noqa: F811
    for op, passes in KINDS.items():
        assert sum(t.count(op) for t in listings) > 50
        monkeypatch.setitem(waits.PASSES, op, passes)
    found = sorted(v for t in listings for v in waits.violations(t))
    assert not found, "%d: %s" % (len(found), found[:5])


def test_no_lane_reads_another_early(listings):  # noqa: F811
    assert sum(t.count("v_fmac_f32_dpp") for t in listings) > 100
    found = [v for t in listings for v in early_reads(t)]
    assert not found, "%d: %s" % (len(found), found[:5])


def test_the_check_sees_an_early_read():
    code = ("0000000000001000 <kernel>:\n"
            "\tv_lshlrev_b32_e32 v5, 16, v6 // 000000001000: 00000000\n"
            "%s"
            "\tv_fmac_f32_dpp v3, v5, v4 quad_perm:[1,1,1,1] row_mask:0xf bank_mask:0xf // 000000001008: 00000000\n")
    assert early_reads(code % "") and early_reads(code % "\tv_mov_b32_e32 v9, v8 // 000000001004: 00000000\n")
    assert not early_reads(code % "\ts_nop 1 // 000000001004: 00000000\n")
    assert not early_reads(code % ("\tv_mov_b32_e32 v9, v8 // 000000001004: 00000000\n" * 2))


def test_units_have_the_wavefronts_that_plans_give(listings):  # noqa: F811
    from paper_2411_16102_amd import binding, workloads as W
    from stream_cases import make_batch
    layer, given = binding.Layer(W.LLAMA3_8B, device=-1), set()
    for n, tokens in ((400, 100), (200, 60), (300, 1000), (128, 4000)):
        given |= {layer.window_plan(make_batch([(1, tokens)] * n), 1 << 20, cache=binding.Kv4(g)).division().waves for g in (32, 64, 128)}
    built = {int(m) for t in listings for m in re.findall(r"<_ZN\S*window_unit4_kernelILi\d+ELi\d+ELi\d+ELi(\d+)E\S*>:", t)}
    assert built == given == {1, 2, 4}
