"""The 8-bit integer products copy rows' codes global memory -> LDS with an instruction the compiler does not see and wait with a count:
"at most N memory operations still in flight".  Operations retire in order, so the copies have landed if exactly N memory instructions
are issued between the last copy and the wait.  Checked on the compiled code (no GPU needed), like the grouped GEMM's."""
import re

from test_gemm_isa_invariants import VMEM, _assembly, _blocks, test_a_wait_state_between_m0_and_the_load_that_reads_it as m0_rule


def test_counted_waits_cover_the_copies():
    lines = _assembly("int8_gemm.hip")
    blocks = _blocks(lines)
    in_asm = {k for b in blocks for k in range(b[0], b[1] + 1)}
    counted = everything = 0
    for b in blocks:
        m = re.search(r"s_waitcnt vmcnt\((\d+)\)", b[2])
        if not m:
            continue
        n = int(m.group(1))
        if n == 0:
            everything += 1
            continue
        issued, k = 0, b[0] - 1
        while not (k in in_asm and "global_load_lds_dwordx4" in lines[k]):
            text = lines[k].strip()
            assert not re.match(r"^\.LBB\d+_\d+:", text) and not re.match(r"s_c?branch", text), "the wait at line %d: control flow behind its copies" % b[0]
            assert not text.startswith("scratch_"), "spilled registers among the loads"
            issued += k not in in_asm and bool(VMEM.match(text))
            k -= 1
        assert issued == n, "the wait at line %d allows %d operations, %d are issued behind the copies" % (b[0], n, issued)
        counted += 1
    # four fragment counts: two shapes of the plain product, two of K split, tall tiles of two projections
    assert counted == 24 and everything >= 24
    # a copy reaches no barrier without a wait of either kind
    for b in blocks:
        if "global_load_lds_dwordx4" not in b[2]:
            continue
        k, waited = b[1] + 1, False
        while "s_barrier" not in lines[k]:
            waited |= k in in_asm and "s_waitcnt vmcnt(" in lines[k]
            k += 1
        assert waited, "copy at line %d" % b[0]


def test_no_kernel_spills():
    for name in ("int8_gemm.hip", "int8_rows.hip", "route_scored.hip"):
        text = "\n".join(_assembly(name))
        kernels = re.findall(r"\.name:\s+(_Z\S+)[\s\S]*?\.vgpr_spill_count:\s+(\d+)", text)
        assert len(kernels) > 4
        # (a row of 131072 values of 32 bits holds 128 registers a thread at 1024 threads: the one that may)
        assert [k for k, n in kernels if int(n)] in ([], [k for k, _ in kernels if "quantize_rows_kernelILi1ELi16ELi16E" in k])


def test_products_and_plan_use_no_scratch_memory():
    text = "\n".join(_assembly("int8_gemm.hip"))
    kernels = re.findall(r"\.name:\s+(_Z\S+)\s+\.private_segment_fixed_size:\s+(\d+)", text)
    assert len(kernels) >= 20 and all(n == "0" for _, n in kernels)


def test_a_wait_state_between_m0_and_the_load():
    m0_rule("int8_gemm.hip")
