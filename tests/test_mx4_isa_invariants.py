"""The microscaled 4-bit products copy rows' codes and exponents global memory -> LDS with instructions the compiler does not see, a few steps ahead,
and wait with a count: "at most N memory operations still in flight".  Operations retire in order, so the next step's copies have landed if
at least N memory instructions were issued behind them.  Checked on the compiled code (no GPU needed): the loop's body is walked several
times over, every memory instruction taken into a queue."""
import re

from test_gemm_isa_invariants import VMEM, _assembly, _blocks, test_a_wait_state_between_m0_and_the_load_that_reads_it as m0_rule


def _kernels(lines):
    """kernel name -> its lines' numbers"""
    at, name = {}, None
    for i, l in enumerate(lines):
        m = re.match(r"^(_ZN5dymoe15mx4_tall_kernel\S+):", l)
        if m:
            name, start = m.group(1), i
        if name and l.startswith(".Lfunc_end"):
            at[name], name = range(start, i), None
    return at


def _straight(lines, rows):
    """straight-line pieces: between labels and branches"""
    piece = []
    for i in rows:
        t = lines[i].strip()
        if re.match(r"^\.LBB\d+_\d+:", t) or re.match(r"^s_c?branch", t):
            yield piece
            piece = []
        else:
            piece.append(i)
    yield piece


def test_counted_waits_cover_the_copies():
    lines = _assembly("mx4_gemm.hip")
    in_asm = {k for b in _blocks(lines) for k in range(b[0], b[1] + 1)}
    kernels = _kernels(lines)
    assert len(kernels) == 10
    loops = 0
    for name, rows in kernels.items():
        ahead = int(re.search(r"Li(\d+)ELi(\d+)ELb[01]EEEvNS", name).group(1))       # ..., steps ahead, operands ahead, rows in tiles
        for piece in _straight(lines, rows):
            if sum("v_mfma" in lines[i] for i in piece) == 0 or sum("s_barrier" in lines[i] for i in piece) != ahead:
                continue                                                          # (the last steps' pieces hold one each: the same code)
            loops += 1
            # (operation, step that asked) in order; a step's copies are the next but ahead - 1's
            queue, step, waits = [], 0, 0
            for _ in range(4):
                for i in piece:
                    t = lines[i].strip()
                    if i in in_asm and "global_load_lds" in t:
                        queue.append(("copy", step))
                    elif i not in in_asm and VMEM.match(lines[i]):
                        assert not t.startswith("scratch_")
                        queue.append(("load", step))
                    elif i in in_asm and "s_waitcnt vmcnt(" in t:
                        n = int(re.search(r"vmcnt\((\d+)\)", t).group(1))
                        waits += 1
                        if step >= 2 * ahead:
                            landed, flying = queue[:-n], queue[-n:]
                            # the next step's rows were asked for at step + 1 - ahead
                            assert all(s > step + 1 - ahead for k, s in flying if k == "copy"), (name, step)
                            assert any(k == "copy" and s == step + 1 - ahead for k, s in landed)
                            # and nothing is waited for that was asked for later than that step's loads
                            assert max(s for _, s in landed) <= step + 1 - ahead
                    elif t.startswith("s_barrier"):
                        step += 1
            assert waits == 4 * ahead
            per = [sum(k == "copy" and s == x for k, s in queue) for x in range(ahead, 2 * ahead)]
            assert len(set(per)) == 1 and per[0] >= 2
    # every number of fragments of every kernel
    assert loops >= 2 * (1 + 2 + 2 + 4) + 2 * 4


def test_the_loop_waits_for_no_load_of_its_own_step():
    """A wait of the compiler's inside the loop lets at least a step's loads fly: the weights are asked for a step or more before they are used."""
    lines = _assembly("mx4_gemm.hip")
    in_asm = {k for b in _blocks(lines) for k in range(b[0], b[1] + 1)}
    for name, rows in _kernels(lines).items():
        strips, ahead = (int(v) for v in re.search(r"Li\d+ELi\d+ELi(\d+)ELi(\d+)ELi\d+ELb[01]EEEvNS", name).groups())
        for piece in _straight(lines, rows):
            if sum("v_mfma" in lines[i] for i in piece) == 0 or sum("s_barrier" in lines[i] for i in piece) != ahead:
                continue
            for i in piece:
                m = re.search(r"s_waitcnt.*vmcnt\((\d+)\)", lines[i])
                if m and i not in in_asm:
                    assert int(m.group(1)) >= 5 * strips * (ahead - 1) - 1, (name, lines[i])


def test_no_kernel_spills_or_uses_scratch_memory():
    for name, least in (("mx4_gemm.hip", 20), ("mx4_rows.hip", 12), ("route_train.hip", 45)):
        text = "\n".join(_assembly(name))
        kernels = re.findall(r"\.name:\s+(_Z\S+)\s+\.private_segment_fixed_size:\s+(\d+)[\s\S]*?\.vgpr_spill_count:\s+(\d+)", text)
        assert len(kernels) >= least, (name, len(kernels))
        assert [k for k, scratch, spilled in kernels if int(scratch) or int(spilled)] == []


def test_a_wait_state_between_m0_and_the_load():
    m0_rule("mx4_gemm.hip")
