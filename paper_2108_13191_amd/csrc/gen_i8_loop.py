#!/usr/bin/env python3
"""Writes ops_i8_loop.inc: the k loop of the four-wavefront 256 x 256 kernel of the products of 8-bit integers (ops_i8_long.hip) as a
hand-scheduled assembly block, plus the operand lists that bind it to the C++ around it.  Structure, fixed registers and the order of MFMAs are those of
gen_w4a_loop.py, which documents them: k steps unrolled six deep over 2 A and 3 B buffers, one barrier a k step, copies of k step j + 2 issued during step j (from
the tile's first k step once that would lie beyond KT).  What differs: a k step is 128 bytes of a row of either operand, both lie with k contiguous, and a
slice is 64 k of them: 64 MFMAs of 16 x 16 x 64 and 16 fragment reads of 16 bytes a lane.

In front of it the accumulators are cleared while the first copies, which the C++ has issued, arrive.

  slice 0 (fragment set 0):
    after MFMA 0..3     scalar: source pointers of this step's copies, advance
    after MFMA 3r + 1   fragment read r (of 16) of slice 1 into set 1
    after MFMA 8t + 4   M0 for copy t of B(j + 2), after MFMA 8t + 6 the copy
    wait: all copies but those 8, all LDS reads; workgroup barrier
  slice 1 (fragment set 1):
    after MFMA 3r + 1   fragment read r of slice 0 of k step j + 1
    after MFMA 8t + 4, 8t + 6   copy t of A(j + 2)
    wait: all LDS reads

Run: python3 gen_i8_loop.py   (writes ops_i8_loop.inc beside itself)
"""
import os

from gen_w4a_loop import A_BUF, B_BUF, B_REGION, S_APTR, S_ASRC, S_BPTR, S_BSRC, S_J, S_J2, acc, asm_macro, block_at, frag_a, frag_b

ROW = 128                                         # bytes of a row of a buffer
SCALAR_CLOBBERS = [f"s{i}" for i in range(64, 74)]
V_CLOBBERED = 128                                 # two fragment sets of 64 registers
NREAD = 16
READ_AFTER = [3 * r + 1 for r in range(NREAD)]    # MFMAs of a slice


def mfma(d, i):
    fm, fn = block_at(i)
    return f"v_mfma_i32_16x16x64_i8 {acc(fm, fn)}, {frag_b(d, fn)}, {frag_a(d, fm)}, {acc(fm, fn)}"


def read(phase, s, d, r):
    """Read r of slice s of the stage of k step phase into fragment set d: the 8 B operands first, then the 8 A operands.  The third B buffer
    is addressed from registers of its own: an instruction's offset has 16 bits."""
    abuf, bbuf = phase % 2, phase % 3
    if r < 8:
        reg, off = (f"%[b_rd{s}]", bbuf * B_BUF) if bbuf < 2 else (f"%[b_rdh{s}]", 0)
        off += r * 16 * ROW
        assert off < 65536
        return f"ds_read_b128 {frag_b(d, r)}, {reg} offset:{off}"
    off = abuf * A_BUF + (r - 8) * 16 * ROW
    assert off < 65536
    return f"ds_read_b128 {frag_a(d, r - 8)}, %[a_rd{s}] offset:{off}"


def k_step(ph):
    """One k step at phase ph = j mod 6."""
    out = []
    b_dst, a_dst = B_REGION + ((ph + 2) % 3) * B_BUF, (ph % 2) * A_BUF
    scalar = [
        [f"s_add_u32 {S_J2}, {S_J}, 2", f"s_cmp_lt_u32 {S_J2}, %[kt]"],
        [f"s_cselect_b32 s66, {S_APTR[0]}, %[a_base_lo]", f"s_cselect_b32 s67, {S_APTR[1]}, %[a_base_hi]"],
        [f"s_cselect_b32 s68, {S_BPTR[0]}, %[b_base_lo]", f"s_cselect_b32 s69, {S_BPTR[1]}, %[b_base_hi]"],
        [f"s_add_u32 {S_APTR[0]}, {S_APTR[0]}, {ROW}", f"s_addc_u32 {S_APTR[1]}, {S_APTR[1]}, 0",
         f"s_add_u32 {S_BPTR[0]}, {S_BPTR[0]}, {ROW}", f"s_addc_u32 {S_BPTR[1]}, {S_BPTR[1]}, 0"],
    ]
    for s, (dst, offsets, source) in enumerate(((b_dst, "b_off", S_BSRC), (a_dst, "a_off", S_ASRC))):
        r = 0
        for i in range(64):
            out.append(mfma(s, i))
            if s == 0 and i < 4:
                out += scalar[i]
            if i in READ_AFTER:
                out.append(read(ph, 1, 1, r) if s == 0 else read((ph + 1) % 6, 0, 0, r))
                r += 1
            if i % 8 == 4:
                out.append(f"s_add_u32 m0, %[lds_wave], {dst + 4096 * (i // 8)}")
            if i % 8 == 6:
                out.append(f"global_load_lds_dwordx4 %[{offsets}{i // 8}], {source}")
            if s == 1 and i == 60:
                out.append(f"s_add_u32 {S_J}, {S_J}, 1")
        assert r == NREAD
        out += ["s_waitcnt vmcnt(8) lgkmcnt(0)", "s_barrier"] if s == 0 else ["s_waitcnt lgkmcnt(0)"]
    out += [f"s_cmp_lt_u32 {S_J}, %[kt]", "s_cbranch_scc1 I8_TOP_%=" if ph == 5 else "s_cbranch_scc0 I8_DONE_%="]
    return out


def block():
    out = [f"v_accvgpr_write_b32 a{i}, 0" for i in range(256)]
    out += [f"s_mov_b32 {S_J}, 0",
            f"s_mov_b32 {S_APTR[0]}, %[a_ptr_lo]", f"s_mov_b32 {S_APTR[1]}, %[a_ptr_hi]",
            f"s_mov_b32 {S_BPTR[0]}, %[b_ptr_lo]", f"s_mov_b32 {S_BPTR[1]}, %[b_ptr_hi]"]
    # k step 0 has landed (or has been written to LDS); the 16 copies of k step 1, if there is one, may be on their way until the wait in the middle of k step 0
    out += ["s_cmp_lt_u32 %[kt], 2", "s_cbranch_scc1 I8_ALONE_%=", "s_waitcnt vmcnt(16) lgkmcnt(0)", "I8_ALONE_%=:",
            "s_cbranch_scc0 I8_LANDED_%=", "s_waitcnt vmcnt(0) lgkmcnt(0)", "I8_LANDED_%=:", "s_barrier"]
    out += [read(0, 0, 0, r) for r in range(NREAD)]
    out += ["s_waitcnt lgkmcnt(0)", "I8_TOP_%=:"]
    for ph in range(6):
        out += k_step(ph)
    return out + ["I8_DONE_%=:", "s_waitcnt vmcnt(0)"]


def rows_of(items, n):
    return ", \\\n    ".join(", ".join(items[i:i + n]) for i in range(0, len(items), n))


def render():
    """The text of ops_i8_loop.inc."""
    text = ["// Generated by gen_i8_loop.py -- edit the generator, not this file.",
            "// I8_LOOP_ASM: the k loop; I8_LOOP_OUTPUTS(acc) / I8_LOOP_INPUTS / I8_LOOP_CLOBBERS: its operands."]
    text += asm_macro("I8_LOOP_ASM", block())
    outs = [f'"=&{{{acc(fm, fn)}}}"(ACC[{fm}][{fn}])' for fm in range(8) for fn in range(8)]
    inputs = [f'[a_rd{s}] "v"(a_rd[{s}])' for s in range(2)] + [f'[b_rd{s}] "v"(b_rd[{s}])' for s in range(2)]
    inputs += [f'[b_rdh{s}] "v"(b_rd[{s}] + {2 * B_BUF}u)' for s in range(2)]
    inputs += [f'[a_off{t}] "v"(a_off[{t}])' for t in range(8)] + [f'[b_off{t}] "v"(b_off[{t}])' for t in range(8)]
    inputs += [f'[{n}] "s"({n})' for n in ("lds_wave", "kt", "a_base_lo", "a_base_hi", "b_base_lo", "b_base_hi", "a_ptr_lo", "a_ptr_hi", "b_ptr_lo", "b_ptr_hi")]
    clobbers = [f'"v{i}"' for i in range(V_CLOBBERED)] + [f'"{s}"' for s in SCALAR_CLOBBERS] + ['"m0"', '"scc"', '"memory"']
    for name, items, n in (("I8_LOOP_OUTPUTS(ACC)", outs, 8), ("I8_LOOP_INPUTS", inputs, 4), ("I8_LOOP_CLOBBERS", clobbers, 16)):
        text += [f"#define {name} \\", "    " + rows_of(items, n)]
    return "\n".join(text) + "\n"


INC_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "ops_i8_loop.inc")


def main():
    with open(INC_PATH, "w") as f:
        f.write(render())
    print(f"wrote {INC_PATH}: {len(block())} instructions")


if __name__ == "__main__":
    main()
