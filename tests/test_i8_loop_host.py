"""CPU checks of the generated assembly k loop of the large products of 8-bit integers (csrc/gen_i8_loop.py -> ops_i8_loop.inc): the committed file is what the generator writes,
and an emulation of its scalar side for 1 to 40 k steps shows that every copy fetches a k step below KT from the right address into the right LDS buffer, that every
fragment read touches its block of the buffer that holds its k step, after that has landed for every wavefront, and that no buffer is overwritten before its last read."""
import pytest

from test_w4a_loop_host import A_BASE, B_BASE, LDS_WAVE, _generator, _run

A_BUF, NCOPY, SLICE, AHEAD = 32768, 8, 64, 2
LINES = _generator("gen_i8_loop").block()


def test_committed_include_is_what_the_generator_writes():
    gen = _generator("gen_i8_loop")
    with open(gen.INC_PATH) as f:
        assert f.read() == gen.render()


def buffer_of(kind, step):
    """(which, where in LDS)"""
    return (("A", step % 2), step % 2 * A_BUF) if kind == "A" else (("B", step % 3), (2 + step % 3) * A_BUF)


def lines_for(kt):
    """The emulator has B step by %[b_step] and its running pointer set up by that; this loop steps both by 128 bytes."""
    b_ptr = B_BASE + AHEAD * 128
    return [ln.replace("%[b_ptr_lo]", str(b_ptr & 0xffffffff)).replace("%[b_ptr_hi]", str(b_ptr >> 32)) for ln in LINES]


@pytest.mark.parametrize("kt", range(1, 41))
def test_copies_reads_waits_and_barriers(kt):
    trace, nmfma = _run(lines_for(kt), kt, AHEAD)
    assert nmfma == 2 * SLICE * kt
    order = [e[2] for e in trace if e[1] == "mfma"]
    for i in range(0, len(order), SLICE):
        assert sorted(order[i:i + SLICE]) == list(range(SLICE))
    # the barrier in front of the loop, behind a wait that leaves out the copies of k step 1 alone
    first = next(i for i, e in enumerate(trace) if e[1] == "barrier")
    assert trace[first - 1][1] == "wait" and trace[first - 1][2] == (16 if kt > 1 else 0)
    barriers = [e[0] for e in trace if e[1] == "barrier"]
    assert len(barriers) == kt + 1
    # copies: those of k steps 0 and 1 that the C++ issues in front of the block, then the block's own
    copies = [(-100 + s, buffer_of(kind, s)[0], s) for s in range(min(kt, AHEAD)) for kind in "AB" for _ in range(NCOPY)]
    for t, what, *rest in trace:
        if what != "copy":
            continue
        voff, src, m0, at = rest
        j = (at - 1) // (2 * SLICE)
        kind, n, want = ("A" if voff.startswith("%[a_off") else "B"), int(voff[-2]), j + AHEAD if j + AHEAD < kt else 0
        buf, where = buffer_of(kind, j + AHEAD)
        assert src == (A_BASE if kind == "A" else B_BASE) + 128 * want and m0 - LDS_WAVE == where + 4096 * n
        copies.append((t, buf, want if j + AHEAD < kt else None))
    assert len(copies) == 2 * NCOPY * (kt + min(kt, AHEAD))
    times = [c[0] for c in copies]

    def landed(i):
        """When copy i has landed for every wavefront: the first barrier behind a wait that leaves out fewer than were issued behind it."""
        for t, what, *rest in trace:
            if what == "wait" and rest[0] is not None and t > times[i] and len(copies) - 1 - i - sum(x > t for x in times) >= rest[0]:
                return next((b for b in barriers if b > t), None)
        return None
    land = [landed(i) for i in range(len(copies))]
    base = {"%[a_rd": 0, "%[b_rd": 2 * A_BUF, "%[b_rdh": 4 * A_BUF}
    last_read = {}
    for t, what, *rest in trace:
        if what != "read":
            continue
        reg, off, at = rest
        h = -1 if at == 0 else (at - 1) // SLICE
        step, s = (h + 1) // 2, (h + 1) % 2
        kind = "A" if reg.startswith("%[a") else "B"
        buf, where = buffer_of(kind, step)
        within = base[reg[:-2]] + off - where
        assert int(reg[-2]) == s and within % 2048 == 0 and 0 <= within < A_BUF // 2
        last_read[t] = buf
        if step < kt:
            here = [i for i, c in enumerate(copies) if c[1] == buf and c[0] < t]
            assert all(copies[i][2] == step for i in here[-NCOPY:]) and all(land[i] is not None and land[i] < t for i in here[-NCOPY:])
    # a copy into a buffer begins behind a barrier that every wavefront reaches with its reads of the buffer done
    lgkm = [e[0] for e in trace if e[1] == "wait" and e[3] == 0]
    for t, buf, _ in copies[2 * NCOPY * min(kt, AHEAD):]:
        for r in (r for r, b in last_read.items() if b == buf and r < t):
            done = next(w for w in lgkm if w > r)
            assert any(done < b < t for b in barriers), "a buffer is overwritten before its reads are done"
    assert trace[-1][1] == "wait" and trace[-1][2] == 0
