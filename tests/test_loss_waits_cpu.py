"""What the streamed loss kernel does behind a wait that was given up.  A warp that goes on must not announce bytes at a barrier whose phase is still open, nor arrive at or
write to another block that has not read what was there; the copying warp must not let the block end in front of its copies.  Read from the source: on a GPU none of
these waits runs out by itself."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1811_02084_b200", "csrc", "loss_rows.cu")


def roles():
    """The kernel's parts: copies, the rows' numbers, walks, and what all run at the end."""
    text = open(SOURCE).read()
    kernel = text[text.index("loss_stream_kernel(const LossRows a"):]
    kernel = kernel[:kernel.index("\n}\n")]
    at = [kernel.index(f"// ------------------------------- {name}") for name in ("copies", "the rows' numbers", "walks")]
    end = kernel.rindex("\n  }\n", 0, kernel.index("if (parts > 1) {             // nobody leaves"))
    return [kernel[a:b] for a, b in zip(at, at[1:] + [end])] + [kernel[end:]]


def test_the_numbers_warps_leave_before_they_announce_or_send():
    _, numbers, walks, _ = roles()
    lines = [line.strip() for line in numbers.splitlines()]
    waits = {re.search(r"0xA0\d", line).group(): i for i, line in enumerate(lines) if "bar_wait(" in line}
    assert list(waits) == ["0xA02", "0xA03", "0xA04", "0xA05"]
    assert all(lines[waits[w] + 1] == "if (given_up(st)) break;" for w in ("0xA03", "0xA04"))
    # what another block sees, and the announcement of bytes, lies behind such a check, whichever wait was given up; the walks have neither
    for what, behind in (("bar_expect(", "0xA03"), ("st.async", "0xA03"), ("mbarrier.arrive.release.cluster", "0xA04")):
        assert numbers.count(what) == 1 and "given_up(st)" in numbers[numbers.index(behind):numbers.index(what)] and what not in walks
    assert numbers.count("in_peer(") == 3 and "in_peer(" not in walks


def test_the_copying_warp_leaves_and_waits_for_its_copies():
    copies, _, _, end = roles()
    wait, check, expect = copies.index("bar_wait(&st.empty"), copies.index("if (*(volatile int*)&st.abort) break;"), copies.index("bar_expect(")
    assert wait < check < expect
    left = copies.index("if (given_up(st)) break;")
    assert expect < left < copies.index("while (!bar_try(&st.full[c]") and "kLandCycles" in copies[left:]
    # the cluster's last barrier behind all of it, whole warps at it
    assert re.search(r"__syncwarp\(\);\s+cluster_arrive\(\);\s+cluster_wait\(\);", end)


def landed_parities(chunks, copies):
    """(what the source waits for, what a slot's barrier needs) per slot after so many copies: slot and phase as the copying warp counts them."""
    slot, phase, fills = 0, 1, [0] * chunks
    for _ in range(copies):
        fills[slot] += 1
        slot += 1
        if slot == chunks:
            slot, phase = 0, phase ^ 1
    return [(phase ^ 1 if c < slot else phase, fills[c]) for c in range(chunks)]


def test_the_phases_that_the_copying_warp_waits_for():
    for chunks in (2, 10, 13):
        for copies in range(4 * chunks + 1):
            # fill number n of a slot (from 1 on) completes the phase of parity (n - 1) % 2; an unused one's wait is for parity 1, which a new barrier is past
            assert all(parity == ((n - 1) % 2 if n else 1) for parity, n in landed_parities(chunks, copies))
