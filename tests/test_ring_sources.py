"""What kernels do after a wait that gave up, kept by reading their sources: no run can show it but a broken one."""
import re

from tests.test_kernel_sources import sources


def test_no_poll_of_both_parities():
    """Of a barrier's two parities one is always that of its last complete phase: a poll for either waits for nothing."""
    for name, text in sources().items():
        assert not re.search(r"mbar_try\(([^;]*), 0u?\) \|\| mbar_try\(\1, 1u?\)", text), name


def test_rings_are_drained_when_their_wait_gives_up():
    for name, call in {"pt_tc_attn.cu": "drain_ring(wbar, kDecStages, 0, kDecStages);", "pt_tc_kv8.cu": "drain_ring(wbar, kDecStages, 0, kDecStages);",
                       "pt_kv4_attn.cu": "drain_ring(bars, C::STAGES, slot, pending);"}.items():
        text = sources()[name]
        assert text.count("bool timed_out = false;") == text.count(call) == 1, name


class Barrier:
    """Phases of an mbarrier: a poll for a parity says yes when the phase before the present one has it."""

    def __init__(self, complete):
        self.complete = complete

    def poll(self, parity):
        return (self.complete - 1) % 2 == parity


def test_the_parity_of_the_copies_under_way():
    """drain_ring's rule, played through: it waits while the present phase is open, and goes on when that is complete."""
    text = sources()["pt_ring.cuh"]
    assert "flying = mbar_try(&bars[s], 1) ? 0u : 1u;" in text and "!mbar_try(&bars[s], flying)" in text
    for complete in range(6):
        b = Barrier(complete)
        flying = 0 if b.poll(1) else 1
        assert not b.poll(flying)
        b.complete += 1
        assert b.poll(flying)


def test_the_stages_under_way():
    """Those from the one that gave up on, as many as tiles are left: each stage is filled again as soon as it is consumed."""
    for stages in (1, 2, 3, 6):
        for total in range(1, 20):
            for consumed in range(total):
                flying = {n % stages for n in range(consumed, min(total, consumed + stages))}
                assert {(consumed + i) % stages for i in range(min(stages, total - consumed))} == flying


def test_blocks_whose_waits_gave_up_let_their_copies_land():
    """Every kernel with an abort flag asks it when all of its warps have met at the end, before tensor memory is freed."""
    found = 0
    for name, text in sources().items():
        for m in re.finditer(r"__syncthreads\(\);\n((?:(?!__syncthreads).)*?)tcgen05\.dealloc", text, re.S):
            assert m.group(1).lstrip().startswith("if (*abort_flag) settle_copies();"), (name, m.group(1))
            found += 1
    assert found == 6
