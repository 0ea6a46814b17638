"""What kernels do after a wait that gave up, kept by reading their sources: no run can show it but a broken one."""
import re

from tests.test_kernel_sources import sources


def test_no_poll_of_both_parities():
    """Of a barrier's two parities one is always that of its last complete phase: a poll for either waits for nothing."""
    for name, text in sources().items():
        calls = re.findall(r"mbar_try\(((?:[^(),]|\([^()]*\))+),\s*([^)]+)\)", text)
        fixed = [(bar.strip(), parity.strip()) for bar, parity in calls if parity.strip() in ("0", "0u", "1", "1u")]
        assert not [bar for bar, parity in fixed if parity[0] == "0" and any(b == bar and p[0] == "1" for b, p in fixed)], name


def test_rings_are_drained_from_the_stage_that_gave_up():
    """A warp that leaves its loop with stages under way drains them, from the slot and parity it waited for on, and no others."""
    for name, call in {"pt_tc_attn.cu": "drain_ring(wbar, kDecStages, it % kDecStages, (it / kDecStages) & 1, (npages - gi + 3) / 4);",
                       "pt_tc_kv8.cu": "drain_ring(wbar, kDecStages, it % kDecStages, (it / kDecStages) & 1, (npages - gi + 3) / 4);",
                       "pt_kv4_attn.cu": "drain_ring(bars, C::STAGES, slot, parity, pending);"}.items():
        text = sources()[name]
        assert text.count("bool timed_out = false;") == text.count(call) == 1, name


def test_the_drained_stages_are_those_in_flight():
    """The rule of drain_ring beside a ring that is played through: stages filled in turn, each refilled when it is consumed."""
    for stages in (1, 2, 3, 6):
        for total in range(0, 20):
            for consumed in range(0, total):
                issued = min(total, consumed + stages)
                flying = {(n % stages, n // stages & 1) for n in range(consumed, issued)}
                slot, parity, drained = consumed % stages, consumed // stages & 1, set()
                for i in range(min(stages, total - consumed)):
                    drained.add((slot, parity))
                    slot += 1
                    if slot == stages:
                        slot, parity = 0, parity ^ 1
                assert drained == flying
