"""When the workspace of ragged calls is replaced."""
from paper_2602_07306_b200 import pt


def test_the_workspace_of_ragged_calls_grows_by_shares():
    """A decoding loop over an E4M3 cache raises the context by 16 tokens at a time: a new buffer is due a handful of times, not every time."""
    have, grown = None, 0
    for step in range(4000):
        want = (32, 8, 16, pt.PT_KV_E4M3, 8 * 2048 + 128 * (step // 16 + 1))
        new = pt._grown(have, want)
        assert new[0] >= want[0] and new[1] >= want[1] and new[2] <= want[2] and new[3] >= want[3] and new[4] >= want[4]
        grown += new != have
        have = new
    assert grown <= 6, grown                                  # the first, and log(48384 / 16512) / log(1.25) = 4.8 more
    # calls that alternate between caches of different formats and page sizes share one buffer
    have = pt._grown(pt._grown(have, (4, 2, 64, pt.PT_KV_MODEL, 0)), (4, 2, 8, pt.PT_KV_MODEL, 0))
    assert pt._grown(have, (4, 2, 64, pt.PT_KV_MODEL, 0)) == have == pt._grown(have, (32, 8, 16, pt.PT_KV_E4M3, 8 * 2048))
