"""When the workspace of ragged calls is replaced, and how long the old one is kept (no GPU: the library's call is a stand-in)."""
import contextlib
import types

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


class Buffer:
    def __init__(self, n):
        self.n, self.streams = n, []

    def numel(self):
        return self.n

    def data_ptr(self):
        return 0x10000

    def record_stream(self, s):
        self.streams.append(s)


def test_a_buffer_is_kept_for_every_stream_that_used_it(monkeypatch):
    """A call of another stream than the buffer's own may still be queued when a larger call replaces the buffer."""
    now, made, calls = ["first"], [], []

    def empty(n, dtype=None, device=None):
        made.append(Buffer(n))
        return made[-1]
    stream = types.SimpleNamespace
    torch = types.SimpleNamespace(empty=empty, uint8=1, float32=2, cuda=types.SimpleNamespace(
        current_stream=lambda device: stream(cuda_stream=0, name=now[0]), device=lambda d: contextlib.nullcontext()))

    class Lib:
        def pt_extend_workspace_bytes(self, h, tokens, batch, page_size, kv_dtype, context, n):
            n._obj.value = 1000 * tokens
            return 0

        def pt_extend(self, *args):
            calls.append(args)
            return 0
    monkeypatch.setattr(pt, "lib", lambda: Lib())
    m = pt.Model.__new__(pt.Model)
    m.torch, m.device, m.h, m.tdtype, m.cfg = torch, "cuda:0", None, 3, types.SimpleNamespace(T=2, hidden=64)
    m.ws = m.ext_ws = m.gen_ws = m.ext_key = None
    cache = types.SimpleNamespace(h=None, page_size=16, kv_dtype=pt.PT_KV_MODEL)

    def extend(tokens, name):
        now[0] = name
        x = types.SimpleNamespace(is_cuda=True, dtype=3, is_contiguous=lambda: True, shape=(2, tokens, 64), data_ptr=lambda: 0x20000)
        out = types.SimpleNamespace(is_cuda=True, dtype=2, is_contiguous=lambda: True, numel=lambda: tokens * 64, data_ptr=lambda: 0x30000)
        m.extend(cache, x, [tokens], [0], out=out)
    extend(4, "first")
    extend(4, "second")
    extend(3, "third")
    extend(9, "third")                                        # a larger buffer
    assert [b.n for b in made] == [4000, 9000] and len(calls) == 4
    assert {"second", "third"} <= {s.name for s in made[0].streams} and "third" in {s.name for s in made[1].streams}
