"""Status words of kernel-level calls, handed out 256 at a time, without a GPU."""
import pytest

from paper_2602_07306_b200 import pt


@pytest.fixture
def cpu_status(monkeypatch):
    """_new_status on the CPU: zeroed memory that remembers no device."""
    import torch
    zeros, made = torch.zeros, []

    def fake(*size, dtype=None, device=None):
        made.append(size)
        return zeros(*size, dtype=dtype)
    monkeypatch.setattr(torch, "zeros", fake)
    monkeypatch.setattr(pt, "_raw_stream", lambda index: 77 + index)
    monkeypatch.setattr(pt, "_status_blocks", {})
    state = {"device": 0, "capturing": ()}
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state["device"], raising=False)

    class device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.was, state["device"] = state["device"], self.index

        def __exit__(self, *_):
            state["device"] = self.was
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["device"] in state["capturing"])
    return state, made


def test_status_words_are_not_shared(cpu_status):
    a = [pt._new_status(0) for _ in range(600)]
    assert len({t.data_ptr() for t in a}) == 600 and all(t.shape == (16,) and not t.any() for t in a)


def test_another_thread_may_take_the_last_status_words(cpu_status):
    class Raced(list):
        """Looks as it does to one thread, and is empty once that thread takes from it."""
        def __bool__(self):
            some = len(self) > 0
            self.clear()
            return some
    pt._new_status(0)
    key = next(iter(pt._status_blocks))
    pt._status_blocks[key] = Raced(pt._status_blocks[key])
    assert pt._new_status(0).shape == (16,)
    pt._status_blocks[key] = Raced()
    assert pt._new_status(0).shape == (16,)


def test_a_capture_on_the_tensors_device_counts_not_on_the_current_one(cpu_status):
    state, made = cpu_status
    state.update(device=0, capturing=(1,))
    pt._new_status(1)                                         # a graph of device 1 is being captured: memory of its own
    assert made == [(16,)] and not pt._status_blocks
    made.clear()
    state.update(capturing=(0,))
    pt._new_status(1)                                         # nothing is captured on device 1
    assert made == [((256, 16),)] and state["device"] == 0
