"""Page copies from Python without a GPU: everything is checked before anything is launched."""
import numpy as np
import pytest

from paper_2602_07306_b200 import pt


class Tensor:
    """What a call looks at of a CUDA tensor."""

    def __init__(self, shape, esz, at, device=0, contiguous=True):
        self.shape, self.esz, self.at, self.device, self.contiguous = tuple(shape), esz, at, device, contiguous
        self.dtype = esz

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous

    def numel(self):
        return int(np.prod(self.shape))

    @property
    def nbytes(self):
        return self.numel() * self.esz

    def data_ptr(self):
        return self.at


@pytest.fixture
def launches(monkeypatch):
    """Page copies that would be launched: calls with pairs to copy; calls without any are the library's own, which launch nothing."""
    pt.lib()
    seen = []

    def call(index, fn, *args):
        if args[8]:
            seen.append(args)
        else:
            pt.check(fn(*args, None))
    monkeypatch.setattr(pt, "_call", call)
    return seen


def planes(pages=10, at=1 << 30, dh=128):
    return Tensor((2, 3, pages, 2, 4, 16, dh), 1, at), Tensor((2, 3, pages, 2, 4, 16), 4, at + (1 << 28))


def test_refused_scales_leave_the_pool_alone(launches):
    pool, scales = planes()
    to, to_scales = planes(12, at=1 << 32)
    bad = {
        "device": dict(scales=Tensor(scales.shape, 4, scales.at, device=1)),
        "strided": dict(scales=Tensor(scales.shape, 4, scales.at, contiguous=False)),
        "layers": dict(scales=Tensor((2, 2) + scales.shape[2:], 4, scales.at)),
        "pages": dict(scales=planes(11)[1]),
        "fewer pages": dict(scales=planes(9)[1]),
        "block of 8 bytes": dict(scales=Tensor((2, 3, 10, 2), 4, scales.at)),
        "misaligned": dict(scales=Tensor(scales.shape, 4, scales.at + 8)),
        "out without out_scales": dict(scales=scales, out=to),
        "out_scales without out": dict(scales=scales, out_scales=to_scales),
        "out_scales without scales": dict(out=to, out_scales=to_scales),
        "out_scales of other pages": dict(scales=scales, out=to, out_scales=planes(13, at=1 << 32)[1]),
        "out_scales over scales": dict(scales=scales, out=to, out_scales=Tensor(to_scales.shape, 4, scales.at + 16)),
        "out of another shape": dict(scales=scales, out=Tensor((2, 3, 12, 2, 4, 16, 64), 1, 1 << 32), out_scales=to_scales),
    }
    for what, args in bad.items():
        with pytest.raises((ValueError, pt.PtError)):
            pt.kernel_kv_copy_pages(pool, [0, 1], [5, 6], **args)
        assert not launches, what


def test_both_planes_are_copied(launches):
    pool, scales = planes()
    pt.kernel_kv_copy_pages(pool, [0, 1], [5, 6], scales=scales)
    assert [(a[0], a[2], a[4], a[5]) for a in launches] == [(pool.at, pool.at, 6, 2 * 4 * 16 * 128), (scales.at, scales.at, 6, 2 * 4 * 16 * 4)]
    launches.clear()
    to, to_scales = planes(12, at=1 << 32)
    pt.kernel_kv_copy_pages(pool, [0], [11], scales=scales, out=to, out_scales=to_scales)
    assert [(a[0], a[1], a[2], a[3]) for a in launches] == [(pool.at, 10, to.at, 12), (scales.at, 10, to_scales.at, 12)]
