"""The 8-bit cache's bindings on the host (no GPU): token counts and row offsets are integers or refused."""
import numpy as np
import pytest

from paper_2511_22533_amd import f3c


@pytest.mark.parametrize("lens,off", [([63.9, 1], [0, 1, 2]), ([5, 1], [0, 1.7, 2]), ([5.0, 1], [0, 1, 2]),
                                      (np.array([5.0, 1.0]), [0, 1, 2]), ([5, 1], np.array([0, 1, 2], np.float32)),
                                      (["5", 1], [0, 1, 2]), ([5, None], [0, 1, 2]), (5, [0, 1]), (None, [0, 1]),
                                      (iter([5, 1.5]), [0, 1, 2]), ([5, 1], iter([0, 1, 2.0]))])
def test_lists_of_anything_but_integers_are_refused(monkeypatch, lens, off):
    import torch

    class Library:
        def __getattr__(self, name):
            raise AssertionError("the library was called")

    monkeypatch.setattr(f3c, "_lib", Library())
    monkeypatch.setattr(f3c, "_device", lambda t, torch: t.get_device())
    monkeypatch.setattr(f3c, "_stream_on", lambda *a: 0)
    e = lambda *s, t=torch.uint8: torch.empty(*s, dtype=t)  # noqa: E731
    cache = f3c.Cache8(e(3, 2, 64, 32), e(3, 2, 32, 64), e(3, 2), e(3, 2), e(2, 3, t=torch.int32))
    q = e(4, 64, t=torch.bfloat16)
    once = [list(x) if hasattr(x, "__next__") else x for x in (lens, off)]
    for call in (lambda lens, off: f3c.op_cache8_append(f3c.F3C_BF16, cache, lens, off, q, q),
                 lambda lens, off: f3c.op_cache8_attention(cache, 2, off, lens, q, q)):
        with pytest.raises(ValueError, match="32-bit integers"):
            call(*(iter(x) if hasattr(y, "__next__") else y for x, y in zip(once, (lens, off))))
