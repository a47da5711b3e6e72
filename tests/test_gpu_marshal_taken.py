"""Well-formed calls are answered by the compiled checks, not by the methods' own, which would hide a compiled form that always declines."""
import pytest
import torch

from test_gpu_marshal import APPEND, ATTEND, ROWS, _inputs
from test_gpu_verifier import BF, Q8

pytestmark = pytest.mark.gpu
CALLS = ("cache_write", "cache_read", "cache_append", "window_attention")


class _Counted:
    def __init__(self, fast):
        for name in CALLS:
            setattr(self, name, self._of(getattr(fast, name)))
        self.answers = []

    def _of(self, f):
        def call(*args):
            rc = f(*args)
            self.answers.append(rc)
            return rc
        return call


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_calls_are_answered(dtype, monkeypatch):
    from paper_2608_20375_b200 import binding
    binding.load_library()
    fast = _Counted(binding._fast)
    monkeypatch.setattr(binding, "_fast", fast)
    g, a = _inputs(dtype)
    rows = dict(key=a["key"].contiguous(), value=a["value"].contiguous())
    good = [(g.cache_append, APPEND, c) for c in (dict(), dict(q_out=None), dict(q=None, q_out=None), dict(position=None), dict(status=None))]
    good += [(g.window_attention, ATTEND, c) for c in (dict(), dict(mask=None, position=None), dict(lse=None, scale=0.3), dict(status=None))]
    good += [(g.cache_write, ROWS, c) for c in (dict(), rows, dict(status=None))] + [(g.cache_read, ROWS, rows)]
    for call, names, change in good:
        call(**{x: (a | change)[x] for x in names})
        assert fast.answers.pop() == 0 and not fast.answers, (call, change)
    g.window_attention(**{x: (a | dict(window=2 ** 40))[x] for x in ATTEND})  # (not a number that the C call takes: the method holds it)
    assert fast.answers == [None]
    torch.cuda.synchronize()
