"""The binding of the block's operators where no GPU is needed."""
import threading

import torch

from paper_1606_03401_amd import binding as mb


def test_first_calls_from_two_threads(monkeypatch):
    """A second thread that comes while the first one is still loading: it finds everything in place, or loads by itself."""
    names = ("_torch", "_DTYPES", "_current_device", "_current_stream")
    for name, value in zip(names, (None, (), None, None)):
        monkeypatch.setattr(mb, name, value)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    inside, release, seen = threading.Event(), threading.Event(), []

    def init():
        if threading.current_thread().name == "first":
            inside.set()
            assert release.wait(20)

    class Tensor:
        def get_device(self):
            return 0

    def second():
        mb._gpu(Tensor())
        seen.append(tuple(getattr(mb, n) for n in names))

    monkeypatch.setattr(torch.cuda, "init", init)
    a = threading.Thread(target=lambda: mb._gpu(Tensor()), name="first")
    b = threading.Thread(target=second, name="second")
    a.start()
    assert inside.wait(20)
    b.start()
    b.join(20)
    release.set()
    a.join(20)
    assert len(seen) == 1 and all(seen[0]), seen
