"""GPU: the objects that the calls on packed new tokens are given, made and used where a program might: on another device than the current one,
inside a capture."""
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from prompt_util import Requests

pytestmark = pytest.mark.gpu


def test_objects_of_another_device_are_refused(monkeypatch):
    r = Requests([(5, 3), (2, 0)], 4, 2, seed=1)
    made, taken = sd.BlockPool(8), sd.BlockPool(8, torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    r.prepare()
    torch.cuda.synchronize()
    here = sd._here()
    monkeypatch.setattr(sd, "_here", lambda: here + 1)       # (as if that were the current device)
    for call in (r.prepare, lambda: made.on(None), lambda: taken.on(None), lambda: r.prompts.on(torch.cuda.current_stream())):
        with pytest.raises(AssertionError):
            call()
    monkeypatch.undo()
    r.prepare()
    r.append()
    r.attend()
    r.check()
