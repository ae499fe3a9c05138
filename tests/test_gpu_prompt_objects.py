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


def test_objects_made_inside_a_capture():
    """Their arrays are the graph's; they may be used outside of it too, on any stream."""
    r = Requests([(40, 100), (1, 300), (64, 0)], 7, 1, seed=4)
    first = r.prompts
    r.prepare()
    r.append()
    r.attend()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    table, lens, new, held = first.block_table, first.len, first.n_new, first.n_blocks
    with torch.cuda.graph(graph):
        r.prompts = sd.Prompts(r.N, 7, 1, 128, table, lens, new, held, num_blocks=r.num_blocks)
        r.prepare()
        r.append()
        r.attend()
    r.out.fill_(7.0)
    r.lse.fill_(7.0)
    graph.replay()
    r.check()
    for stream in (None, side):                              # the current stream was not the capture's
        r.out.fill_(7.0)
        r.lse.fill_(7.0)
        torch.cuda.synchronize()
        r.prepare(stream)
        r.append(stream)
        r.attend(stream)
        r.check()
