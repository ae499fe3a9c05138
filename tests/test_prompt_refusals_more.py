"""Argument checks of the calls on packed new tokens, on the host (no GPU here): what has to be accepted."""
from test_prompt_refusals import append, attend, b, ctypes, prompts


def test_no_rows_need_no_workspace():
    assert b.lib.sd_prompt_workspace_bytes(ctypes.byref(prompts(N=0))) == 0
    assert attend(N=0, q=None, out=None, ws=None, ws_bytes=0) == b.SD_OK
    assert append(N=0, k=None, v=None) == b.SD_OK
    # ... but everything else that is always needed
    for bad in (dict(scale=0.0), dict(lse=4097), dict(cache=(None, 4096, 8)), dict(st=None)):
        assert attend(N=0, q=None, out=None, ws=None, ws_bytes=0, **bad) == b.SD_ERR_INVALID_ARG, bad
