"""Rows in use of the calls on rows of logits: refused on the host, before any launch (no GPU here)."""
import ctypes

from paper_2509_18824_b200 import binding as b

ok = 4096


def test_rows_in_use():
    for n_used, per in ((ok, 0), (ok, -1), (4098, 4)):
        c = b.sd_sampling(None, None, None, None, n_used, per)
        assert b.lib.sd_filter_logits(ok, 0, 100, 4, 100, ctypes.byref(c), 8192, ok, None, ok, None) == b.SD_ERR_INVALID_ARG
        assert b.lib.sd_sample_logits(ok, 0, 100, 4, 100, ctypes.byref(c), ok, 1, ok, None, None, None, ok, None) == b.SD_ERR_INVALID_ARG
