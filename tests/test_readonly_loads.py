"""The read-only path (__ldg) is for what no kernel writes that may still run when the reader begins: kernels of the library begin while the
one ahead of them in the stream runs, and the read-only path may give them what stood there before that one wrote."""
import os
import re

from paper_2509_18824_b200 import build

# what is read that way: a caller's inputs (block tables, hidden states and W's rows, the draft's features), and what the LM-head tiles
# leave, which let nobody begin early.  Logits, draft distributions, their probabilities and log-sum-exps come from sd_filter_logits and
# sd_sample_logits, which do.
FROM_NO_KERNEL_THAT_MAY_RUN = {"table", "seq_table", "src", "a", "qr", "group_stats"}


def test_what_is_read_through_the_read_only_path():
    seen = set()
    for f in sorted(os.listdir(build.CSRC)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, f)).read())
        for m in re.finditer(r"__ldg\s*\(\s*([A-Za-z_]\w*)", text):
            assert m.group(1) in FROM_NO_KERNEL_THAT_MAY_RUN, (f, text[m.start():m.start() + 60])
            seen.add(m.group(1))
    assert seen == FROM_NO_KERNEL_THAT_MAY_RUN
