"""A wait over a cluster that gives up leaves its position without a result, so that no position of the row
is the last to finish: who gives up rejects the row itself.  Nothing on a GPU that works makes these waits
run out, so it is checked in the source."""
import os
import re

from paper_2607_20791_gb300.build import CSRC


def _kernel():
    text = open(os.path.join(CSRC, "verify.cu")).read()
    return text[text.index("verify_kernel(const VerifyParams p)"):text.index("int launch_verify(")]


def test_every_exchange_that_gives_up_rejects_its_row():
    body = _kernel()
    waits = re.findall(r"if \([^;]*?!exchanged?\([^;]*;", body)
    assert len(waits) == body.count("!exchange(") + body.count("!exchanged(") == 4
    assert all(w.endswith("return give_up(p);") for w in waits), waits


def test_a_rejected_row_is_written_whole():
    text = open(os.path.join(CSRC, "verify.cu")).read()
    give_up = text[text.index("void give_up("):]
    give_up = give_up[:give_up.index("\n}")]
    assert "i <= K" in give_up and "p.token_out[(int64_t)row * (K + 1) + i] = -1;" in give_up and "p.accepted_out[row] = 0;" in give_up
