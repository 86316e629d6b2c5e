"""Every function of the kernels' headers has a caller."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_20791_gb300", "csrc")


def test_every_helper_of_a_header_is_called():
    text = {f: re.sub(r"//.*", "", open(f).read()) for f in sorted(glob.glob(os.path.join(CSRC, "*")))}
    everything = "\n".join(text.values())
    defined = {name for f, t in text.items() if f.endswith((".h", ".cuh"))
               for name in re.findall(r"(?:__forceinline__|inline|constexpr)\s[\w:&*<> ]*?\b(\w+)\([^;{]*\)\s*\{", t)}
    assert len(defined) > 60 and {"mbar_wait_soon", "elect_one", "warp_sum", "set_error"} & defined
    unused = sorted(n for n in defined if len(re.findall(rf"\b{n}\b", everything)) < 2)
    assert unused == []
