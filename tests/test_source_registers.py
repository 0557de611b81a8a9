"""A warpgroup that raises its registers waits, without a limit, until the others of its block have given up as many: shown on the source."""
import os
import re

from paper_2609_36938_b200 import build


def test_register_shares_add_up():
    for name in sorted(os.listdir(build.CSRC)):
        with open(os.path.join(build.CSRC, name)) as f:
            code = re.sub(r"//[^\n]*", "", f.read())
        if "setmaxnreg" not in code:
            continue
        (up,), (down,) = re.findall(r"setmaxnreg\.inc\.sync\.aligned\.u32 (\d+)", code), re.findall(r"setmaxnreg\.dec\.sync\.aligned\.u32 (\d+)", code)
        threads, softmax = int(re.search(r"ST_THREADS = (\d+)", code).group(1)), 32 * int(re.search(r"ST_SOFTMAX_WARPS = (\d+)", code).group(1))
        launched = 65536 // threads // 8 * 8
        assert softmax * int(up) + (threads - softmax) * int(down) <= threads * launched
        assert softmax % 128 == 0 and (threads - softmax) % 128 == 0
        # every warp that is not one of the softmax warps passes the one place where registers are given up, before its role
        assert code.count("fewer_registers()") == 1 and code.count("more_registers()") == 1
        assert re.search(r"warp >= ST_SOFTMAX_WARPS\) \{\s*fewer_registers\(\);\s*if \(warp == ST_COPY_WARP\)", code)
