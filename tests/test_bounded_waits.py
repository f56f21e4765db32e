"""The device waits' limits, followed in the kernels' own text (CPU): a wait that
gives up has looked at the clock, since a try may come back at any time, and no
thread leaves its warp behind."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_07144_gb300", "csrc")


def _functions():
    """(file, text) of every function at the outermost level."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*")) + glob.glob(os.path.join(CSRC, "*.h"))):
        for text in re.split(r"\n}\n", open(path).read()):
            yield os.path.basename(path), text


def test_a_wait_that_gives_up_has_looked_at_the_clock():
    waits = [(f, t) for f, t in _functions() if re.search(r"atomicOr\([^;]*FKV_ST_TIMEOUT", t)]
    assert len(waits) >= 4
    for f, t in waits:
        assert re.search(r"globaltimer_(ns|lo)\(\)", t), (f, t[-600:])


def test_no_thread_leaves_its_warp_behind():
    """A thread that gave up and left its loop would be waited for by its warp at the next step that is for all
    threads: a wait of the step kernel is voted on, and one of the prompt kernel leads to no way out."""
    text = {f: open(os.path.join(CSRC, f)).read() for f in ("attend.cu", "attend_prompt.cu")}
    waits = [m.start() for m in re.finditer(r"mbar_wait\(", text["attend.cu"])]
    drain = "a.status, 2000000);\n            __syncwarp();"         # after a wait that was voted on
    voted = [w for w in waits if text["attend.cu"][:w].endswith("__all_sync(~0u, ")]
    assert len(voted) == 1 and len(waits) == 2 and drain in text["attend.cu"]
    t = text["attend_prompt.cu"]
    assert len(re.findall(r"mbar_park\(|wait\([A-Z]+_FULL", t)) >= 8
    way_out = r"(?:mbar_park|wait)\((?:[^;{}]|\([^()]*\))*\)\s*(?:break|return|continue)|if \(!ok\)|&& ok; \+\+|&& ok\)\s*break"
    assert not re.search(way_out, t), re.search(way_out, t).group(0)
