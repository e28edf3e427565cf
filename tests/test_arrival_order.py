"""A lane that arrives at a barrier for its warp does so behind a meeting that orders the other lanes' stores: read from the sources, since
what goes wrong otherwise is a race."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_00529_b200", "csrc")


def test_one_lane_arrives_right_behind_its_warp_s_meeting():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        lines = [re.sub(r"\s*//.*", "", line).rstrip() for line in open(path)]
        lines = [(i + 1, line) for i, line in enumerate(lines) if line.strip()]
        for (_, before), (n, line) in zip(lines, lines[1:]):
            if not re.search(r"\bmbar_arrive\w*\(", line) or "__device__" in line:
                continue
            seen += 1
            assert re.search(r"if \(lane == 0\) mbar_arrive", line) and before.strip() == "__syncwarp();", "%s:%d" % (os.path.basename(path), n)
    assert seen >= 5
