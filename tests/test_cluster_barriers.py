"""The cluster barriers of the sources: an .aligned one asks that a warp's lanes execute it together, which nothing but a
__syncwarp() in front of it says (the compiler may leave lanes apart behind a branch or a loop)."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2109_12497_b200" / "csrc"


def test_a_warp_converges_in_front_of_every_aligned_cluster_barrier():
    found = 0
    for path in sorted(CSRC.glob("*.cu*")):
        text = re.sub(r"//[^\n]*", "", path.read_text())
        for m in re.finditer(r"asm\s*(?:volatile)?\s*\(\s*\"barrier\.cluster[^\"]*\.aligned", text):
            found += 1
            before = text[:m.start()].rstrip()
            assert before.endswith("__syncwarp();"), f"{path.name}: ...{before[-80:]}"
    assert found >= 3
