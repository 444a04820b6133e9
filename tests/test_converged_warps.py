"""`bar.sync`, `bar.arrive` and the `.aligned` cluster barriers are undefined unless all lanes of a warp execute them together.  Where lanes may
come apart before one (a lane that prepares something, a wait that ends for each lane by itself), a __syncwarp has to bring them together."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_12128_b200", "csrc")
BARRIER = re.compile(r'asm volatile\("(bar\.(?:sync|arrive)|barrier\.cluster\.(?:arrive|wait)[^;"]*\.aligned)')


def test_barriers_of_the_scan_are_reached_by_whole_warps():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hla_scan.cu")).read())
    found = list(BARRIER.finditer(text))
    assert len(found) == 4
    for m in found:
        body = text[text.rindex("{", 0, m.start()):m.start()]      # (of a function that is the barrier alone)
        if "cluster.wait" in m.group(1):
            assert "barrier.cluster.arrive" in body                 # directly behind the arrival
        assert re.match(r"\{\s*__syncwarp\(\);", body), m.group(1)


def test_a_block_of_the_scan_whose_wait_ran_out_takes_no_further_part():
    """Maps that it announced or sent after that would be counted by barriers that are still in an earlier phase."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hla_scan.cu")).read())
    start = text.index("float2 exchange(Exchange& e")
    body = text[start:text.index("\n}\n", start)]
    loop = body[body.index("for (int s = 0"):]
    assert re.search(r"if \(!lost && !tc::mbar_wait\([^{]*\{[^}]*lost = true;", loop)
    assert re.search(r"if \(!lost && lane == 0\) tc::mbar_arrive_expect_tx", loop) and re.search(r"if \(!lost\) \{[^{}]*\"st\.async", loop)
    assert len(re.findall("mbar_wait|mbar_arrive_expect_tx|st\\.async", loop)) == 3
