"""The backward of the recurrence counts on as many blocks of an SM as its shared memory lets run: two of the convex backward of a 16-bit type,
which stages four inputs, three of the others."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_12128_b200", "csrc")


def test_launch_bounds_and_schedule_go_by_shared_memory():
    """The figures follow from the kernel's constants; the source asserts them at every build, and nothing counts on three blocks by itself."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hla_scan.cu")).read())
    number = lambda name: int(re.search(rf"constexpr int {name} = (\d+)", text).group(1))
    threads, lanes = number("kThreads"), number("kLanes")
    runs, tile = threads // lanes, 2 * lanes
    exchange = 3 * runs // 2 * lanes * 8 + 2 * number("kMaxCluster") * tile * 8 + 16
    def blocks(size, run, inputs):
        row = tile * size
        stage = 2 * (run * row + (row if row < 128 else 0))
        return (228 << 10) // (threads // 32 * 2 * inputs * stage + -(-exchange // 128) * 128 + 1024)
    assert [blocks(2, 8, 4), blocks(2, 8, 3), blocks(4, 4, 4), blocks(4, 4, 3)] == [2, 3, 3, 4]
    assert re.search(r"struct Bwd \{[^}]*kBlocksBack<T, CONVEX>", text)
    host = text[text.index("struct hla_scan {"):]
    assert "kBlocks " not in host and "kBlocks)" not in host and "kBlocks," not in host and "kBlocks>" not in host
    for user in ("segments_of", "cluster_of"):
        body = host[host.index(f"int {user}("):]
        assert "places_of(c, back)" in body[:body.index("\n}")]


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["log", "sigmoid"])
@pytest.mark.parametrize("B,N,C,fused", [(1, 4100, 1536, True), (1, 2051, 1100, False), (1, 9000, 768, False), (1, 20000, 64, False), (1, 600, 1537, False), (3, 1030, 352, True)])
def test_convex_backward_of_a_16_bit_type(B, N, C, fused, gate):
    from test_gpu_scan import verify
    verify(B, N, C, "bf16", gate, True, carry=N % 2 == 0, fused=fused, seed=N)
