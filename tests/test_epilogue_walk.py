"""How the warps of an epilogue walk over their tiles, on the host: the header that the kernel uses, with threads for warps
and a barrier for theirs.  Whatever warp gives up at whatever tile, all of them come to the end."""
import os
import subprocess

from paper_2410_13056_b200 import build as cuda_build

PROGRAM = r"""
#include <atomic>
#include <barrier>
#include <cstdio>
#include <cstdlib>
#include <thread>
#include <vector>
#include "walk.cuh"

int main(int argc, char** argv) {
    const int first = atoi(argv[1]), tiles = atoi(argv[2]), step = atoi(argv[3]), warps = 8, who = atoi(argv[4]), at = atoi(argv[5]);
    std::barrier meet(warps);
    std::atomic<int> failed{0}, taken{0}, wrong{0};
    std::vector<std::thread> threads;
    for (int w = 0; w < warps; ++w)
        threads.emplace_back([&, w] {
            int seen = 0, phases[2] = {0, 0};
            cmpq::walk_tiles(
                first, tiles, step, [&](int, int) { meet.arrive_and_wait(); },
                [&](int acc, int parity) {
                    if (acc != (seen & 1) || parity != (phases[acc]++ & 1)) wrong = 1;
                    if (w == who && seen == at) return failed = 1, false;
                    ++seen;
                    return true;  // the others' accumulators were there in time
                },
                [&](int, int) { ++taken; });
        });
    for (auto& t : threads) t.join();
    printf("%d %d\n", taken.load(), wrong.load());
}
"""


def test_walk_ends_whichever_warp_gives_up(tmp_path):
    src, exe = tmp_path / "walk.cpp", str(tmp_path / "walk")
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++20", "-O1", "-pthread", "-I", cuda_build.CSRC, str(src), "-o", exe], check=True)
    assert os.path.exists(exe)
    for first, tiles, step in ((0, 1, 74), (3, 300, 74), (0, 9, 1), (5, 5, 1)):
        count = len(range(first, tiles, step))
        for who in (-1, 0, 3, 7):
            for at in {0, 1, 2, count - 1}:
                run = subprocess.run([exe] + [str(x) for x in (first, tiles, step, who, at)], capture_output=True, text=True, timeout=20)
                lost = count - at if who >= 0 and 0 <= at < count else 0
                assert run.stdout.split() == [str(8 * count - lost), "0"], (first, tiles, step, who, at, run.stdout)
