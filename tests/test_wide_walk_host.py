"""Warps that meet at barriers leave a walk over tasks together, whichever wait runs out in whichever of them.

``csrc/lagkv_wide_walk.h`` is compiled for the host: a thread stands for a warp, a barrier that gives up after a second for one
that never would, and every wait of a task can be made to run out in one thread and not in the others."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "lagkv_wide_walk.h"
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <mutex>
#include <thread>
#include <vector>

struct Barrier {  // of n threads; gives the OR of what they bring; stuck once somebody waited in vain
    int n, here = 0, turn = 0;
    bool any = false, result = false, stuck = false;
    std::mutex mu;
    std::condition_variable cv;
    bool meet(bool bring) {
        std::unique_lock<std::mutex> lock(mu);
        any |= bring;
        if (++here == n) {
            here = 0, ++turn, result = any, any = false;
            cv.notify_all();
            return result;
        }
        const int mine = turn;
        if (!cv.wait_for(lock, std::chrono::milliseconds(1000), [&] { return turn != mine || stuck; })) stuck = true, cv.notify_all();
        return result;
    }
};

// `threads` walk `tasks` tasks of two waits and a barrier behind each; in thread `who` wait `which` (of 3 a task, the task's own
// first) runs out.  Returns the tasks that were begun in all, or -1: stuck, -2: not the same in all of them.
int walk(int threads, int tasks, int who, int which, bool together) {
    Barrier bar;
    bar.n = threads;
    std::vector<int> begun(threads, 0);
    std::vector<std::thread> pool;
    for (int t = 0; t < threads; ++t)
        pool.emplace_back([&, t] {
            bool ok = true;
            int waits = 0;
            auto wait = [&] { return !(t == who && waits++ == which); };
            auto agree = [&](bool mine) { return together ? !bar.meet(!mine) : mine; };
            for (int k = 0; k < tasks && lagkv::wide_go_on(ok, wait, agree) && !bar.stuck; ++k) {
                ++begun[t];
                for (int i = 0; i < 2; ++i) {
                    if (ok) ok = wait();
                    bar.meet(false);
                }
            }
        });
    for (auto& th : pool) th.join();
    if (bar.stuck) return -1;
    for (int n : begun)
        if (n != begun[0]) return -2;
    return begun[0];
}

int main(int argc, char** argv) {
    if (argc > 1) return walk(2, 3, 0, std::atoi(argv[1]), false) < 0 ? 3 : 0;  // each for itself
    for (int threads : {1, 2, 8})
        for (int who = 0; who < threads; ++who)
            for (int which = 0; which < 15; ++which) {
                // a task whose wait ran out is not begun, one with a wait that ran out is the last one
                const int want = which % 3 == 0 ? which / 3 : which / 3 + 1, got = walk(threads, 5, who, which, true);
                if (got != want) return std::printf("threads %d who %d which %d: %d, not %d\n", threads, who, which, got, want), 1;
            }
    return walk(8, 5, -1, 0, true) == 5 ? 0 : 2;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("walk")
    (at / "walk.cpp").write_text(SOURCE)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-pthread", f"-I{ROOT}/paper_2504_04704_b200/csrc", "-o", str(at / "walk"),
                    str(at / "walk.cpp")], check=True)
    return str(at / "walk")


def test_all_leave_together(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout)


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_each_for_itself_gets_stuck(program, which):
    """What the barrier between tasks is for: without it the others wait for one that has left."""
    assert subprocess.run([program, str(which)], timeout=60).returncode == 3


if __name__ == "__main__":
    sys.exit(pytest.main([__file__, "-q"]))
