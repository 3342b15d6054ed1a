"""The wait of a whole warp (csrc/warp_wait.cuh), compiled for the host and run with a
thread a lane: whatever each lane's own tries say, all lanes take part in the same
votes and leave with the same answer.  A vote that a lane never comes to ends the
program with an error after a second, where a GPU would wait for good."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_02514_gb300", "csrc")

PROGRAM = r"""
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <mutex>
#include <random>
#include <thread>
#include <vector>
#include "warp_wait.cuh"

constexpr int LANES = 32;
struct Warp {  // a vote that all lanes have to come to
    std::mutex m;
    std::condition_variable cv;
    int here = 0;
    long round = 0;
    bool every = true, answer = true;
    bool all(bool x) {
        std::unique_lock<std::mutex> l(m);
        every = every && x;
        const long mine = round;
        if (++here == LANES) {
            answer = every, every = true, here = 0, ++round;
            cv.notify_all();
            return answer;
        }
        if (!cv.wait_for(l, std::chrono::seconds(1), [&] { return round != mine; })) {
            std::printf("a vote that a lane never came to\n");
            std::fflush(stdout);
            std::_Exit(2);
        }
        return answer;
    }
};

int main() {
    std::mt19937 gen(7);
    int got = 0, gave_up = 0;
    for (int rep = 0; rep < 60; ++rep) {
        // from which try on each lane sees the phase over (others: only in its slow wait, or never)
        std::vector<int> from(LANES), slow(LANES);
        const int last = rep % 3 == 0 ? 6 : 24;
        for (int i = 0; i < LANES; ++i) from[i] = gen() % last, slow[i] = rep % 5 != 4 || gen() % 8 != 0;
        Warp w;
        std::vector<int> answer(LANES), votes(LANES);
        std::vector<std::thread> t;
        for (int i = 0; i < LANES; ++i)
            t.emplace_back([&, i] {
                int tries = 0;
                const auto ready = [&] { return tries++ >= from[i]; };
                const auto all = [&](bool x) { ++votes[i]; return w.all(x); };
                answer[i] = aces::warp_wait(ready, [&] { return slow[i] != 0; }, all);
                // what follows in the kernel: another vote of all lanes
                if (w.all(answer[i] != 0) != (answer[i] != 0)) std::_Exit(3);
            });
        for (auto &x : t) x.join();
        for (int i = 1; i < LANES; ++i)
            if (answer[i] != answer[0] || votes[i] != votes[0]) return 4;
        int most = 0, all_slow = 1;
        for (int i = 0; i < LANES; ++i) most = from[i] > most ? from[i] : most, all_slow &= slow[i];
        if (answer[0] != (most < aces::WARP_TRIES || all_slow)) return 5;
        (answer[0] ? got : gave_up)++;
    }
    return got > 10 && gave_up > 2 ? 0 : 6;
}
"""


def test_lanes_stay_together(tmp_path):
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "lanes.cpp", tmp_path / "lanes"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-pthread", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_the_tensor_core_kernel_waits_so():
    """The issuing warp's wait is that one (its lanes have different work in between)."""
    text = open(os.path.join(CSRC, "kv4_many.cu")).read()
    assert "warp_wait(" in text and text.count("__all_sync") == 1
