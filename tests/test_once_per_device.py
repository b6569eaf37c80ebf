"""Values that are made once per device, from several threads (a C++ program on the CPU)."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_04722_b200", "csrc")

PROGRAM = r"""
#include "once_per_device.h"
#include <cassert>
#include <cstdio>
#include <thread>
#include <vector>

struct Value { int a = 0, b = 0; };
using Once = kvq::OncePerDevice<Value>;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
    {   // a thread that is still filling does not touch what another has finished, and cannot be seen
        Once once;
        std::atomic<int> stage{0};
        std::thread slow([&] {
            once.make(3, [&](Value& v) {
                v.a = -1;                              // half done
                stage = 1;
                while (stage != 2) std::this_thread::yield();
                v.a = -2;
                stage = 3;
                while (stage != 4) std::this_thread::yield();
                v.a = v.b = 8;
                return 0;
            });
        });
        while (stage != 1) std::this_thread::yield();
        const Value* before = once.of(3);
        const int e = once.make(3, [](Value& v) { v.a = v.b = 7; return 0; });
        const Value* fast = once.of(3);
        const int a = fast ? fast->a : 0;
        stage = 2;
        while (stage != 3) std::this_thread::yield();
        const int again = fast ? fast->a : 0;
        stage = 4;
        slow.join();
        CHECK(before == nullptr && e == 0 && a == 7 && again == 7);
        CHECK(once.of(3) == fast && fast->a == 7 && fast->b == 7);
        CHECK(once.of(2) == nullptr && once.of(4) == nullptr);
    }
    {   // a failure is returned and leaves nothing behind; it may be tried again, and is made once then
        Once once;
        int calls = 0;
        CHECK(once.make(0, [&](Value& v) { v.a = 5; ++calls; return 11; }) == 11 && once.of(0) == nullptr);
        CHECK(once.make(0, [&](Value& v) { v.a = 6; ++calls; return 0; }) == 0 && once.of(0)->a == 6);
        CHECK(once.make(0, [&](Value& v) { v.a = 7; ++calls; return 12; }) == 0 && once.of(0)->a == 6 && calls == 2);
    }
    {   // devices out of range
        Once once;
        for (int d : {-1, Once::kDevices}) CHECK(once.make(d, [](Value&) { return 9; }) == 0 && once.of(d) == nullptr);
    }
    {   // many at once: everybody sees the same complete value as soon as its own call has returned
        for (int round = 0; round < 200; ++round) {
            Once once;
            std::vector<std::thread> threads;
            std::vector<const Value*> seen(8);
            std::atomic<int> wrong{0};
            for (int t = 0; t < 8; ++t)
                threads.emplace_back([&, t] {
                    once.make(1, [&](Value& v) { v.a = t + 1; std::this_thread::yield(); v.b = t + 1; return 0; });
                    seen[t] = once.of(1);
                    if (!seen[t] || seen[t]->a == 0 || seen[t]->a != seen[t]->b) ++wrong;
                });
            for (auto& t : threads) t.join();
            for (auto* s : seen) CHECK(s == seen[0]);
            CHECK(wrong == 0);
        }
    }
    return 0;
}
"""


@pytest.mark.parametrize("flags", [[], ["-fsanitize=thread"]])
def test_values_are_complete_and_never_change(tmp_path, flags):
    source, program = tmp_path / "once.cpp", tmp_path / "once"
    source.write_text(PROGRAM)
    built = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-pthread", *flags, "-I", CSRC, str(source), "-o", str(program)],
                           capture_output=True, text=True)
    if flags and built.returncode != 0 and "tsan" in built.stderr:
        pytest.skip("no thread sanitizer here")
    assert built.returncode == 0, built.stderr
    ran = subprocess.run([str(program)], capture_output=True, text=True, timeout=120)
    if flags and "unexpected memory mapping" in ran.stderr:
        pytest.skip("no thread sanitizer in this address space")
    assert ran.returncode == 0, ran.stdout + ran.stderr
