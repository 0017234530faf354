"""What is done once on each device (csrc/once.h), as letting a kernel have large LDS: on every device, again after a failure, from several threads."""
import glob
import os
import subprocess

import paper_2210_12415_amd as alt

CSRC = os.path.join(os.path.dirname(alt.__file__), "csrc")

PROGRAM = r'''
#include "once.h"
#include <thread>
#include <vector>
#include <cstdio>

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main()
{
    enum status { ok = 0, bad = 3 };
    alt::OncePerDevice once;
    int calls[80] = {}, fails = 1;
    auto on = [&](int device) { return once(device, [&] { ++calls[device]; return device == 5 && fails-- > 0 ? bad : ok; }); };
    for (int round = 0; round < 3; ++round)
        for (int device : {0, 1, 7, 63}) CHECK(on(device) == ok);
    CHECK(calls[0] == 1 && calls[1] == 1 && calls[7] == 1 && calls[63] == 1);
    CHECK(on(5) == bad && on(5) == ok && on(5) == ok && calls[5] == 2);       // a failure is not remembered
    CHECK(on(64) == ok && on(64) == ok && calls[64] == 2 && on(79) == ok && calls[79] == 1);
    CHECK(on(0) == ok && calls[0] == 1 && calls[2] == 0);
    alt::OncePerDevice another;                                              // (another kernel's)
    CHECK(another(0, [&] { return bad; }) == bad);
    for (int round = 0; round < 200; ++round) {
        alt::OncePerDevice shared;
        std::atomic<int> done[8] = {}, early{0};
        std::vector<std::thread> all;
        for (int t = 0; t < 4; ++t)
            all.emplace_back([&, t] {
                for (int i = 0; i < 8; ++i) {
                    const int device = (i + t * 2) % 8;
                    shared(device, [&] { ++done[device]; return ok; });
                    if (!done[device]) ++early;
                }
            });
        for (auto &t : all) t.join();
        CHECK(early == 0);
        for (auto &d : done) CHECK(d >= 1 && d <= 4);
        for (int device = 0; device < 8; ++device) CHECK(shared(device, [&] { return bad; }) == ok);
    }
    return 0;
}
'''


def test_once_per_device(tmp_path):
    source, program = str(tmp_path / "once.cpp"), str(tmp_path / "once")
    with open(source, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + CSRC, source, "-o", program, "-pthread"], check=True)
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout


def test_every_kernel_of_large_lds_asks_on_every_device():
    """One place asks for it, by what is kept for each device."""
    asking = [os.path.basename(f) for f in sorted(glob.glob(os.path.join(CSRC, "*.h*")) + glob.glob(os.path.join(CSRC, "*.cpp"))) if "hipFuncSetAttribute" in open(f).read()]
    assert asking == ["common.h"]
