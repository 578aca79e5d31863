"""What the library does once per device of a process (csrc/per_device.h), on the host: per device and not per process, again where it
failed, and by host threads that come together."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1910_00932_amd", "csrc")
MAIN = r"""
#include <thread>
#include <vector>
#include "per_device.h"
static tsm::OncePerDevice once;
static int calls[70];
static bool ask(int device, bool works) { return once(device, [&] { ++calls[device]; return works; }); }
#define CHECK(x) if (!(x)) return __LINE__
int main() {
    CHECK(ask(0, true) && ask(0, true) && calls[0] == 1);
    CHECK(calls[1] == 0 && ask(1, true) && ask(1, true) && calls[1] == 1);      // another device is another matter
    CHECK(!ask(2, false) && !ask(2, false) && calls[2] == 2);                   // what failed is not taken as done
    CHECK(ask(2, true) && ask(2, false) && calls[2] == 3);
    CHECK(ask(63, true) && ask(63, true) && calls[63] == 1 && ask(64, true) && ask(64, true) && calls[64] == 2);
    std::atomic<int> ran{0}, went{0};
    std::vector<std::thread> threads;
    for (int i = 0; i < 8; ++i)
        threads.emplace_back([&] {
            for (int d = 10; d < 60; ++d)
                if (once(d, [&] { ran += 1; return true; })) went += 1;
        });
    for (auto& t : threads) t.join();
    CHECK(went == 8 * 50 && ran >= 50 && ran <= 8 * 50);
    for (int d = 10; d < 60; ++d) CHECK(once(d, [] { return false; }));
    return 0;
}
"""


def test_once_per_device(tmp_path):
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], timeout=60)
    assert r.returncode == 0, "line %d" % r.returncode


def test_kernels_do_not_remember_their_lds_limit_per_process():
    """Every launch that needs more than the usual dynamic LDS asks per device."""
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        assert "hipFuncSetAttribute" not in text or name == "shift.hip", name
    assert open(os.path.join(CSRC, "shift.hip")).read().count("hipFuncSetAttribute") == 1
