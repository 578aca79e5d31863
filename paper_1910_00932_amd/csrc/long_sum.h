// Sums of any number of values in fp32.
#pragma once
#include "common.h"

namespace tsm {

// A thread's sum: what it adds goes up a level after 64 additions, and again after 64 of those, so that a value is among at most 128 and
// n / 4096 additions in turn, where n in turn lean by up to n / 2 units of the last place for values of one sign.
struct LongSum {
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    int n = 0;
    __device__ __forceinline__ void add(float v) {
        s0 += v;
        if ((++n & 63) == 0) {
            s1 += s0;
            s0 = 0.f;
            if ((n & 4095) == 0) {
                s2 += s1;
                s1 = 0.f;
            }
        }
    }
    __device__ __forceinline__ float get() const { return s0 + (s1 + s2); }
};

}  // namespace tsm
