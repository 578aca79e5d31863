// Host-side argument checks shared by the entry points.
#pragma once
#include "common.h"

namespace tsm {

struct Span {             // a tensor argument; bytes == 0 or p == null: absent
    const void* p;
    size_t bytes;
    const char* name;
};

inline bool spans_overlap(const Span& a, const Span& b) {
    if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return x < y + b.bytes && y < x + a.bytes;
}

// Alignment of every tensor, and no output over an input or another output.
inline int check_spans(const char* who, const Span* in, int nin, const Span* out, int nout) {
    for (int i = 0; i < nin; ++i)
        if (!aligned16(in[i].p)) return fail(TSM_ERR_ALIGN, "%s: %s must be 16-byte aligned", who, in[i].name);
    for (int i = 0; i < nout; ++i) {
        if (!aligned16(out[i].p)) return fail(TSM_ERR_ALIGN, "%s: %s must be 16-byte aligned", who, out[i].name);
        for (int j = 0; j < nin; ++j)
            if (spans_overlap(out[i], in[j])) return fail(TSM_ERR_SHAPE, "%s: %s and %s overlap", who, out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            if (spans_overlap(out[i], out[j])) return fail(TSM_ERR_SHAPE, "%s: %s and %s overlap", who, out[i].name, out[j].name);
    }
    return TSM_OK;
}

}  // namespace tsm
