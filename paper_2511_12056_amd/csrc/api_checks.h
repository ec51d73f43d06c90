// Checks of arguments that the C entry points of the training and projection sides share.
#pragma once
#include <hip/hip_runtime.h>
#include <initializer_list>
#include "../../include/pipedit_train.h"
#include "train_internal.h"

namespace pda {

inline int hip_error(hipError_t e, const char* what) { return report(PDA_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline bool bad_type(int t) { return t != PDA_F32 && t != PDA_BF16; }

// Do the ranges [a, a + na) and [b, b + nb) share a byte?
inline bool overlap(const void* a, double na, const void* b, double nb) {
    const double x = (double)reinterpret_cast<uintptr_t>(a), y = (double)reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && x < y + nb && y < x + na;
}

struct Range {
    const void* p;           // null: not there
    double bytes;
    const char* name;
};
inline int check_apart(std::initializer_list<Range> written, std::initializer_list<Range> others) {
    for (const Range& w : written)
        for (const Range& x : others)
            if (w.p && x.p && overlap(w.p, w.bytes, x.p, x.bytes)) return report(PDA_ERR_INVALID_ARG, "%s overlaps %s", w.name, x.name);
    return PDA_OK;
}

// B x H blocks of `bytes` bytes, `batch` and `head` bytes apart.
struct View {
    const void* p;           // null: not there
    int64_t bytes, B, H, batch, head;
    const char* name;
    int64_t span() const { return (B - 1) * batch + (H - 1) * head + bytes; }
};
inline View view(const void* p, int64_t n, int size, int64_t B, int64_t H, int64_t batch, int64_t head, const char* name) {
    View v{p, n * size, B, H, batch * size, head * size, name};
    if (v.head == v.bytes || H == 1) v = View{p, v.bytes * H, B, 1, v.batch, 0, name};       // one piece a batch, or one in all
    if (v.H == 1 && v.batch == v.bytes) v = View{p, v.bytes * B, 1, 1, 0, 0, name};
    return v;
}
// Do two views share a byte?  Every block of one against the blocks of the other that its place leaves.
inline bool overlap(const View& x, const View& y) {
    if (!x.p || !y.p || x.bytes == 0 || y.bytes == 0) return false;
    const int64_t from = (int64_t)(reinterpret_cast<uintptr_t>(x.p) - reinterpret_cast<uintptr_t>(y.p));
    if (from >= y.span() || from + x.span() <= 0) return false;
    const bool heads_out = y.head > y.batch;                   // the outer axis of y is the one of the larger stride
    const int64_t n1 = heads_out ? y.H : y.B, s1 = heads_out ? y.head : y.batch, n2 = heads_out ? y.B : y.H, s2 = heads_out ? y.batch : y.head;
    const int64_t span2 = (n2 - 1) * s2 + y.bytes;
    // first of the places i * s whose `len` bytes end behind `at`
    const auto first = [](int64_t at, int64_t len, int64_t s) -> int64_t { return at < len ? 0 : s == 0 ? INT64_MAX : (at - len) / s + 1; };
    for (int64_t b = 0; b < x.B; ++b)
        for (int64_t h = 0; h < x.H; ++h) {
            const int64_t at = from + b * x.batch + h * x.head, end = at + x.bytes;
            for (int64_t i = first(at, span2, s1); i < n1 && i * s1 < end; ++i) {
                const int64_t j = first(at - i * s1, y.bytes, s2);
                if (j < n2 && j * s2 < end - i * s1) return true;
                if (s1 == 0) break;
            }
        }
    return false;
}
inline int check_apart(std::initializer_list<View> written, std::initializer_list<View> others) {
    for (const View& w : written)
        for (const View& x : others)
            if (overlap(w, x)) return report(PDA_ERR_INVALID_ARG, "%s overlaps %s", w.name, x.name);
    return PDA_OK;
}

// The blocks of n elements at b * batch + h * head must not share any, whichever of the two axes is the outer one.
inline int check_blocks(int64_t B, int64_t H, int64_t batch, int64_t head, int64_t n, const char* name) {
    if (n == 0 || B == 0 || H == 0) return PDA_OK;
    if (H > 1 && head < n) return report(PDA_ERR_INVALID_ARG, "heads of %s overlap (head stride too small)", name);
    for (int64_t i = 1; i < B; ++i) {                          // block (0, h) against (i, 0); differences with h on the other side are larger
        const int64_t x = i * batch;
        if (x >= (H - 1) * head + n) break;
        int64_t h = H > 1 ? x / head : 0;                      // the nearest ones
        h = h < H - 1 ? h : H - 1;
        if (x - h * head < n || (h + 1 < H && (h + 1) * head - x < n))
            return report(PDA_ERR_INVALID_ARG, "batches of %s overlap (batch stride %lld, head stride %lld)", name, (long long)batch, (long long)head);
    }
    return PDA_OK;
}

}  // namespace pda
