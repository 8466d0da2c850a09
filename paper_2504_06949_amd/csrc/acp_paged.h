// What the kernels of the paged cache share: sequences, pages and the pointer search.
#pragma once

#include "acp_device.h"
#include "acp_ops_internal.h"

namespace acp {

constexpr int kFlagPage = 64;      // a page number out of range or a table too narrow
constexpr int kFlagMaxNew = 128;   // a sequence brings more rows than max_new
constexpr int kFlagScales = 256;   // the weights of a row left the range that the scales promise

// Rows and positions of a sequence, confined to the arrays of the call whatever cu and
// past hold.
struct Seq {
    int row0, n;       // packed rows row0 .. row0 + n - 1
    int past;          // position of row0
};
__device__ __forceinline__ Seq seq_of(const PagedArgs& a, int s) {
    Seq q;
    q.row0 = min(max(a.cu[s], 0), a.T);
    q.n = min(max(a.cu[s + 1], q.row0), a.T) - q.row0;
    q.past = min(max(a.past[s], 0), 0x7fffffff - q.n);
    return q;
}

// The sequence that holds packed row t, or -1: the last one that starts at or before it
__device__ __forceinline__ int sequence_of(const PagedArgs& a, int t) {
    int lo = 0, hi = a.N;                             // first s with cu[s + 1] > t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo < a.N && a.cu[lo] <= t ? lo : -1;
}

// Page n of sequence s, or -1
__device__ __forceinline__ int page_of(const PagedArgs& a, int s, int n) {
    if (n >= a.W) return -1;
    const int p = a.table[(int64_t)s * a.W + n];
    return p >= 0 && p < a.P ? p : -1;
}

__device__ __forceinline__ const double* gates_of(const PagedArgs& a, int page, int h) {
    return a.cp + ((int64_t)page * a.H + h) * 64;
}

}  // namespace acp
