// What the kernels of attention over packed sequences share: arguments, and a sequence's rows read from the device lists.
#pragma once

#include "common.cuh"
#include "tcgen05_ptx.cuh"

struct PackedArgs {
    const void *q, *k, *v;
    void* out;
    long long q_stride, k_stride, v_stride, out_stride;      // elements between rows
    const int *q_offsets, *kv_offsets, *kv_lengths;
    int q_rows, kv_rows, n_seqs, max_q, max_kv;
    int heads, kv_heads, group, causal;
    float c;                                                 // scale * log2(e)
    int* status;
};


// the tcgen05 kernel (attention_packed_tc.cu); a.kv_rows > 0
cudaError_t launch_packed_tc(const Launch& L, const PackedArgs& a, int head_dim, int n_sms);

namespace {

struct Segment { int q0, nq, k0, nk; };

// Rows of sequence s.  Lists that are malformed, lie outside the buffers or exceed the call's limits give a sequence without
// queries, so nothing is read or written because of them.
__device__ __forceinline__ Segment packed_segment(const PackedArgs& a, int s) {
    const int q0 = a.q_offsets[s], q1 = a.q_offsets[s + 1];
    int k0 = q0, nk = q1 - q0;
    bool ok = q0 >= 0 && q1 >= q0 && q1 <= a.q_rows && q1 - q0 <= a.max_q;
    if (a.kv_offsets) k0 = a.kv_offsets[s];
    if (a.kv_lengths) nk = a.kv_lengths[s];
    else if (a.kv_offsets) {
        const int k1 = a.kv_offsets[s + 1];
        ok = ok && k0 >= 0 && k1 >= k0;
        nk = ok ? k1 - k0 : 0;
    }
    ok = ok && k0 >= 0 && nk >= 0 && nk <= a.max_kv && (long long)k0 + nk <= a.kv_rows;
    if (!ok) {
        atomicCAS(a.status, 0, (int)PM_ERR_ARG);
        return Segment{0, 0, 0, 0};
    }
    return Segment{q0, q1 - q0, k0, nk};
}
// Keys that query j of a sequence sees.
__device__ __forceinline__ int packed_visible(const Segment& g, int j, int causal) {
    return causal ? min(g.nk, max(0, j + 1 + g.nk - g.nq)) : g.nk;
}

}  // namespace
