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
    int* status;                                             // or null, see packed_status
};


// The tcgen05 kernel (attention_packed_tc.cu); a.kv_rows > 0.  splits > 1: that many units share a tile pair's keys and leave their parts in the
// workspace (packed_tc_workspace bytes), where a second kernel joins them.
size_t packed_tc_workspace(const PackedArgs& a, int head_dim, int splits);
cudaError_t launch_packed_tc(const Launch& L, const PackedArgs& a, int head_dim, int n_sms, int splits, void* workspace);

namespace {

// Where calls without a status word of their own leave what they find, until pm_operators_status reads it.  A word of each source file: its address
// would have to be asked of the runtime, which a first call may not do while it is captured.
__device__ int packed_status_word;
cudaError_t take_packed_status(int* found) {
    const int none = 0;
    const cudaError_t e = consumed(cudaMemcpyFromSymbol(found, packed_status_word, sizeof(int)));
    // kernels write to a word that is zero only, so none is lost in between
    return e != cudaSuccess || *found == 0 ? e : consumed(cudaMemcpyToSymbol(packed_status_word, &none, sizeof(int)));
}
__device__ __forceinline__ int* packed_status(const PackedArgs& a) { return a.status ? a.status : &packed_status_word; }

struct Segment { int q0, nq, k0, nk; };

// Rows of sequence s.  Lists that are malformed, lie outside the buffers or exceed the call's limits give a sequence without
// queries, so nothing is read or written because of them.
__device__ __forceinline__ Segment packed_segment(const PackedArgs& a, int s) {
    // all loads first: they take as long as one
    const int q0 = a.q_offsets[s], q1 = a.q_offsets[s + 1];
    const int k_at = a.kv_offsets ? a.kv_offsets[s] : q0;
    const int length = a.kv_lengths ? a.kv_lengths[s] : 0, k_next = a.kv_lengths ? 0 : a.kv_offsets ? a.kv_offsets[s + 1] : q1;
    const long long n_q = (long long)q1 - q0, n_k = a.kv_lengths ? (long long)length : (long long)k_next - k_at;
    const bool ok = q0 >= 0 && n_q >= 0 && q1 <= a.q_rows && n_q <= a.max_q && k_at >= 0 && n_k >= 0 && n_k <= a.max_kv && k_at + n_k <= a.kv_rows;
    if (!ok) {
        atomicCAS(packed_status(a), 0, (int)PM_ERR_ARG);
        return Segment{0, 0, 0, 0};
    }
    return Segment{q0, (int)n_q, k_at, (int)n_k};
}
// Keys that query j < nq of a sequence sees.
__device__ __forceinline__ int packed_visible(const Segment& g, int j, int causal) {
    return causal ? max(0, g.nk - (g.nq - 1 - j)) : g.nk;
}

}  // namespace
