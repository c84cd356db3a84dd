// Attention over packed sequences (pm_attention_packed):  out[j] = sum_{t < vis(j)} softmax(scale q[j].k[t]) v[t]  per query head.
//
// The rows of a (sequence, K/V head) pair are its (query, head of the group) pairs, row r = query r / group, head r % group, so
// keys and values are read once for all heads that share them.  Three kernels: attention_packed_tc_kernel (tcgen05, tiles of 256
// rows; attention_packed_tc.cu), and here
//   attention_rows_kernel   few rows (single tokens, short sequences): 16 rows per CTA, the keys split among warps and CTAs
//   attention_f32_kernel    fp32 on CUDA cores
// Both keep the running maximum m, sum l and unnormalised output O of a row in fp32 while they pass over the keys once, and join
// the parts of a row as  m = max m_i,  l = sum l_i 2^(m_i - m),  O = sum O_i 2^(m_i - m)  through shared memory, that of the
// cluster or a workspace where the keys are split among CTAs: no atomics, the order of every sum fixed.
#include <math.h>

#include <algorithm>

#include "f32x2.cuh"
#include "packed.cuh"

#define BUMP(L) do { if ((L).launches) ++*(L).launches; } while (0)

namespace {

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 16 bytes to shared memory, or zeros without a look at the source
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// ---------------------------------------------------------------------------------------
// Few rows.  A CTA of ROWS_WARPS warps owns 16 rows of a (sequence, K/V head) pair; the warps of the cluster take its keys 16 at a
// time in turn, each with a ring of its own in shared memory (cp.async, ROWS_STAGES chunks of 16 keys and values ahead; rows behind
// the last key a row of the tile sees are filled with zeros and never read), and no warp waits for another before the join.
// Both products on mma.sync m16n8k16 with the 16 rows as M: memory-bound from the first key on (a chunk of 8 KB costs about 250 issue
// slots), so the legacy tensor instructions do.
// ---------------------------------------------------------------------------------------
constexpr int ROWS_WARPS = 4;
constexpr int ROWS_STAGES = 3;
constexpr int ROWS_MAX_CLUSTER = 8;
constexpr int PACKED_TC_ROWS = 256;          // rows of a unit of the tcgen05 kernel
constexpr int ROWS_SPLIT_KEYS = 64;          // keys of a warp below which a split is not worth its part

template <int D>
struct RowsSmem {
    static constexpr int RING = ROWS_STAGES * 2 * 16 * D * 2;           // bytes of a warp's ring
    static constexpr int PART = D + 8;                                  // floats between the rows of a part
    uint8_t ring[ROWS_WARPS][RING];                                     // a warp's part takes its ring's place at the end
    float m[ROWS_WARPS][16], l[ROWS_WARPS][16];
    float o_cta[16][D];                                                 // what the cluster joins
    float m_cta[16], l_cta[16];
};

// What a split leaves of a row tile for attention_join_kernel, at ((sequence * K/V heads + head) * tiles + tile) * splits + split.
template <int D>
struct RowsPart {
    float o[16][D], m[16], l[16];
};

// cluster: CTAs that share a row tile's keys and join their parts through shared memory.  splits (without clusters): the same through `parts`.
template <int D>
__global__ void __launch_bounds__(32 * ROWS_WARPS) attention_rows_kernel(const __grid_constant__ PackedArgs a, int cluster, int splits, RowsPart<D>* parts) {
    constexpr int CH = D / 8;                                           // 16-byte pieces of a row
    using Smem = RowsSmem<D>;
    static_assert(Smem::RING >= 16 * Smem::PART * 4, "a part fits its ring");
    extern __shared__ __align__(128) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, mi = lane >> 3, l7 = lane & 7;
    const int share = cluster * splits, rank = blockIdx.x % share, in_grid = gridDim.x / share;
    const int h = blockIdx.y;
    dep_release();
    dep_wait();
    const Segment seg = packed_segment(a, blockIdx.z);
    const int rows = seg.nq * a.group, tiles = (rows + 15) / 16;
    for (int tile = blockIdx.x / share; tile < tiles; tile += in_grid) {  // the same for a whole cluster
        const int r0 = tile * 16;
        const int r_lo = min(r0 + g, rows - 1), r_hi = min(r0 + g + 8, rows - 1), r_last = min(r0 + 15, rows - 1);
        const int vis_lo = packed_visible(seg, r_lo / a.group, a.causal), vis_hi = packed_visible(seg, r_hi / a.group, a.causal);
        const int k_end = packed_visible(seg, r_last / a.group, a.causal), k_all = packed_visible(seg, r0 / a.group, a.causal);
        // query fragments from global memory; rows past the end repeat the last one and are not stored
        uint32_t qa[D / 16][4];
        {
            const bf16* lo = (const bf16*)a.q + (long long)(seg.q0 + r_lo / a.group) * a.q_stride + (h * a.group + r_lo % a.group) * D;
            const bf16* hi = (const bf16*)a.q + (long long)(seg.q0 + r_hi / a.group) * a.q_stride + (h * a.group + r_hi % a.group) * D;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const int c = ks * 16 + 2 * t;
                qa[ks][0] = *reinterpret_cast<const uint32_t*>(lo + c);
                qa[ks][1] = *reinterpret_cast<const uint32_t*>(hi + c);
                qa[ks][2] = *reinterpret_cast<const uint32_t*>(lo + c + 8);
                qa[ks][3] = *reinterpret_cast<const uint32_t*>(hi + c + 8);
            }
        }
        const uint32_t ring = smem_u32(sm.ring[warp]);
        const bf16* kp = (const bf16*)a.k + (long long)seg.k0 * a.k_stride + h * D;
        const bf16* vp = (const bf16*)a.v + (long long)seg.k0 * a.v_stride + h * D;
        const int chunks = (k_end + 15) >> 4, step = share * ROWS_WARPS;
        auto fetch = [&](int chunk, int stage) {
            const uint32_t ks = ring + (uint32_t)(stage * 2 * 16 * D * 2), vs = ks + 16 * D * 2;
#pragma unroll
            for (int i = 0; i < 16 * CH / 32; ++i) {
                const int at = i * 32 + lane, r = at / CH, c = at % CH, key = chunk * 16 + r;
                const bool real = key < k_end;
                const long long row = real ? key : 0;
                const uint32_t to = (uint32_t)(r * D * 2 + ((c ^ (r & 7)) << 4));
                copy16(ks + to, kp + row * a.k_stride + c * 8, real);
                copy16(vs + to, vp + row * a.v_stride + c * 8, real);
            }
        };
        float o[D / 8][4], m_lo = -INFINITY, m_hi = -INFINITY, l_lo = 0.f, l_hi = 0.f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        const int first = rank * ROWS_WARPS + warp;
#pragma unroll
        for (int i = 0; i < ROWS_STAGES - 1; ++i) {
            if (first + i * step < chunks) fetch(first + i * step, i);
            copy_commit();
        }
        int stage = 0;
        for (int chunk = first; chunk < chunks; chunk += step) {
            const int ahead = chunk + (ROWS_STAGES - 1) * step, ahead_stage = stage == 0 ? ROWS_STAGES - 1 : stage - 1;
            if (ahead < chunks) fetch(ahead, ahead_stage);                  // the stage read one step ago
            copy_commit();
            copy_wait<ROWS_STAGES - 1>();
            __syncwarp();
            const uint32_t ks_at = ring + (uint32_t)(stage * 2 * 16 * D * 2), vs_at = ks_at + 16 * D * 2;
            float s[2][4] = {};
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const int r = (mi >> 1) * 8 + l7, c = ks * 2 + (mi & 1);
                uint32_t b[4];
                ldsm4(ks_at + r * D * 2 + ((c ^ (r & 7)) << 4), b);
                mma16816(s[0], qa[ks], b[0], b[1]);
                mma16816(s[1], qa[ks], b[2], b[3]);
            }
            const bool whole = chunk * 16 + 16 <= k_all;
            float b_lo = m_lo, b_hi = m_hi;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = chunk * 16 + i * 8 + 2 * t + (e & 1);
                    const float x = s[i][e] * a.c;
                    s[i][e] = whole || key < (e < 2 ? vis_lo : vis_hi) ? x : -INFINITY;
                    if (e < 2) b_lo = fmaxf(b_lo, s[i][e]);
                    else b_hi = fmaxf(b_hi, s[i][e]);
                }
            b_lo = fmaxf(b_lo, __shfl_xor_sync(0xFFFFFFFFu, b_lo, 1));
            b_lo = fmaxf(b_lo, __shfl_xor_sync(0xFFFFFFFFu, b_lo, 2));
            b_hi = fmaxf(b_hi, __shfl_xor_sync(0xFFFFFFFFu, b_hi, 1));
            b_hi = fmaxf(b_hi, __shfl_xor_sync(0xFFFFFFFFu, b_hi, 2));
            if (__any_sync(0xFFFFFFFFu, b_lo > m_lo || b_hi > m_hi)) {      // a larger maximum: what is there is taken down to it
                const float f_lo = b_lo == m_lo ? 1.f : ex2(m_lo - b_lo), f_hi = b_hi == m_hi ? 1.f : ex2(m_hi - b_hi);
                m_lo = b_lo; m_hi = b_hi;
                l_lo *= f_lo; l_hi *= f_hi;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) { o[i][0] *= f_lo; o[i][1] *= f_lo; o[i][2] *= f_hi; o[i][3] *= f_hi; }
            }
            // a row that has seen nothing yet keeps -inf and adds nothing
            const float n_lo = m_lo == -INFINITY ? 0.f : m_lo, n_hi = m_hi == -INFINITY ? 0.f : m_hi;
            uint32_t pa[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float p0 = ex2(s[i][0] - n_lo), p1 = ex2(s[i][1] - n_lo), p2 = ex2(s[i][2] - n_hi), p3 = ex2(s[i][3] - n_hi);
                l_lo += p0 + p1;
                l_hi += p2 + p3;
                pa[i * 2] = pack(p0, p1);
                pa[i * 2 + 1] = pack(p2, p3);
            }
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                const int r = (mi & 1) * 8 + l7, c = n * 2 + (mi >> 1);
                uint32_t b[4];
                ldsm4_t(vs_at + r * D * 2 + ((c ^ (r & 7)) << 4), b);
                mma16816(o[2 * n], pa, b[0], b[1]);
                mma16816(o[2 * n + 1], pa, b[2], b[3]);
            }
            __syncwarp();                                                   // this stage is fetched into again at the next step
            stage = stage == ROWS_STAGES - 1 ? 0 : stage + 1;
        }
        copy_wait<0>();
        __syncwarp();
        l_lo += __shfl_xor_sync(0xFFFFFFFFu, l_lo, 1);
        l_lo += __shfl_xor_sync(0xFFFFFFFFu, l_lo, 2);
        l_hi += __shfl_xor_sync(0xFFFFFFFFu, l_hi, 1);
        l_hi += __shfl_xor_sync(0xFFFFFFFFu, l_hi, 2);
        float* part = reinterpret_cast<float*>(sm.ring[warp]);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            *reinterpret_cast<float2*>(part + g * Smem::PART + i * 8 + 2 * t) = make_float2(o[i][0], o[i][1]);
            *reinterpret_cast<float2*>(part + (g + 8) * Smem::PART + i * 8 + 2 * t) = make_float2(o[i][2], o[i][3]);
        }
        if (t == 0) {
            sm.m[warp][g] = m_lo; sm.l[warp][g] = l_lo;
            sm.m[warp][g + 8] = m_hi; sm.l[warp][g + 8] = l_hi;
        }
        __syncthreads();
        // the warps' parts: eight threads a row
        {
            constexpr int EACH = D / 8;
            const int row = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * 4;   // columns c0 .. c0 + 3 of every 32
            float m = sm.m[0][row];
#pragma unroll
            for (int w = 1; w < ROWS_WARPS; ++w) m = fmaxf(m, sm.m[w][row]);
            const float base = m == -INFINITY ? 0.f : m;
            float l = 0.f, acc[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) acc[e] = 0.f;
#pragma unroll
            for (int w = 0; w < ROWS_WARPS; ++w) {
                const float f = ex2(sm.m[w][row] - base);                   // 0 for a warp that has seen nothing
                l = fmaf(sm.l[w][row], f, l);
                const float* p = reinterpret_cast<const float*>(sm.ring[w]) + row * Smem::PART + c0;
#pragma unroll
                for (int e = 0; e < EACH; e += 4) {
                    const float4 x = *reinterpret_cast<const float4*>(p + e * 8);
                    acc[e] = fmaf(x.x, f, acc[e]); acc[e + 1] = fmaf(x.y, f, acc[e + 1]);
                    acc[e + 2] = fmaf(x.z, f, acc[e + 2]); acc[e + 3] = fmaf(x.w, f, acc[e + 3]);
                }
            }
            if (splits > 1) {
                if (r0 + row >= rows) return;                               // all tiles are in the grid
                RowsPart<D>& part = parts[((size_t)(blockIdx.z * a.kv_heads + h) * in_grid + tile) * splits + rank];
#pragma unroll
                for (int e = 0; e < EACH; e += 4) *reinterpret_cast<float4*>(&part.o[row][c0 + e * 8]) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
                if ((threadIdx.x & 7) == 0) { part.m[row] = m; part.l[row] = l; }
                return;
            }
            if (cluster == 1) {
                const int r = r0 + row;
                if (r < rows) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    bf16* to = (bf16*)a.out + (long long)(seg.q0 + r / a.group) * a.out_stride + (h * a.group + r % a.group) * D + c0;
#pragma unroll
                    for (int e = 0; e < EACH; e += 4)
                        *reinterpret_cast<uint2*>(to + e * 8) = make_uint2(pack(acc[e] * inv, acc[e + 1] * inv), pack(acc[e + 2] * inv, acc[e + 3] * inv));
                }
                if (tile + in_grid >= tiles) return;
                __syncthreads();                                            // the next tile's keys land on the parts
                continue;
            }
#pragma unroll
            for (int e = 0; e < EACH; e += 4) *reinterpret_cast<float4*>(&sm.o_cta[row][c0 + e * 8]) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
            if ((threadIdx.x & 7) == 0) { sm.m_cta[row] = m; sm.l_cta[row] = l; }
        }
        cluster_sync_all();
        // the CTAs' parts: each CTA joins 16 / cluster rows, a pair of columns per thread and turn
        const int mine = 16 / cluster;
        for (int i = threadIdx.x; i < mine * D / 2; i += 32 * ROWS_WARPS) {
            const int row = rank * mine + i / (D / 2), col = i % (D / 2) * 2, r = r0 + row;
            if (r >= rows) continue;
            float ms[ROWS_MAX_CLUSTER], m = -INFINITY;
#pragma unroll
            for (int k = 0; k < ROWS_MAX_CLUSTER; ++k)
                if (k < cluster) {
                    ms[k] = ld_cluster(mapa_cluster(smem_u32(&sm.m_cta[row]), k));
                    m = fmaxf(m, ms[k]);
                }
            const float base = m == -INFINITY ? 0.f : m;
            float l = 0.f, x = 0.f, y = 0.f;
#pragma unroll
            for (int k = 0; k < ROWS_MAX_CLUSTER; ++k)
                if (k < cluster) {
                    const float f = ex2(ms[k] - base);
                    const float2 v = ld_cluster2(mapa_cluster(smem_u32(&sm.o_cta[row][col]), k));
                    l = fmaf(ld_cluster(mapa_cluster(smem_u32(&sm.l_cta[row]), k)), f, l);
                    x = fmaf(v.x, f, x);
                    y = fmaf(v.y, f, y);
                }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<uint32_t*>((bf16*)a.out + (long long)(seg.q0 + r / a.group) * a.out_stride + (h * a.group + r % a.group) * D + col) =
                pack(x * inv, y * inv);
        }
        cluster_sync_all();                                                 // nobody leaves, or goes on, while its part is read
    }
}

// Joins the splits of a row: a CTA per row, the splits in turn over its warps, lanes over the columns (one warp per row took 6 us for 74
// splits, one read behind the other).
constexpr int JOIN_WARPS = 8;
template <int D>
__global__ void __launch_bounds__(32 * JOIN_WARPS) attention_join_kernel(const __grid_constant__ PackedArgs a, int splits, int tiles, const RowsPart<D>* parts) {
    constexpr int EACH = D / 32;
    __shared__ float so[JOIN_WARPS][D], sm[JOIN_WARPS], sl[JOIN_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y, r = blockIdx.x, tile = r >> 4, row = r & 15;
    dep_release();
    dep_wait();
    const Segment seg = packed_segment(a, blockIdx.z);
    if (r >= seg.nq * a.group) return;
    const RowsPart<D>* p = parts + ((size_t)(blockIdx.z * a.kv_heads + h) * tiles + tile) * splits;
    float m = -INFINITY, l = 0.f, o[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) o[e] = 0.f;
    for (int k = warp; k < splits; k += JOIN_WARPS) m = fmaxf(m, p[k].m[row]);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 4
    for (int k = warp; k < splits; k += JOIN_WARPS) {
        const float f = ex2(p[k].m[row] - base);
        l = fmaf(p[k].l[row], f, l);
#pragma unroll
        for (int e = 0; e < EACH; e += 2) {
            const float2 x = *reinterpret_cast<const float2*>(&p[k].o[row][lane * EACH + e]);
            o[e] = fmaf(x.x, f, o[e]);
            o[e + 1] = fmaf(x.y, f, o[e + 1]);
        }
    }
#pragma unroll
    for (int e = 0; e < EACH; e += 2) *reinterpret_cast<float2*>(&so[warp][lane * EACH + e]) = make_float2(o[e], o[e + 1]);
    if (lane == 0) { sm[warp] = m; sl[warp] = l; }
    __syncthreads();
    if (threadIdx.x >= D) return;
    float top = sm[0];
#pragma unroll
    for (int w = 1; w < JOIN_WARPS; ++w) top = fmaxf(top, sm[w]);
    const float to = top == -INFINITY ? 0.f : top;
    float x = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) {
        const float f = ex2(sm[w] - to);
        sum = fmaf(sl[w], f, sum);
        x = fmaf(so[w][threadIdx.x], f, x);
    }
    ((bf16*)a.out)[(long long)(seg.q0 + r / a.group) * a.out_stride + (h * a.group + r % a.group) * D + threadIdx.x] =
        __float2bfloat16_rn(sum == 0.f ? 0.f : x / sum);
}

// ---------------------------------------------------------------------------------------
// fp32 on CUDA cores: R rows (64, or 16 where there are few) per CTA, keys 64 at a time.  256 threads as 16 x 16: thread (ty, tx) forms
// the scores of rows ty + 16 i and keys tx + 16 j and the output of its rows at columns 4 tx + 64 j.  Rows of Q and K lie D + 4 floats
// apart, so that the 16-byte reads of eight neighbouring threads touch all banks once; with 64 rows P takes the place of K.  Products run packed, two
// results per instruction: one at a time the floating-point unit gives half its rate.
// ---------------------------------------------------------------------------------------
constexpr int F32_KEYS = 64;
template <int D, int R>
struct F32Smem {
    // Few rows: P has a place of its own, and the next keys are fetched meanwhile (8 streams of 8 / 2 heads of 64, a token each over 8000
    // keys: 40.1 -> 34.2 us).  With 64 rows two CTAs cover one another's copies, and it costs 2 %.
    static constexpr bool AHEAD = R == 16;
    float q[R][D + 4];
    float k[F32_KEYS][D + 4];            // unless AHEAD, then P: [R][F32_KEYS + 4]
    float v[F32_KEYS][D];
    float p[AHEAD ? R : 1][F32_KEYS + 4];
    float m[R], l[R];
};

template <int D, int R>
__global__ void __launch_bounds__(256, 2) attention_f32_kernel(const __grid_constant__ PackedArgs a, int cluster) {
    constexpr int RT = R / 16, DT = D / 64;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    F32Smem<D, R>& sm = *reinterpret_cast<F32Smem<D, R>*>(smem_raw);
    constexpr bool AHEAD = F32Smem<D, R>::AHEAD;
    static_assert(R * (F32_KEYS + 4) <= F32_KEYS * (D + 4), "P fits the keys");
    float (*ps)[F32_KEYS + 4] = AHEAD ? sm.p : reinterpret_cast<float (*)[F32_KEYS + 4]>(&sm.k[0][0]);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int rank = blockIdx.x % cluster, in_grid = gridDim.x / cluster, h = blockIdx.y;
    dep_release();
    dep_wait();
    const Segment seg = packed_segment(a, blockIdx.z);
    const int rows = seg.nq * a.group, tiles = (rows + R - 1) / R;
    for (int tile = blockIdx.x / cluster; tile < tiles; tile += in_grid) {
        const int r0 = tile * R;
        const int k_end = packed_visible(seg, min(r0 + R - 1, rows - 1) / a.group, a.causal);
        for (int i = threadIdx.x; i < R * D / 4; i += 256) {
            const int r = i / (D / 4), c = i % (D / 4) * 4, row = r0 + r;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row < rows)
                x = *reinterpret_cast<const float4*>((const float*)a.q + (long long)(seg.q0 + row / a.group) * a.q_stride + (h * a.group + row % a.group) * D + c);
            *reinterpret_cast<float4*>(&sm.q[r][c]) = x;
        }
        int vis[RT];
        float m[RT], l[RT];
        uint64_t o[RT][DT][2];                                              // four columns, packed
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            vis[i] = packed_visible(seg, min(r0 + ty + 16 * i, rows - 1) / a.group, a.causal);
            m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
            for (int j = 0; j < DT; ++j) o[i][j][0] = o[i][j][1] = 0ull;
        }
        // a warp (two thread rows) without a real row in it only helps to copy; the warp as a whole, for its shuffles
        const bool active = R > 16 || r0 + (ty & ~1) < rows;
        const float* kp = (const float*)a.k + (long long)seg.k0 * a.k_stride + h * D;
        const float* vp = (const float*)a.v + (long long)seg.k0 * a.v_stride + h * D;
        auto fetch = [&](bool keys, bool values, int b0) {
            if (b0 < k_end)
                for (int i = threadIdx.x; i < F32_KEYS * D / 4; i += 256) {
                    const int r = i / (D / 4), c = i % (D / 4) * 4, key = b0 + r;
                    const bool real = key < k_end;
                    const long long row = real ? key : 0;
                    if (keys) copy16(smem_u32(&sm.k[r][c]), kp + row * a.k_stride + c, real);
                    if (values) copy16(smem_u32(&sm.v[r][c]), vp + row * a.v_stride + c, real);
                }
            copy_commit();
        };
        const int hop = cluster * F32_KEYS;
        if (AHEAD) {
            fetch(true, false, rank * F32_KEYS);
            fetch(false, true, rank * F32_KEYS);
        }
        for (int b0 = rank * F32_KEYS; b0 < k_end; b0 += hop) {
            if (AHEAD) {
                copy_wait<1>();                                             // the keys
            } else {
                __syncthreads();                                            // the block before has been read
                fetch(true, true, b0);
                copy_wait<0>();
            }
            __syncthreads();
            float s[RT][4];
            if (active) {
                uint64_t s2[RT][4];                                         // sums of the even and of the odd dimensions
#pragma unroll
                for (int i = 0; i < RT; ++i) s2[i][0] = s2[i][1] = s2[i][2] = s2[i][3] = 0ull;
#pragma unroll 4
                for (int d = 0; d < D; d += 4) {
                    ulonglong2 q[RT], k[4];
#pragma unroll
                    for (int i = 0; i < RT; ++i) q[i] = *reinterpret_cast<const ulonglong2*>(&sm.q[ty + 16 * i][d]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const ulonglong2*>(&sm.k[tx + 16 * j][d]);
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s2[i][j] = fma2(q[i].y, k[j].y, fma2(q[i].x, k[j].x, s2[i][j]));
                }
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float a0, a1;
                        upk2(s2[i][j], a0, a1);
                        s[i][j] = a0 + a1;
                    }
            }
            __syncthreads();                                                // the keys have been read; P goes where they were
            if (AHEAD) fetch(true, false, b0 + hop);
            if (active) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    float bm = m[i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = b0 + tx + 16 * j < vis[i] ? s[i][j] * a.c : -INFINITY;
                        bm = fmaxf(bm, s[i][j]);
                    }
#pragma unroll
                    for (int x = 1; x < 16; x <<= 1) bm = fmaxf(bm, __shfl_xor_sync(0xFFFFFFFFu, bm, x, 16));
                    const float f = bm == m[i] ? 1.f : exp2f(m[i] - bm), base = bm == -INFINITY ? 0.f : bm;
                    m[i] = bm;
                    l[i] *= f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = exp2f(s[i][j] - base);
                        l[i] += p;
                        ps[ty + 16 * i][tx + 16 * j] = p;
                    }
#pragma unroll
                    for (int j = 0; j < DT; ++j) { o[i][j][0] = mul2(o[i][j][0], pk2(f, f)); o[i][j][1] = mul2(o[i][j][1], pk2(f, f)); }
                }
            }
            if (AHEAD) copy_wait<1>();                                      // the values
            __syncthreads();
            if (active) {
#pragma unroll 2
                for (int t = 0; t < F32_KEYS; t += 4) {
                    float4 p[RT];
#pragma unroll
                    for (int i = 0; i < RT; ++i) p[i] = *reinterpret_cast<const float4*>(&ps[ty + 16 * i][t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint64_t w[RT];
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            const float x = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
                            w[i] = pk2(x, x);
                        }
#pragma unroll
                        for (int j = 0; j < DT; ++j) {
                            const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&sm.v[t + e][4 * tx + 64 * j]);
#pragma unroll
                            for (int i = 0; i < RT; ++i) {
                                o[i][j][0] = fma2(w[i], v.x, o[i][j][0]);
                                o[i][j][1] = fma2(w[i], v.y, o[i][j][1]);
                            }
                        }
                    }
                }
            }
            if (AHEAD) {
                __syncthreads();                                            // the block has been read
                fetch(false, true, b0 + hop);
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], x, 16);
        auto address = [&](int row, int col) {
            return (float*)a.out + (long long)(seg.q0 + row / a.group) * a.out_stride + (h * a.group + row % a.group) * D + col;
        };
        if (cluster == 1) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int row = r0 + ty + 16 * i;
                const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
                if (row < rows)
#pragma unroll
                    for (int j = 0; j < DT; ++j)
                        *reinterpret_cast<ulonglong2*>(address(row, 4 * tx + 64 * j)) = make_ulonglong2(mul2(o[i][j][0], pk2(inv, inv)), mul2(o[i][j][1], pk2(inv, inv)));
            }
            if (tile + in_grid >= tiles) return;
            __syncthreads();                                                // the next tile's queries take the place of these
            continue;
        }
        // parts: O where the queries were
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
#pragma unroll
            for (int j = 0; j < DT; ++j) *reinterpret_cast<ulonglong2*>(&sm.q[ty + 16 * i][4 * tx + 64 * j]) = make_ulonglong2(o[i][j][0], o[i][j][1]);
            if (tx == 0) { sm.m[ty + 16 * i] = m[i]; sm.l[ty + 16 * i] = l[i]; }
        }
        cluster_sync_all();
        const int mine = R / cluster;
        for (int i = threadIdx.x; i < mine * D / 2; i += 256) {
            const int row = rank * mine + i / (D / 2), col = i % (D / 2) * 2;
            if (r0 + row >= rows) continue;
            float top = -INFINITY;
            for (int k = 0; k < cluster; ++k) top = fmaxf(top, ld_cluster(mapa_cluster(smem_u32(&sm.m[row]), k)));
            const float base = top == -INFINITY ? 0.f : top;
            float sum = 0.f, x = 0.f, y = 0.f;
            for (int k = 0; k < cluster; ++k) {
                const float f = exp2f(ld_cluster(mapa_cluster(smem_u32(&sm.m[row]), k)) - base);
                const float2 v = ld_cluster2(mapa_cluster(smem_u32(&sm.q[row][col]), k));
                sum = fmaf(ld_cluster(mapa_cluster(smem_u32(&sm.l[row]), k)), f, sum);
                x = fmaf(v.x, f, x);
                y = fmaf(v.y, f, y);
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            *reinterpret_cast<float2*>(address(r0 + row, col)) = make_float2(x * inv, y * inv);
        }
        cluster_sync_all();
    }
}

// The lists of a call that leaves no row to attend (max_q or q_rows 0): sequences that have queries all the same, or are malformed, are reported as by
// the other kernels.
__global__ void check_lists_kernel(const __grid_constant__ PackedArgs a) {
    dep_release();
    dep_wait();
    const int s = blockIdx.x * blockDim.x + threadIdx.x;
    if (s < a.n_seqs) packed_segment(a, s);
}

// CTAs that share the keys of a row tile: while the grid leaves room for them and each still has `least` keys; and of long histories, whose
// lengths may differ, up to eight times as many CTAs as run at once, each with `even` keys still, so that they end together (48 streams of
// up to 8192 keys: 133 us with a CTA each, 126 with two, 118 with four)
constexpr int ROWS_EVEN_KEYS = 512, F32_EVEN_KEYS = 256;
int key_split(long long ctas, long long slots, int max_kv, int least, int even) {
    int c = 1;
    while (c < ROWS_MAX_CLUSTER && ((ctas * c * 2 <= slots && (long long)max_kv >= 2ll * c * least) ||
                                    (ctas * c * 2 <= 8 * slots && (long long)max_kv >= 2ll * c * even)))
        c *= 2;
    return c;
}

// Row tiles that a call has: as many as the longest sequence may have for each, or those that the rows of the buffer can fill.
long long tiles_of(const PackedArgs& a, int tiles, int rows) {
    return std::min((long long)tiles * a.n_seqs, (long long)a.q_rows * a.group / rows + a.n_seqs);
}
// Tiles per sequence in the grid.  A CTA without a tile costs 1 ns, so with a limit far above the lengths (max_q = all rows, say) the empty
// ones would take the time.  So no more than four times the CTAs that the rows can fill, or 16384; a longer sequence's CTAs take several
// tiles in turn (512 frames of 197 tokens, 12 heads of 64, fp32, max_q 100864: 16.2 -> 3.0 ms, 2.9 with max_q 197).
int tiles_in_grid(const PackedArgs& a, int tiles, int rows, int share) {
    const long long each = std::max(4 * tiles_of(a, tiles, rows) / a.n_seqs, 16384ll / ((long long)share * a.kv_heads * a.n_seqs));
    return (int)std::min((long long)tiles, std::max(each, 1ll));
}

// How the keys of a row tile are shared: a cluster joins in shared memory, up to eight CTAs; where even those leave most of the GPU idle and
// there is a workspace, any number of CTAs leave their parts there and a second kernel joins them.
struct RowsForm { int tiles, cluster, splits; };
RowsForm rows_form(const PackedArgs& a, int n_sms, bool workspace) {
    const int tiles = (int)(((long long)a.max_q * a.group + 15) / 16);
    const long long ctas = tiles_of(a, tiles, 16) * a.kv_heads, slots = 2ll * n_sms;
    RowsForm f = {tiles, key_split(ctas, slots, a.max_kv, 16 * ROWS_WARPS, ROWS_EVEN_KEYS), 1};
    if (workspace && f.cluster == ROWS_MAX_CLUSTER && ctas * f.cluster * 2 <= slots) {
        const long long splits = std::min(slots / ctas, (long long)a.max_kv / (ROWS_SPLIT_KEYS * ROWS_WARPS));
        if (splits >= 2 * ROWS_MAX_CLUSTER) return {tiles, 1, (int)splits};
    }
    f.tiles = tiles_in_grid(a, tiles, 16, f.cluster);
    return f;
}
// What both kernels take, in us, as measured on a B200 (twenty shapes of 1 to 256 sequences, 16 to 1024 rows per K/V head and 17 to 16000 keys:
// within a third of either kernel's time, and the faster one is chosen in every one of them).  Units of uneven length are taken for even ones: 985 to 250 new
// tokens of four streams over up to 4985 keys, 12 / 4 heads of 64, are 66 here and 55 with their keys cut in two, and take 77 either way.
//   16-row tiles:  3, joining 2 (4 through a workspace), 0.001 for a CTA without a tile; one with a tile 0.55 and per 16 keys 0.07 (head dim 64)
//                  or 0.15 (128) beside another on its multiprocessor, 1.6 times that alone
//   tcgen05:       5, joining 4 and what the parts take at 4 TB/s; a unit of 256 rows 1.3 and per block of 64 keys 0.76, whatever its rows: two
//                  tiles' chains of dependent steps.  Units of unequal length (causal order) fill the multiprocessors by falling length, equal ones in rounds,
//                  and the longest one is a bound (a limit above four times the mean length is taken for a loose one).
// Lengths are the call's limits, or what the buffers hold per sequence; in causal order a query sees all keys but half of the queries' on average.
struct PackedWork { double seqs, queries, keys, seen; };
PackedWork packed_work(const PackedArgs& a) {
    const double seqs = a.n_seqs, queries = std::min(seqs * a.max_q, (double)a.q_rows), keys = std::min((double)a.max_kv, a.kv_rows / seqs);
    return {seqs, queries, keys, a.causal ? keys - std::min(keys, queries / seqs) / 2 : keys};
}
double rows_time(const PackedArgs& a, int head_dim, const RowsForm& f, int n_sms) {
    const PackedWork w = packed_work(a);
    const double share = (double)f.cluster * f.splits, all = w.seqs * f.tiles * a.kv_heads * share;
    const double ctas = std::min(w.seqs * ((a.max_q * (double)a.group + 15) / 16), w.queries * a.group / 16 + w.seqs) * a.kv_heads * share;
    const double per_16 = (head_dim == 64 ? 0.07 : 0.15) * (ctas < n_sms ? 1.6 : 1.0);
    return 3.0 + (f.splits > 1 ? 4.0 : f.cluster > 1 ? 2.0 : 0.0) + std::max(ctas / n_sms, 1.0) * (0.55 + per_16 * w.seen / (16.0 * share)) + 1e-3 * std::max(all - ctas, 0.0);
}
double tc_time(const PackedArgs& a, int head_dim, int splits, int n_sms) {
    const PackedWork w = packed_work(a);
    const double per_unit = PACKED_TC_ROWS / a.group * a.group;
    const double units = std::min(w.seqs * ceil((double)a.max_q * a.group / per_unit), w.queries * a.group / per_unit + w.seqs) * a.kv_heads * splits;
    auto unit = [&](double keys) { return 1.3 + 0.76 * ceil(ceil(keys / 64.0) / splits); };
    const double run = std::max(unit(std::min((double)a.max_kv, 4 * w.keys)), w.seen < w.keys ? units / n_sms * unit(w.seen) : ceil(units / n_sms) * unit(w.keys));
    return 5.0 + run + (splits > 1 ? 4.0 + (double)packed_tc_workspace(a, head_dim, splits) * 2 / 4e6 : 0.0);
}
// units that share a tile pair's keys, with a workspace of that size
constexpr int TC_MAX_SPLITS = 8;
constexpr size_t TC_MAX_WORKSPACE = (size_t)256 << 20;
int tc_splits(const PackedArgs& a, int head_dim, int n_sms, size_t bytes) {
    int best = 1;
    for (int s = 2; s <= TC_MAX_SPLITS; ++s)
        if (packed_tc_workspace(a, head_dim, s) <= std::min(bytes, TC_MAX_WORKSPACE) && tc_time(a, head_dim, s, n_sms) < 0.9 * tc_time(a, head_dim, best, n_sms)) best = s;
    return best;
}
size_t rows_workspace(const PackedArgs& a, int head_dim, const RowsForm& f) {
    if (f.splits == 1) return 0;
    return (size_t)a.n_seqs * a.kv_heads * f.tiles * f.splits * (head_dim == 64 ? sizeof(RowsPart<64>) : sizeof(RowsPart<128>));
}

template <int D>
cudaError_t launch_rows(const Launch& L, const PackedArgs& a, const RowsForm& f, void* workspace) {
    RowsPart<D>* parts = (RowsPart<D>*)workspace;
    static SmemGrant grant;
    if (cudaError_t e = grant.ensure(attention_rows_kernel<D>, (int)sizeof(RowsSmem<D>)); e != cudaSuccess) return e;
    ProfScope ps(L, KC_ATTENTION);
    cudaError_t e = launch_overlapped(L, attention_rows_kernel<D>, dim3(f.tiles * f.cluster * f.splits, a.kv_heads, a.n_seqs), 32 * ROWS_WARPS, sizeof(RowsSmem<D>),
                                      f.cluster, a, f.cluster, f.splits, parts);
    BUMP(L);
    if (e != cudaSuccess || f.splits == 1) return e;
    e = launch_overlapped(L, attention_join_kernel<D>, dim3(a.max_q * a.group, a.kv_heads, a.n_seqs),
                          32 * JOIN_WARPS, 0, 1, a, f.splits, f.tiles, (const RowsPart<D>*)parts);
    BUMP(L);
    return e;
}
struct F32Form { int rows, tiles, cluster; };
F32Form f32_form(const PackedArgs& a, int n_sms) {
    const long long rows = (long long)a.max_q * a.group;
    F32Form f = {rows <= 16 ? 16 : 64, 0, 1};
    f.tiles = (int)((rows + f.rows - 1) / f.rows);
    f.cluster = key_split(tiles_of(a, f.tiles, f.rows) * a.kv_heads, 2ll * n_sms, a.max_kv, F32_KEYS, F32_EVEN_KEYS);
    f.tiles = tiles_in_grid(a, f.tiles, f.rows, f.cluster);
    return f;
}
template <int D, int R>
cudaError_t launch_f32(const Launch& L, const PackedArgs& a, const F32Form& f) {
    static SmemGrant grant;
    if (cudaError_t e = grant.ensure(attention_f32_kernel<D, R>, (int)sizeof(F32Smem<D, R>)); e != cudaSuccess) return e;
    ProfScope ps(L, KC_ATTENTION);
    cudaError_t e = launch_overlapped(L, attention_f32_kernel<D, R>, dim3(f.tiles * f.cluster, a.kv_heads, a.n_seqs), 256, sizeof(F32Smem<D, R>), f.cluster, a, f.cluster);
    BUMP(L);
    return e;
}

bool heads_ok(const void* p, long long stride, int heads, int dim, int dtype) {
    return p && ((uintptr_t)p & 15) == 0 && stride >= (long long)heads * dim && stride % (dtype == 0 ? 8 : 4) == 0;
}

// Whether 16-row tiles serve a bf16 call with that much workspace; their form, and the units that share keys otherwise.
bool bf16_form(const PackedArgs& a, int head_dim, int n_sms, size_t bytes, RowsForm& f, int& splits) {
    f = rows_form(a, n_sms, true);
    if (bytes < rows_workspace(a, head_dim, f)) f = rows_form(a, n_sms, false);
    splits = 1;
    if (a.kv_rows == 0) return true;
    splits = tc_splits(a, head_dim, n_sms, bytes);
    return rows_time(a, head_dim, f, n_sms) < tc_time(a, head_dim, splits, n_sms);
}

// scores are taken to powers of two
constexpr float LOG2E = 1.4426950408889634f;

// Checks everything the host can see; PM_OK with nothing to attend leaves a.heads 0, and a.n_seqs is then the number of lists to check.
int packed_args(const pm_packed_attention* p, PackedArgs& a) {
    if (!p || p->q_rows < 0 || p->kv_rows < 0 || p->n_seqs < 0 || p->max_q < 0 || p->max_kv < 0 || p->heads <= 0 || p->kv_heads <= 0 ||
        p->heads % p->kv_heads || (p->head_dim != 64 && p->head_dim != 128) || (p->dtype != 0 && p->dtype != 1) || !(p->scale >= 0.f) || !isfinite(p->scale * LOG2E))
        return PM_ERR_ARG;
    if (p->n_seqs > PM_PACKED_MAX_SEQS || p->heads / p->kv_heads > PM_PACKED_MAX_GROUP || p->kv_heads > 65535 ||
        (long long)std::min(p->max_q, p->q_rows) * (p->heads / p->kv_heads) > INT32_MAX / 2)
        return PM_ERR_CAPACITY;
    a = PackedArgs{};
    a.q_offsets = p->q_offsets; a.kv_offsets = p->kv_offsets; a.kv_lengths = p->kv_lengths;
    a.q_rows = p->q_rows; a.kv_rows = p->kv_rows;
    a.max_q = std::min(p->max_q, p->q_rows);
    // Equal weights of 1 add up exactly in 32 bits to 2^24 terms and not at all from there on.  (And a unit of 2^27 keys would take longer than the bounded
    // waits allow: 0.76 us per 64.)
    a.max_kv = std::min({p->max_kv, p->kv_rows, PM_PACKED_MAX_KEYS});
    if (p->n_seqs == 0 || a.max_q == 0) {
        if (p->q_offsets && (p->kv_offsets || !p->kv_lengths)) a.n_seqs = p->n_seqs;
        return PM_OK;
    }
    a.n_seqs = p->n_seqs;
    if (!heads_ok(p->q, p->q_stride, p->heads, p->head_dim, p->dtype) || !heads_ok(p->out, p->out_stride, p->heads, p->head_dim, p->dtype) ||
        !p->q_offsets || (p->kv_lengths && !p->kv_offsets) || ((uintptr_t)p->workspace & 31))
        return PM_ERR_ARG;
    if (p->kv_rows > 0 && (!heads_ok(p->k, p->k_stride, p->kv_heads, p->head_dim, p->dtype) ||
                           !heads_ok(p->v, p->v_stride, p->kv_heads, p->head_dim, p->dtype)))
        return PM_ERR_ARG;
    a.q = p->q; a.k = p->k; a.v = p->v; a.out = p->out;
    a.q_stride = p->q_stride; a.k_stride = p->k_stride; a.v_stride = p->v_stride; a.out_stride = p->out_stride;
    a.heads = p->heads; a.kv_heads = p->kv_heads; a.group = p->heads / p->kv_heads; a.causal = p->causal != 0;
    a.c = (p->scale > 0.f ? p->scale : 1.f / sqrtf((float)p->head_dim)) * LOG2E;
    return PM_OK;
}

}  // namespace

cudaError_t packed_rows_take_status(int* found) { return take_packed_status(found); }

extern "C" {

int pm_attention_packed_workspace(const pm_packed_attention* p, int n_sms, size_t* bytes) {
    PackedArgs a;
    if (!bytes || n_sms <= 0) return PM_ERR_ARG;
    if (const int rc = packed_args(p, a); rc != PM_OK) return rc;
    *bytes = 0;
    if (a.heads > 0 && p->dtype == 0) {
        RowsForm f;
        int splits;
        *bytes = bf16_form(a, p->head_dim, n_sms, SIZE_MAX, f, splits) ? rows_workspace(a, p->head_dim, f) : packed_tc_workspace(a, p->head_dim, splits);
    }
    return PM_OK;
}

int pm_attention_packed_kernel(const pm_packed_attention* p, int n_sms, int32_t* form) {
    PackedArgs a;
    if (!form || n_sms <= 0) return PM_ERR_ARG;
    if (const int rc = packed_args(p, a); rc != PM_OK) return rc;
    form[0] = -1; form[1] = form[2] = 1;
    if (a.heads == 0) return PM_OK;
    if (p->dtype == 1) {
        const F32Form f = f32_form(a, n_sms);
        form[0] = 2; form[1] = f.cluster;
        return PM_OK;
    }
    RowsForm f;
    int splits;
    if (bf16_form(a, p->head_dim, n_sms, p->workspace ? p->workspace_bytes : 0, f, splits)) {
        form[0] = 0; form[1] = f.cluster; form[2] = f.splits;
    } else {
        form[0] = 1; form[2] = splits;
    }
    return PM_OK;
}

int pm_attention_packed(const pm_packed_attention* p, void* cuda_stream) {
    PackedArgs a;
    if (const int rc = packed_args(p, a); rc != PM_OK) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int dev = 0, n_sms = 0;
    if (const int rc = stream_device(st, &dev); rc != PM_OK) return rc;
    if (p->status_out && consumed(cudaMemsetAsync(p->status_out, 0, sizeof(int32_t), st)) != cudaSuccess) return PM_ERR_CUDA;
    a.status = p->status_out;
    Launch L;
    L.st = st;
    L.status = a.status;
    if (a.heads == 0) {
        if (a.n_seqs == 0) return PM_OK;
        return launch_overlapped(L, check_lists_kernel, (a.n_seqs + 127) / 128, 128, 0, 1, a) == cudaSuccess ? PM_OK : PM_ERR_CUDA;
    }
    if (consumed(cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return PM_ERR_CUDA;
    cudaError_t e;
    RowsForm f;
    int splits = 1;
    if (p->dtype == 1) {
        const F32Form f = f32_form(a, n_sms);
        e = p->head_dim == 64 ? (f.rows == 16 ? launch_f32<64, 16>(L, a, f) : launch_f32<64, 64>(L, a, f))
                              : (f.rows == 16 ? launch_f32<128, 16>(L, a, f) : launch_f32<128, 64>(L, a, f));
    } else if (bf16_form(a, p->head_dim, n_sms, p->workspace ? p->workspace_bytes : 0, f, splits)) {
        e = p->head_dim == 64 ? launch_rows<64>(L, a, f, p->workspace) : launch_rows<128>(L, a, f, p->workspace);
    } else {
        e = launch_packed_tc(L, a, p->head_dim, n_sms, splits, p->workspace);
    }
    return e == cudaSuccess ? PM_OK : PM_ERR_CUDA;
}

}  // extern "C"
