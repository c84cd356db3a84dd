// Attention over packed sequences on the tcgen05 tensor cores (bf16; the operator is described in attention_packed.cu).
//
// A persistent CTA per SM walks units: two tiles of 128 rows of a (sequence, K/V head) pair -- a row is a (query, head of the group)
// pair, so a tile holds TT = 128 / group queries of all the heads that share K and V, and the keys and values of a block serve 256
// rows.  Key blocks of 64 pass through a ring in shared memory.  Per tile and block
//     S = Q K^T             UMMA 128 x 64 x 16 steps, fp32 scores in tensor memory
//     P = 2^(c S - c m)     one row per thread: its 64 scores in registers, written back over S as packed bf16
//     O += P V              UMMA 128 x D x 16 steps, P read from tensor memory, V as an MN-major operand
//     out = O / sum         after the last block, by the same threads
// m is the row's running maximum, but it only moves when it has grown by more than 2^8 in the exponential's scale: then the thread
// takes its row of O and of the sum down to the new one (no overflow can come of the lag: terms stay below 2^8, sums below 2^8 n).
//     warps 0..3, 4..7    softmax and output of the two tiles
//     warps 8, 11         MMA issue, one tile each (one thread for both was the limit: it waits for either tile's step)
//     warp 9              units, TMA loads
//     warp 10             the rows of a value block that lie behind the sequence's last key are set to zero (at most 15 of them
//                         take part in a product, with weight zero; what lies there may be NaN)
// What bounds it is a tile's chain of dependent steps -- wait, load, maximum, exponentials, store, signal, product, scores -- and, of the
// units, the issue slots (half of them used) and the special-function unit, so a quarter of the exponentials are worked out by a cubic.
// Each tile has two buffers of scores, so that the next ones are formed meanwhile, and the tiles take turns.  Measured, 37 heads of
// 4096 tokens without causal order: head dim 64 660 TFLOP/s (tensor pipe 32 % busy), 128 1120 TFLOP/s (59 %; causal 1015): a block costs
// the softmax the same and the products twice as much.  Two CTAs per SM, sixteen softmax warps, halves of P handed on early, scores loaded
// half a block ahead and masks added in tensor memory gained nothing.
// Where units are few and the keys many, SPLIT units share a tile pair's keys and leave O, m and the sum in a workspace, which a second
// kernel joins: 256 tokens over 8000 keys of 8 / 2 heads of 128 33 us, 76 without.
// Units are visited by falling cost, there and back over the CTAs: up to PT_SORTED sequences are ranked by every CTA when it starts (more of
// them are taken in their own order).
#include <algorithm>

#include "f32x2.cuh"
#include "packed.cuh"

#define BUMP(L) do { if ((L).launches) ++*(L).launches; } while (0)

namespace {

constexpr int PT_SOFTMAX = 4;                                 // softmax warps of a tile
constexpr int PT_THREADS = 32 * (2 * PT_SOFTMAX + 4);
constexpr int PT_ROWS = 128;                                  // rows of a tile
constexpr int PT_KEYS = 64;                                   // keys of a block
constexpr int PT_SORTED = 256;                                // sequences up to which a CTA ranks them
constexpr int PT_UNITS = 4;                                   // units announced ahead
constexpr int PT_TAILS = 2 * PT_UNITS;                        // barriers of value blocks to be cleared; the loads are at most PT_UNITS units ahead of warp 10
constexpr int PT_POLY = 2;                                    // of eight pairs of exponentials, those worked out by ex2_poly
constexpr float PT_LAG = 8.f;                                 // log2 of how far a row's terms may exceed 1

template <int D>
struct PtLayout {
    static constexpr uint32_t TMEM = 512;
    static constexpr int Q_BYTES = PT_ROWS * D * 2, KV_BYTES = PT_KEYS * D * 2;       // of a tile's queries, of a K or V block
    // Query tiles in turn, a ring for each tile: a wait tells one phase of a barrier from the next only, so whoever waits on a slot has to be the one
    // whose signal frees it.
    static constexpr int Q_SLOTS = 4, KV_SLOTS = D == 64 ? 12 : 5;
    static __host__ __device__ constexpr uint32_t q_slot(int i, uint32_t use) { return 2 * i + use % 2; }
    // a tile's columns: two buffers of scores, O
    static __host__ __device__ constexpr uint32_t s_col(int i, uint32_t buffer) { return i * 256 + buffer * PT_KEYS; }
    static __host__ __device__ constexpr uint32_t o_col(int i) { return i * 256 + 2 * PT_KEYS; }
};

struct __align__(16) PtUnit {
    int q0, nq, k0, nk;                                       // the sequence
    int tok0, kv_head, blocks0, blocks1;                      // first query; key blocks of the two tiles; blocks0 < 0: no more units
    int first, part, pad[2];                                  // first key block; which of the units that share the keys
};

template <int D>
struct PtControl {
    Segment sorted[PT_SORTED];                                // by falling cost
    int before[PT_SORTED];                                    // units of the sequences ahead of it; in causal order the level of its first unit
    int many[PT_SORTED];                                      // its units
    int key[PT_SORTED], count[PT_SORTED];                     // in the caller's order: cost, units
    PtUnit units[PT_UNITS];
    unsigned long long q_full[PtLayout<D>::Q_SLOTS], q_empty[PtLayout<D>::Q_SLOTS];
    unsigned long long kv_full[PtLayout<D>::KV_SLOTS], kv_empty[PtLayout<D>::KV_SLOTS];
    // a buffer of scores each: a wait tells one phase from the next, not from the one after, and both sides may be a step ahead
    unsigned long long s_ready[2][2], p_ready[2][2], pv_done[2], o_ready[2];
    unsigned long long tail[PT_TAILS], unit_full[PT_UNITS], unit_empty[PT_UNITS];
    uint32_t tmem;
    int abort;
};
template <int D>
__host__ __device__ constexpr size_t pt_smem() {
    return (size_t)PtLayout<D>::Q_SLOTS * PtLayout<D>::Q_BYTES + (size_t)PtLayout<D>::KV_SLOTS * PtLayout<D>::KV_BYTES + sizeof(PtControl<D>);
}
static_assert(pt_smem<64>() <= 227 * 1024 && pt_smem<128>() <= 227 * 1024, "shared memory");

struct PtArgs {
    PackedArgs a;
    int tile_tokens;                                          // TT
    // parts of shared keys, at (part * q_rows + row) * heads + head: output before the division, row maximum (times c) and sum
    int splits;
    float* part_o;
    float2* part_ml;
};

// Bounded wait in which the hardware lets the warp sleep, after a look that costs less than falling asleep.
__device__ __forceinline__ uint32_t test_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
__device__ __forceinline__ uint32_t try_wait_asleep(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(20000u)                  // ns
        : "memory");
    return ok;
}
__device__ __forceinline__ bool wait_asleep(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status) {
    if (test_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (!try_wait_asleep(bar, parity)) {
        if (*abort_flag) return false;
        if (clock64() - t0 > WAIT_LIMIT_CYCLES) {
            *abort_flag = 1;
            atomicCAS(status, 0, (int)PM_ERR_TIMEOUT);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 2^x of a pair without the special-function unit: x = n + f with n whole and |f| <= 1/2 by adding a large number, 2^f by a cubic (least
// largest relative error, 2^-13.7; the rounding of P to bf16 is up to 2^-8), 2^n from the exponent bits.  x <= 127; below -126.5 the result is
// 0.  A NaN stays one.
__device__ __forceinline__ uint64_t ex2_poly(uint64_t z) {
    constexpr float BIG = 12582912.f + 127.f;                 // 1.5 * 2^23; the last bits of t hold n + 127
    float x0, x1, t0, t1;
    upk2(z, x0, x1);
    asm("max.NaN.f32 %0, %1, 0fC2FE0000;" : "=f"(x0) : "f"(x0));             // -127
    asm("max.NaN.f32 %0, %1, 0fC2FE0000;" : "=f"(x1) : "f"(x1));
    const uint64_t x = pk2(x0, x1), t = add2(x, pk2(BIG, BIG)), f = fma2(add2(t, pk2(-BIG, -BIG)), pk2(-1.f, -1.f), x);
    uint64_t p = fma2(f, pk2(0.055171322f, 0.055171322f), pk2(0.24261133f, 0.24261133f));
    p = fma2(p, f, pk2(0.69326109f, 0.69326109f));
    p = fma2(p, f, pk2(0.99992806f, 0.99992806f));
    upk2(t, t0, t1);
    return mul2(p, pk2(__uint_as_float(__float_as_uint(t0) << 23), __uint_as_float(__float_as_uint(t1) << 23)));
}
// V block as the MN-major B operand of O += P V: 64-wide pieces of the head dim lie one behind the other
template <int D>
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr) {
    return D == 64 ? smem_desc(saddr, 128)
                   : ((uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(PT_KEYS * 128 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61));
}
__device__ __forceinline__ int round16(int n) { return (n + 15) & ~15; }
// Whether the unit's last value block holds rows behind the sequence's last key that a product reads (it takes keys by 16).  That block
// lands on a barrier of its own, where warp 10 awaits it, and passes it on to those who await the ring.
__device__ __forceinline__ bool has_tail(const PtUnit& u) {
    const int blocks = max(u.blocks0, u.blocks1);
    return blocks > 0 && (u.first + blocks) * PT_KEYS > u.nk && (u.nk & 15) != 0;
}

// Key blocks of a tile whose first query is `tok` (0: no queries, or none of them sees a key).
__device__ __forceinline__ int tile_blocks(const Segment& g, int tok, int tile_tokens, int causal) {
    if (tok >= g.nq) return 0;
    return (packed_visible(g, min(tok + tile_tokens, g.nq) - 1, causal) + PT_KEYS - 1) / PT_KEYS;
}
// Keys of block j that the tile's last query sees, at most a block.
__device__ __forceinline__ int block_keys(const PtUnit& u, int tile, int j, int tile_tokens, int causal) {
    const Segment g{u.q0, u.nq, u.k0, u.nk};
    return min(PT_KEYS, packed_visible(g, min(u.tok0 + (tile + 1) * tile_tokens, u.nq) - 1, causal) - (u.first + j) * PT_KEYS);
}

template <int D, bool SPLIT>
__global__ void __launch_bounds__(PT_THREADS, 1)
attention_packed_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                           const __grid_constant__ PtArgs args) {
    using Lay = PtLayout<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t base = smem_u32(smem_raw);
    const PackedArgs& a = args.a;
    int* const status = packed_status(a);
    if (base & 1023u) {                       // swizzled operands need a 1024-byte aligned window
        if (threadIdx.x == 0) atomicCAS(status, 0, (int)PM_ERR_CUDA);
        return;
    }
    PtControl<D>& ctl = *reinterpret_cast<PtControl<D>*>(smem_raw + Lay::Q_SLOTS * Lay::Q_BYTES + Lay::KV_SLOTS * Lay::KV_BYTES);
    auto q_s = [&](int slot) { return base + (uint32_t)(slot * Lay::Q_BYTES); };
    auto kv_s = [&](int slot) { return base + (uint32_t)(Lay::Q_SLOTS * Lay::Q_BYTES + slot * Lay::KV_BYTES); };
    auto bar = [&](const unsigned long long& b) { return smem_u32(&b); };
    volatile int* abort_flag = &ctl.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int TT = args.tile_tokens;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Lay::Q_SLOTS; ++i) { mbar_init(bar(ctl.q_full[i]), 1); mbar_init(bar(ctl.q_empty[i]), 1); }
        for (int i = 0; i < Lay::KV_SLOTS; ++i) { mbar_init(bar(ctl.kv_full[i]), 1); mbar_init(bar(ctl.kv_empty[i]), 2); }
        for (int i = 0; i < 2; ++i) {
            for (int b = 0; b < 2; ++b) { mbar_init(bar(ctl.s_ready[i][b]), 1); mbar_init(bar(ctl.p_ready[i][b]), PT_SOFTMAX); }
            mbar_init(bar(ctl.pv_done[i]), 1); mbar_init(bar(ctl.o_ready[i]), 1);
        }
        for (int i = 0; i < PT_TAILS; ++i) mbar_init(bar(ctl.tail[i]), 1);
        // consumers of a unit: the softmax warps, the two issuing threads, warp 10
        for (int i = 0; i < PT_UNITS; ++i) { mbar_init(bar(ctl.unit_full[i]), 1); mbar_init(bar(ctl.unit_empty[i]), 2 * PT_SOFTMAX + 3); }
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    if (warp == 8) {
        tmem_alloc(smem_u32(&ctl.tmem), Lay::TMEM);
        tmem_relinquish();
    }
    dep_wait();                                               // everything below follows from what is read from here on
    const bool ranked = a.n_seqs <= PT_SORTED;
    const int per_unit = 2 * TT;
    if (ranked) {
        Segment g{0, 0, 0, 0};
        int key = 0, count = 0, low = 0;
        const int me = (int)threadIdx.x;
        if (me < a.n_seqs) {
            g = packed_segment(a, me);
            count = (g.nq + per_unit - 1) / per_unit;
            low = max(0, g.nk - g.nq) / per_unit;
            key = a.causal ? low + count : g.nk;
            ctl.key[me] = key;
            ctl.count[me] = count;
        }
        __syncthreads();
        if (me < a.n_seqs) {
            int rank = 0, before = 0;
            for (int k = 0; k < a.n_seqs; ++k) {
                const int other = ctl.key[k];
                if (other > key || (other == key && k < me)) { ++rank; before += ctl.count[k]; }
            }
            ctl.sorted[rank] = g;
            ctl.before[rank] = a.causal ? low : before;
            ctl.many[rank] = count;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    // only now: a kernel that starts earlier might take the tensor memory and wait for this one
    dep_release();

    // unit number n of this CTA; false once the CTA is aborting
    auto take_unit = [&](uint32_t n, PtUnit& u) {
        if (!wait_asleep(bar(ctl.unit_full[n % PT_UNITS]), (n / PT_UNITS) & 1u, abort_flag, status)) return false;
        const int4* p = reinterpret_cast<const int4*>(&ctl.units[n % PT_UNITS]);
        const int4 x = p[0], y = p[1], z = SPLIT ? p[2] : make_int4(0, 0, 0, 0);
        u = PtUnit{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, {0, 0}};
        return true;
    };

    if (warp < 2 * PT_SOFTMAX) {
        // ------------------------------------------------------------------ softmax, output
        const int tile = warp / PT_SOFTMAX, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_o = lanes + Lay::o_col(tile);
        const int row_tok = row / a.group, head_at = row % a.group * D;
        // 32-byte stores, a whole sector each, where the rows allow it
        const bool sectors = ((uintptr_t)a.out & 31) == 0 && a.out_stride % 16 == 0;
        const float c = a.c, lag = PT_LAG / a.c;
        const uint64_t c2 = pk2(c, c);
        uint32_t steps = 0, tiles = 0;                        // blocks, tiles with blocks so far
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            int blocks, vis, vis_all;                         // vis_all: keys that every row sees
            bool real;
            bf16* to;                                         // this thread's row of the output, or of its part
            long long part = 0;
            {
                PtUnit u;
                ok = take_unit(n, u);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                if (lane == 0) mbar_arrive(bar(ctl.unit_empty[n % PT_UNITS]));
                blocks = tile ? u.blocks1 : u.blocks0;
                const Segment seg{u.q0, u.nq, u.k0, u.nk};
                const int tok0 = u.tok0 + tile * TT;
                vis = packed_visible(seg, min(tok0 + row_tok, u.nq - 1), a.causal) - u.first * PT_KEYS;
                vis_all = packed_visible(seg, tok0, a.causal) - u.first * PT_KEYS;
                real = row_tok < TT && tok0 + row_tok < u.nq;
                to = (bf16*)a.out + (long long)(u.q0 + tok0 + row_tok) * a.out_stride + u.kv_head * a.group * D + head_at;
                if (SPLIT) part = ((long long)u.part * a.q_rows + u.q0 + tok0 + row_tok) * a.heads + u.kv_head * a.group + row % a.group;
                if (u.blocks0 < 0) break;
            }
            float m = -INFINITY;
            uint64_t sum0 = pk2(0.f, 0.f), sum1 = sum0;
            for (int j = 0; j < blocks; ++j, ++steps) {
                const uint32_t buffer = steps % 2, t_s = lanes + Lay::s_col(tile, buffer);
                ok = wait_asleep(bar(ctl.s_ready[tile][buffer]), (steps / 2) & 1u, abort_flag, status);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after();
                uint32_t v[PT_KEYS];
                tmem_ld32(t_s, v);
                tmem_ld32(t_s + 32, v + 32);
                tmem_ld_wait();
                // hidden keys, and columns that were not formed, count as -inf
                if (vis_all < (j + 1) * PT_KEYS) {
                    const int lim = vis - j * PT_KEYS;
#pragma unroll
                    for (int e = 0; e < PT_KEYS; ++e) v[e] = e < lim ? v[e] : 0xFF800000u;
                }
                float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < PT_KEYS; e += 2) t[(e >> 1) & 3] = max3(t[(e >> 1) & 3], __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                const float top = fmaxf(max3(t[0], t[1], t[2]), t[3]);
                if (j == 0) {
                    m = top;
                } else if (__any_sync(0xFFFFFFFFu, top > m + lag)) {
                    // what is there comes down to the new maximum, once the product before has been added
                    const float up = fmaxf(m, top), f = up == m ? 1.f : ex2f((m - up) * c);
                    m = up;
                    sum0 = mul2(sum0, pk2(f, f));
                    sum1 = mul2(sum1, pk2(f, f));
                    ok = wait_asleep(bar(ctl.pv_done[tile]), (steps - 1) & 1u, abort_flag, status);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int k = 0; k < D; k += 8) {
                        uint32_t o[8];
                        tmem_ld8(t_o + k, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st8(t_o + k, o);
                    }
                }
                const float mc = m == -INFINITY ? 0.f : -m * c;              // a row that sees nothing: all terms 0
                const uint64_t mc2 = pk2(mc, mc);
                // P of a piece lies over scores that have been read
#pragma unroll
                for (int k = 0; k < PT_KEYS; k += 32) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        uint64_t p = fma2(pk2(__uint_as_float(v[k + 2 * e]), __uint_as_float(v[k + 2 * e + 1])), c2, mc2);
                        float x, y;
                        if ((e & 7) >= 8 - PT_POLY) {
                            p = ex2_poly(p);
                            upk2(p, x, y);
                        } else {
                            upk2(p, x, y);
                            x = ex2f(x);
                            y = ex2f(y);
                            p = pk2(x, y);
                        }
                        if (e & 1) sum1 = add2(sum1, p);
                        else sum0 = add2(sum0, p);
                        pk[e] = pack_bf16(x, y);
                    }
                    tmem_st16(t_s + k / 2, pk);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.p_ready[tile][buffer]));
            }
            if (!ok) break;
            float inv = 0.f, l = 0.f;
            if (blocks > 0) {
                ok = wait_asleep(bar(ctl.o_ready[tile]), tiles & 1u, abort_flag, status);
                ++tiles;
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after();
                float x, y;
                upk2(add2(sum0, sum1), x, y);
                l = x + y;
                inv = l == 0.f ? 0.f : 1.f / l;
            }
            if constexpr (SPLIT) {
                // -inf and 0 if this part sees nothing, and then its output is not read; not so if its sum is no number
                if (real) args.part_ml[part] = make_float2(l == l ? m * c : 0.f, l);
                if (blocks > 0) {
                    float* po = args.part_o + part * D;
#pragma unroll
                    for (int k = 0; k < D; k += 32) {
                        uint32_t o[32];
                        tmem_ld32(t_o + k, o);
                        tmem_ld_wait();
                        if (real)
#pragma unroll
                            for (int e = 0; e < 32; e += 8)
                                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                                             ::"l"(po + k + e), "r"(o[e]), "r"(o[e + 1]), "r"(o[e + 2]), "r"(o[e + 3]), "r"(o[e + 4]), "r"(o[e + 5]), "r"(o[e + 6]),
                                               "r"(o[e + 7])
                                             : "memory");
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < D; k += 32) {
                    uint32_t o[32];
                    if (blocks > 0) {
                        tmem_ld32(t_o + k, o);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0u;
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = pack_bf16(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
                    if (real && sectors) {
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                                         ::"l"(to + k + 2 * e), "r"(o[e]), "r"(o[e + 1]), "r"(o[e + 2]), "r"(o[e + 3]), "r"(o[e + 4]), "r"(o[e + 5]), "r"(o[e + 6]), "r"(o[e + 7])
                                         : "memory");
                    } else if (real) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(to + k + 2 * e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                }
            }
            // O is in registers before the next unit's first P is announced, and that comes before the product that overwrites it
            tc_fence_before();
        }
    } else {
        if (warp == 8 || warp == 11) {
            if (elect_one()) {
                // -------------------------------------------------------------- MMA issue, a thread for each tile
                // Steps: key blocks of the units, in order; kv: ring position of a step's K block (V follows it).  A step that the other tile has
                // alone only passes the ring on -- not before the block has landed, or the signal would count for the slot's use before.
                struct Step { PtUnit u; int j, blocks, mine; uint32_t kv, q; };                // q: which of the tile's query tiles
                const int i = warp == 8 ? 0 : 1;
                const uint32_t idesc_pv = instr_desc_b_mn(D), idesc_s = instr_desc(PT_KEYS), t_o = tmem + Lay::o_col(i);
                uint32_t units = 0, kv_next = 0, q_next = 0, s_count = 0, p_count = 0;
                bool ok = true;
                // the step after `s`, or the next unit's first; false: none
                auto advance = [&](Step& s, bool first) {
                    if (!first && s.j + 1 < s.blocks) {
                        ++s.j;
                        s.kv = kv_next;
                        kv_next += 2;
                        return true;
                    }
                    for (;;) {                                // units without a visible key have no steps
                        ok = take_unit(units, s.u);
                        if (!ok) return false;
                        mbar_arrive(bar(ctl.unit_empty[units % PT_UNITS]));
                        ++units;
                        if (s.u.blocks0 < 0) return false;
                        s.blocks = max(s.u.blocks0, s.u.blocks1);
                        if (s.blocks > 0) break;
                    }
                    s.j = 0;
                    s.kv = kv_next;
                    kv_next += 2;
                    s.mine = i ? s.u.blocks1 : s.u.blocks0;
                    s.q = q_next;
                    if (s.mine > 0) ++q_next;
                    return true;
                };
                auto full = [&](uint32_t at) { return wait_asleep(bar(ctl.kv_full[at % Lay::KV_SLOTS]), (at / Lay::KV_SLOTS) & 1u, abort_flag, status); };
                auto scores = [&](const Step& s) {
                    const uint32_t k_slot = s.kv % Lay::KV_SLOTS;
                    if (s.j >= s.mine) {
                        ok = full(s.kv);
                        mbar_arrive(bar(ctl.kv_empty[k_slot]));
                        return;
                    }
                    const uint32_t q_slot = Lay::q_slot(i, s.q), buffer = s_count++ & 1u, to = tmem + Lay::s_col(i, buffer);
                    const uint64_t dq = smem_desc(q_s((int)q_slot), 128), dk = smem_desc(kv_s((int)k_slot), 128);
                    const uint32_t idesc = s.j + 1 < s.mine ? idesc_s : instr_desc(round16(block_keys(s.u, i, s.j, TT, a.causal)));
                    if (s.j == 0) ok = wait_asleep(bar(ctl.q_full[q_slot]), (s.q >> 1) & 1u, abort_flag, status);
                    ok = ok && full(s.kv);
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)          // 64-wide pieces of the head dim lie one behind the other
                        umma_bf16(to, dq + (uint64_t)((k / 4) * (PT_ROWS * 128 >> 4) + 2 * (k % 4)), dk + (uint64_t)((k / 4) * (PT_KEYS * 128 >> 4) + 2 * (k % 4)), idesc, k > 0);
                    umma_commit(bar(ctl.s_ready[i][buffer]));
                    umma_commit(bar(ctl.kv_empty[k_slot]));
                    if (s.j + 1 == s.mine) umma_commit(bar(ctl.q_empty[q_slot]));
                };
                auto product = [&](const Step& s) {
                    const uint32_t v_slot = (s.kv + 1) % Lay::KV_SLOTS;
                    ok = full(s.kv + 1);
                    if (s.j >= s.mine) {
                        mbar_arrive(bar(ctl.kv_empty[v_slot]));
                        return;
                    }
                    const uint32_t buffer = p_count & 1u, p = tmem + Lay::s_col(i, buffer);
                    const uint64_t dv = v_desc<D>(kv_s((int)v_slot));
                    const int pieces = s.j + 1 < s.mine ? PT_KEYS / 16 : round16(block_keys(s.u, i, s.j, TT, a.causal)) / 16;
                    const uint32_t add = s.j > 0 ? 1u : 0u;
                    ok = ok && wait_asleep(bar(ctl.p_ready[i][buffer]), (p_count++ >> 1) & 1u, abort_flag, status);
                    if (!ok) return;
                    tc_fence_after();
                    if (pieces == PT_KEYS / 16) {
#pragma unroll
                        for (int k = 0; k < PT_KEYS / 16; ++k) umma_bf16_ts(t_o, p + 8 * k, dv + 128 * k, idesc_pv, k > 0 ? 1u : add);
                    } else {
                        for (int k = 0; k < pieces; ++k) umma_bf16_ts(t_o, p + 8 * k, dv + 128 * k, idesc_pv, k > 0 ? 1u : add);
                    }
                    umma_commit(bar(ctl.pv_done[i]));
                    umma_commit(bar(ctl.kv_empty[v_slot]));
                    if (s.j + 1 == s.mine) umma_commit(bar(ctl.o_ready[i]));
                };
                // whether the K block that comes next in the ring has landed
                auto arrived = [&]() { return test_wait(bar(ctl.kv_full[kv_next % Lay::KV_SLOTS]), (kv_next / Lay::KV_SLOTS) & 1u) != 0; };
                Step cur, next;
                bool more = advance(cur, true);
                if (more) scores(cur);
                while (more && ok) {
                    // The next scores go ahead of this product (the other buffer's has been issued), unless they are another unit's that is not there yet.
                    next = cur;
                    const bool same = cur.j + 1 < cur.blocks;
                    const bool ahead = same || (test_wait(bar(ctl.unit_full[units % PT_UNITS]), (units / PT_UNITS) & 1u) && arrived());
                    if (!ahead) product(cur);
                    if (ok) more = advance(next, false);
                    if (!ok) break;
                    if (more) scores(next);
                    if (ok && ahead) product(cur);
                    cur = next;
                }
            }
        } else if (warp == 9) {
            // ------------------------------------------------------------------ units and loads
            // The walk over the units: in causal order level by level from the highest, a level holding the units that see about as many keys: unit L of a
            // sequence that begins with a history of h units' length is at level h + L; in a level 32 sequences at a time.  Without causal order sequence
            // by sequence.  `left` counts K/V heads of units from where the
            // walk stands (and the parts of each); the CTAs take them in turn, there and back, so that none has the longest of every turn.
            const int n_seqs = a.n_seqs;
            const uint32_t splits = SPLIT ? (uint32_t)args.splits : 1u, shares = (uint32_t)a.kv_heads * splits;
            auto units_of = [&](const Segment& g) { return (g.nq + per_unit - 1) / per_unit; };
            int level = 0, reach = 0, block = 0;
            bool any = false;                                 // a unit at this level, in the blocks of sequences passed so far
            const bool here = ranked && lane < n_seqs;        // the levels of this lane's sequence, of up to 32
            const int low = here ? ctl.before[lane] : 0, high = here ? low + ctl.many[lane] - 1 : -1;
            Segment mine{0, 0, 0, 0};                         // not ranked: a sequence per lane
            if (!ranked) mine = lane < n_seqs ? packed_segment(a, lane) : mine;
            else if (a.causal) level = ctl.before[0] + ctl.many[0] - 1;
            uint32_t left = blockIdx.x;                       // all units together are fewer than 2^31 (see the launch)
            uint32_t units = 0, kv = 0, q0 = 0, q1 = 0, tails = 0;
            bool ok = true;
            while (ok) {
                Segment g{0, 0, 0, 0};
                int tile = -1;                                // of the sequence, in units
                if (ranked && a.causal) {
                    if (n_seqs <= 32) {
                        // all levels at once that hold the same sequences as this one
                        while (level >= 0) {
                            const bool in = low <= level && level <= high;
                            const uint32_t set = __ballot_sync(0xFFFFFFFFu, in);
                            const int until = __reduce_max_sync(0xFFFFFFFFu, in ? low - 1 : high < level ? high : -1);
                            const uint32_t each = __popc(set) * shares, here = each * (uint32_t)(level - until);
                            if (left < here) {
                                level -= (int)(left / each);
                                left %= each;
                                break;
                            }
                            left -= here;
                            level = until;
                        }
                    }
                    while (level >= 0) {
                        const int at = block + lane, unit = at < n_seqs ? level - ctl.before[at] : -1;
                        uint32_t set = __ballot_sync(0xFFFFFFFFu, unit >= 0 && unit < (at < n_seqs ? ctl.many[at] : 0));
                        const uint32_t here = __popc(set) * shares;
                        if (left < here) {
                            for (int nth = (int)(left / shares); nth > 0; --nth) set &= set - 1;
                            const int from = __ffs((int)set) - 1;
                            g = ctl.sorted[block + from];
                            tile = __shfl_sync(0xFFFFFFFFu, unit, from);
                            any = true;
                            break;
                        }
                        left -= here;
                        any |= here > 0;
                        block += 32;
                        if (block >= n_seqs) {
                            block = 0;
                            if (any) {
                                --level;
                            } else {
                                // Below a level without units, straight to the next one that has any: histories are long and levels a few keys high where
                                // heads are grouped (33 streams of 16 tokens, 64 heads on one K/V head, one with 200000 kept: 14.5 ms level by level,
                                // 0.73 of 32 streams)
                                int next = -1;
                                for (int i = lane; i < n_seqs; i += 32) {
                                    const int high = ctl.before[i] + ctl.many[i] - 1;
                                    if (ctl.many[i] > 0 && high < level) next = max(next, high);
                                }
                                level = __reduce_max_sync(0xFFFFFFFFu, next);
                            }
                            any = false;
                        }
                    }
                } else if (ranked) {
                    const int at = (int)(left / shares);      // of all units
                    while (reach + 1 < n_seqs && ctl.before[reach + 1] <= at) ++reach;
                    g = ctl.sorted[reach];
                    if (at - ctl.before[reach] < ctl.many[reach]) tile = at - ctl.before[reach];
                } else {
                    while (block < n_seqs) {
                        const int mass = units_of(mine);
                        int sum = mass;                       // of the lanes up to this one
#pragma unroll
                        for (int x = 1; x < 32; x <<= 1) {
                            const int y = __shfl_up_sync(0xFFFFFFFFu, sum, x);
                            if (lane >= x) sum += y;
                        }
                        const uint32_t here = (uint32_t)__shfl_sync(0xFFFFFFFFu, sum, 31) * shares;
                        if (left < here) {
                            const int nth = (int)(left / shares);
                            const int from = __ffs((int)__ballot_sync(0xFFFFFFFFu, sum > nth)) - 1;
                            g = Segment{__shfl_sync(0xFFFFFFFFu, mine.q0, from), __shfl_sync(0xFFFFFFFFu, mine.nq, from), __shfl_sync(0xFFFFFFFFu, mine.k0, from),
                                        __shfl_sync(0xFFFFFFFFu, mine.nk, from)};
                            tile = nth - __shfl_sync(0xFFFFFFFFu, sum - mass, from);
                            break;
                        }
                        left -= here;
                        block += 32;
                        mine = block + lane < n_seqs ? packed_segment(a, block + lane) : Segment{0, 0, 0, 0};
                    }
                }
                PtUnit u = {0, 0, 0, 0, 0, 0, -1, -1, 0, 0, {0, 0}};
                if (tile >= 0) {
                    u.q0 = g.q0; u.nq = g.nq; u.k0 = g.k0; u.nk = g.nk;
                    u.tok0 = tile * per_unit;
                    u.kv_head = (int)(left % shares / splits);
                    u.part = SPLIT ? (int)(left % splits) : 0;
                    const int all0 = tile_blocks(g, u.tok0, TT, a.causal), all1 = tile_blocks(g, u.tok0 + TT, TT, a.causal), all = max(all0, all1);
                    u.first = SPLIT ? (int)((long long)all * u.part / splits) : 0;
                    const int end = SPLIT ? (int)((long long)all * (u.part + 1) / splits) : all;
                    u.blocks0 = max(0, min(all0, end) - u.first);
                    u.blocks1 = max(0, min(all1, end) - u.first);
                    left += 2 * ((units & 1u) ? blockIdx.x : gridDim.x - 1 - blockIdx.x) + 1;
                }
                const int at = (int)(units % PT_UNITS);
                ok = wait_asleep(bar(ctl.unit_empty[at]), ((units / PT_UNITS) & 1u) ^ 1u, abort_flag, status);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                if (lane == 0) {
                    int4* p = reinterpret_cast<int4*>(&ctl.units[at]);
                    p[0] = make_int4(u.q0, u.nq, u.k0, u.nk);
                    p[1] = make_int4(u.tok0, u.kv_head, u.blocks0, u.blocks1);
                    if (SPLIT) p[2] = make_int4(u.first, u.part, 0, 0);
                    mbar_arrive(bar(ctl.unit_full[at]));
                }
                __syncwarp();
                ++units;
                if (u.blocks0 < 0) break;
                const int blocks = max(u.blocks0, u.blocks1);
                const bool tail = has_tail(u);
                if (elect_one()) {
                    auto load_q = [&](int i) {
                        uint32_t& use = i ? q1 : q0;
                        const int slot = (int)Lay::q_slot(i, use);
                        ok = ok && wait_asleep(bar(ctl.q_empty[slot]), ((use >> 1) & 1u) ^ 1u, abort_flag, status);
                        if (!ok) return;
                        mbar_expect_tx(bar(ctl.q_full[slot]), (uint32_t)(TT * a.group * D * 2));
                        for (int x = 0; x < D / 64; ++x)
                            tma_load_3d(q_s(slot) + x * PT_ROWS * 128, &tm_q, x * 64, u.kv_head * a.group, u.q0 + u.tok0 + i * TT, bar(ctl.q_full[slot]));
                        ++use;
                    };
                    auto load_kv = [&](const CUtensorMap* tm, int j, unsigned long long* full) {
                        const int slot = (int)(kv % Lay::KV_SLOTS);
                        ok = ok && wait_asleep(bar(ctl.kv_empty[slot]), ((kv / Lay::KV_SLOTS) & 1u) ^ 1u, abort_flag, status);
                        if (!ok) return;
                        const uint32_t on = full ? bar(*full) : bar(ctl.kv_full[slot]);
                        mbar_expect_tx(on, (uint32_t)Lay::KV_BYTES);
                        for (int x = 0; x < D / 64; ++x) tma_load_3d(kv_s(slot) + x * PT_KEYS * 128, tm, x * 64, u.kv_head, u.k0 + (u.first + j) * PT_KEYS, on);
                        ++kv;
                    };
                    for (int j = 0; j < blocks && ok; ++j) {
                        if (j == 0 && u.blocks0 > 0) load_q(0);
                        load_kv(&tm_k, j, nullptr);
                        if (j == 0 && u.blocks1 > 0) load_q(1);
                        load_kv(&tm_v, j, tail && j == blocks - 1 ? &ctl.tail[tails % PT_TAILS] : nullptr);
                    }
                }
                tails += tail ? 1u : 0u;
                ok = __all_sync(0xFFFFFFFFu, ok);
                // the counters of the lane that loaded
                kv = __reduce_max_sync(0xFFFFFFFFu, kv);
                q0 = __reduce_max_sync(0xFFFFFFFFu, q0);
                q1 = __reduce_max_sync(0xFFFFFFFFu, q1);
            }
        } else if (warp == 10) {
            // ------------------------------------------------------------------ values behind a sequence's last key
            uint32_t kv = 0, tails = 0;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                PtUnit u;
                ok = take_unit(n, u);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                if (lane == 0) mbar_arrive(bar(ctl.unit_empty[n % PT_UNITS]));
                if (u.blocks0 < 0) break;
                const int blocks = max(u.blocks0, u.blocks1);
                kv += 2 * (uint32_t)blocks;
                if (!has_tail(u)) continue;
                const int slot = (int)((kv - 1) % Lay::KV_SLOTS);
                ok = wait_asleep(bar(ctl.tail[tails % PT_TAILS]), (tails / PT_TAILS) & 1u, abort_flag, status);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                ++tails;
                const int first = u.nk - (u.first + blocks - 1) * PT_KEYS, rows = round16(first) - first;
                for (int i = lane; i < rows * D / 8; i += 32) {              // whole rows, so their swizzle does not matter
                    const int r = first + i / (D / 8), c = i % (D / 8);
                    st_shared_v4(kv_s(slot) + (uint32_t)((c / 8) * PT_KEYS * 128 + r * 128 + (c % 8) * 16), make_uint4(0, 0, 0, 0));
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.kv_full[slot]));
            }
        }
    }

    // -------------------------------------------------------------------------- teardown
    __syncwarp();
    dep_wait();               // never finish before the kernel this one was allowed to overtake
    if (*abort_flag) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);    // let copies / MMAs in flight land
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, Lay::TMEM);
    }
}

// Joins the parts of a row: a warp per (query, head).
constexpr int PT_JOIN_WARPS = 8;
template <int D>
__global__ void __launch_bounds__(32 * PT_JOIN_WARPS) attention_join_tc_kernel(const __grid_constant__ PtArgs args) {
    constexpr int EACH = D / 32;
    const PackedArgs& a = args.a;
    const int lane = threadIdx.x & 31;
    dep_release();
    dep_wait();
    const Segment g = packed_segment(a, blockIdx.y);
    const long long stride = (long long)a.q_rows * a.heads;
    for (long long i = (long long)blockIdx.x * PT_JOIN_WARPS + (threadIdx.x >> 5); i < (long long)g.nq * a.heads; i += (long long)gridDim.x * PT_JOIN_WARPS) {
        const long long at = (long long)g.q0 * a.heads + i;
        float m = -INFINITY;
        for (int k = 0; k < args.splits; ++k) m = fmaxf(m, args.part_ml[k * stride + at].x);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f, o[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) o[e] = 0.f;
        for (int k = 0; k < args.splits; ++k) {
            const float2 ml = args.part_ml[k * stride + at];
            if (ml.x == -INFINITY) continue;                  // saw nothing, left no output
            const float f = ex2f(ml.x - base);
            l = fmaf(ml.y, f, l);
#pragma unroll
            for (int e = 0; e < EACH; e += 2) {
                const float2 x = *reinterpret_cast<const float2*>(args.part_o + (k * stride + at) * D + lane * EACH + e);
                o[e] = fmaf(x.x, f, o[e]);
                o[e + 1] = fmaf(x.y, f, o[e + 1]);
            }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16* to = (bf16*)a.out + (g.q0 + i / a.heads) * a.out_stride + i % a.heads * D + lane * EACH;
#pragma unroll
        for (int e = 0; e < EACH; e += 2) *reinterpret_cast<uint32_t*>(to + e) = pack_bf16(o[e] * inv, o[e + 1] * inv);
    }
}

template <int D>
cudaError_t launch_tc(const Launch& L, const PackedArgs& a, int n_sms, int splits, void* workspace) {
    PtArgs args = {};
    args.a = a;
    args.tile_tokens = PT_ROWS / a.group;
    args.splits = splits;
    if (splits > 1) {
        args.part_o = (float*)workspace;
        args.part_ml = (float2*)(args.part_o + (size_t)splits * a.q_rows * a.heads * D);
    }
    CUtensorMap tm_q, tm_k, tm_v;
    if (!tm_encode_3d(&tm_q, a.q, D, a.heads, a.q_rows, D * 2, (uint64_t)a.q_stride * 2, 64, a.group, args.tile_tokens, 128) ||
        !tm_encode_3d(&tm_k, a.k, D, a.kv_heads, a.kv_rows, D * 2, (uint64_t)a.k_stride * 2, 64, 1, PT_KEYS, 128) ||
        !tm_encode_3d(&tm_v, a.v, D, a.kv_heads, a.kv_rows, D * 2, (uint64_t)a.v_stride * 2, 64, 1, PT_KEYS, 128))
        return cudaErrorInvalidValue;
    static SmemGrant grant[2];
    const auto kernel = splits > 1 ? attention_packed_tc_kernel<D, true> : attention_packed_tc_kernel<D, false>;
    if (cudaError_t e = grant[splits > 1].ensure(kernel, (int)pt_smem<D>()); e != cudaSuccess) return e;
    const long long units = (a.q_rows / (2 * args.tile_tokens) + (long long)a.n_seqs) * a.kv_heads * splits;         // at most
    if (units >= 1ll << 31) return cudaErrorInvalidValue;
    ProfScope ps(L, KC_ATTENTION);
    cudaError_t e = launch_overlapped(L, kernel, dim3((unsigned)std::min<long long>(units, n_sms)), PT_THREADS, pt_smem<D>(), 1, tm_q, tm_k,
                                      tm_v, args);
    BUMP(L);
    if (e != cudaSuccess || splits == 1) return e;
    // a warp per row of the longest sequence, but where the limit is far above the sequences' mean not more than 16 times the warps that all rows
    // need: those of shorter sequences find nothing to do
    const long long rows = std::min((long long)a.max_q * a.heads, ((long long)a.q_rows * a.heads * 16 + a.n_seqs - 1) / a.n_seqs);
    e = launch_overlapped(L, attention_join_tc_kernel<D>, dim3((unsigned)((rows + PT_JOIN_WARPS - 1) / PT_JOIN_WARPS), a.n_seqs), 32 * PT_JOIN_WARPS, 0, 1, args);
    BUMP(L);
    return e;
}

}  // namespace

size_t packed_tc_workspace(const PackedArgs& a, int head_dim, int splits) {
    return splits > 1 ? (size_t)splits * a.q_rows * a.heads * (head_dim + 2) * sizeof(float) : 0;
}

cudaError_t launch_packed_tc(const Launch& L, const PackedArgs& a, int head_dim, int n_sms, int splits, void* workspace) {
    return head_dim == 64 ? launch_tc<64>(L, a, n_sms, splits, workspace) : launch_tc<128>(L, a, n_sms, splits, workspace);
}

cudaError_t packed_tc_take_status(int* found) { return take_packed_status(found); }
