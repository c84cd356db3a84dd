// Attention over packed sequences on the tcgen05 tensor cores (bf16; the operator is described in attention_packed.cu).
//
// One persistent CTA per SM walks units: two tiles of 128 rows of a (sequence, K/V head) pair -- a row is a (query, head of the group) pair,
// so a tile holds TT = 128 / group queries of all the heads that share K and V, and the keys and values of a block serve 256 rows.  Key
// blocks of 128 pass through a ring in shared memory.  Per tile and block
//     S = Q K^T             UMMA 128 x 128 x 16 steps, fp32 scores in tensor memory
//     P = 2^(c S - c m)     one row per thread: the row's scores in registers, written back as packed bf16
//     O += P V              UMMA 128 x D x 16 steps, P read from tensor memory, V as an MN-major operand
// m is the row's running maximum, but it only moves when it has grown by more than 2^8 in the exponential's scale: then the thread
// takes its row of O and of the sum down to the new one (no overflow can come of the lag: terms stay below 2^8, sums below 2^8 n).
//     warps 0..3, 4..7    softmax of the two tiles
//     warps 8..11         output of both: O / sum to global memory, while the softmax is at the next unit
//     warp 12             MMA issue: the scores of step g + 1 before or right after the products of step g
//     warp 13             units, TMA loads
//     warp 14             the rows of a value block that lie behind the sequence's last key are set to zero (at most 15 of them
//                         take part in a product, with weight zero; what lies there may be NaN)
// Scores of head dim 64 have tensor memory of their own beside P, so the next block's are formed while this one's
// exponentials run; with 128 P lies over S and the two tiles take turns.
// Units are visited from the last rows of the sequences to the first, so in causal order the long ones come first.
#include <algorithm>

#include "f32x2.cuh"
#include "packed.cuh"

#define BUMP(L) do { if ((L).launches) ++*(L).launches; } while (0)

namespace {

constexpr int PT_THREADS = 512;
constexpr int PT_ROWS = 128;                                  // rows of a tile
constexpr int PT_KEYS = 128;                                  // keys of a block
constexpr int PT_UNITS = 4;                                   // units announced ahead
constexpr int PT_TAILS = 2 * PT_UNITS;                        // barriers of value blocks to be cleared; the loads are at most PT_UNITS units ahead of warp 14
constexpr float PT_LAG = 8.f;                                 // log2 of how far a row's terms may exceed 1
// registers per thread of the warpgroups; their sum is what the launch brings (512 threads x 128)
constexpr int PT_REGS_SOFTMAX = 200, PT_REGS_OUT = 64, PT_REGS_ISSUE = 48;
static_assert(2 * PT_REGS_SOFTMAX + PT_REGS_OUT + PT_REGS_ISSUE <= 4 * 128, "register shares");

template <int D>
struct PtLayout {
    static constexpr bool OWN_P = D == 64;                    // P beside S: the next scores need not wait for the product
    static constexpr int SLOT = 128 * D * 2;                  // bytes of a Q tile, a K block, a V block
    static constexpr int Q_SLOTS = 3, KV_SLOTS = D == 64 ? 8 : 4;
    static constexpr int SUMS = OWN_P ? 4 : 2;                // buffers of row sums (see the softmax warps)
    static __host__ __device__ constexpr uint32_t s_col(int i) { return OWN_P ? i * 256 : i * 128; }
    static __host__ __device__ constexpr uint32_t p_col(int i) { return OWN_P ? i * 256 + 128 : i * 128; }
    static __host__ __device__ constexpr uint32_t o_col(int i) { return OWN_P ? i * 256 + 192 : 256 + i * 128; }
};

struct PtUnit {                                               // 32 bytes
    int q0, nq, k0, nk;                                       // the sequence
    int tok0, kv_head, blocks0, blocks1;                      // first query; key blocks of the two tiles; blocks0 < 0: no more units
};

template <int D>
struct PtControl {
    float sums[PtLayout<D>::SUMS][2][PT_ROWS];
    PtUnit units[PT_UNITS];
    unsigned long long q_full[PtLayout<D>::Q_SLOTS], q_empty[PtLayout<D>::Q_SLOTS];
    unsigned long long kv_full[PtLayout<D>::KV_SLOTS], kv_empty[PtLayout<D>::KV_SLOTS];
    unsigned long long s_ready[2], s_read[2], p_ready[2], pv_done[2], o_ready[2], o_read[2], l_ready[2];
    unsigned long long tail[PT_TAILS], unit_full[PT_UNITS], unit_empty[PT_UNITS];
    uint32_t tmem;
    int abort;
};
template <int D>
__host__ __device__ constexpr size_t pt_smem() {
    return (size_t)(PtLayout<D>::Q_SLOTS + PtLayout<D>::KV_SLOTS) * PtLayout<D>::SLOT + sizeof(PtControl<D>);
}
static_assert(pt_smem<64>() <= 227 * 1024 && pt_smem<128>() <= 227 * 1024, "shared memory");

struct PtArgs {
    PackedArgs a;
    int tile_tokens;                                          // TT
};

template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// V block as the MN-major B operand of O += P V: 64-wide pieces of the head dim lie 16 KB apart
template <int D>
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr) {
    return D == 64 ? smem_desc(saddr, 128)
                   : ((uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(16384 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61));
}
__device__ __forceinline__ int round16(int n) { return (n + 15) & ~15; }
// Whether the unit's last value block holds rows behind the sequence's last key that a product reads (it takes keys by 16).  That block
// lands on a barrier of its own, where warp 14 awaits it, and warp 14 passes it on to those who await the ring.
__device__ __forceinline__ bool has_tail(const PtUnit& u) {
    const int blocks = max(u.blocks0, u.blocks1);
    return blocks * PT_KEYS > u.nk && (u.nk & 15) != 0;
}

// Key blocks of a tile whose first query is `tok` (0: no queries, or none of them sees a key).
__device__ __forceinline__ int tile_blocks(const Segment& g, int tok, int tile_tokens, int causal) {
    if (tok >= g.nq) return 0;
    return (packed_visible(g, min(tok + tile_tokens, g.nq) - 1, causal) + PT_KEYS - 1) / PT_KEYS;
}
// Keys of block j that the tile's last query sees, at most a block.
__device__ __forceinline__ int block_keys(const PtUnit& u, int tile, int j, int tile_tokens, int causal) {
    const Segment g{u.q0, u.nq, u.k0, u.nk};
    return min(PT_KEYS, packed_visible(g, min(u.tok0 + (tile + 1) * tile_tokens, u.nq) - 1, causal) - j * PT_KEYS);
}

template <int D>
__global__ void __launch_bounds__(PT_THREADS, 1)
attention_packed_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                           const __grid_constant__ PtArgs args) {
    using Lay = PtLayout<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t base = smem_u32(smem_raw);
    const PackedArgs& a = args.a;
    if (base & 1023u) {                       // swizzled operands need a 1024-byte aligned window
        if (threadIdx.x == 0) atomicCAS(a.status, 0, (int)PM_ERR_CUDA);
        return;
    }
    PtControl<D>& ctl = *reinterpret_cast<PtControl<D>*>(smem_raw + (Lay::Q_SLOTS + Lay::KV_SLOTS) * Lay::SLOT);
    auto q_s = [&](int slot) { return base + (uint32_t)(slot * Lay::SLOT); };
    auto kv_s = [&](int slot) { return base + (uint32_t)((Lay::Q_SLOTS + slot) * Lay::SLOT); };
    auto bar = [&](const unsigned long long& b) { return smem_u32(&b); };
    volatile int* abort_flag = &ctl.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int TT = args.tile_tokens;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Lay::Q_SLOTS; ++i) { mbar_init(bar(ctl.q_full[i]), 1); mbar_init(bar(ctl.q_empty[i]), 1); }
        for (int i = 0; i < Lay::KV_SLOTS; ++i) { mbar_init(bar(ctl.kv_full[i]), 1); mbar_init(bar(ctl.kv_empty[i]), 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(ctl.s_ready[i]), 1); mbar_init(bar(ctl.s_read[i]), 4); mbar_init(bar(ctl.p_ready[i]), 4); mbar_init(bar(ctl.pv_done[i]), 1);
            mbar_init(bar(ctl.o_ready[i]), 1); mbar_init(bar(ctl.o_read[i]), 4); mbar_init(bar(ctl.l_ready[i]), 4);
        }
        for (int i = 0; i < PT_TAILS; ++i) mbar_init(bar(ctl.tail[i]), 1);
        // consumers of a unit: twelve softmax and output warps, the issuing thread, warp 14
        for (int i = 0; i < PT_UNITS; ++i) { mbar_init(bar(ctl.unit_full[i]), 1); mbar_init(bar(ctl.unit_empty[i]), 14); }
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    if (warp == 12) {
        tmem_alloc(smem_u32(&ctl.tmem), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    dep_release();

    // unit number n of this CTA; false once the CTA is aborting
    auto take_unit = [&](uint32_t n, PtUnit& u) {
        if (!mbar_wait(bar(ctl.unit_full[n % PT_UNITS]), (n / PT_UNITS) & 1u, abort_flag, a.status)) return false;
        const int4* p = reinterpret_cast<const int4*>(&ctl.units[n % PT_UNITS]);
        const int4 x = p[0], y = p[1];
        u = PtUnit{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        return true;
    };

    if (warp < 8) {
        // ------------------------------------------------------------------ softmax
        regs_up<PT_REGS_SOFTMAX>();
        const int tile = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + Lay::s_col(tile), t_p = tmem + lanes + Lay::p_col(tile), t_o = tmem + lanes + Lay::o_col(tile);
        const int row_tok = row / a.group;
        const float c = a.c, lag = PT_LAG / a.c;
        const uint64_t c2 = pk2(c, c);
        uint32_t steps = 0, sums = 0;                         // blocks, tiles so far
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            PtUnit u;
            ok = take_unit(n, u);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            if (lane == 0) mbar_arrive(bar(ctl.unit_empty[n % PT_UNITS]));
            if (u.blocks0 < 0) break;
            const int blocks = tile ? u.blocks1 : u.blocks0;
            if (blocks == 0) continue;
            const Segment seg{u.q0, u.nq, u.k0, u.nk};
            const int tok0 = u.tok0 + tile * TT;
            const int vis = packed_visible(seg, min(tok0 + row_tok, u.nq - 1), a.causal);
            const int vis_all = packed_visible(seg, tok0, a.causal);         // keys that every row sees
            const int vis_end = packed_visible(seg, min(tok0 + TT, u.nq) - 1, a.causal);
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < blocks; ++j, ++steps) {
                const int ncols = round16(min(PT_KEYS, vis_end - j * PT_KEYS));
                ok = mbar_wait(bar(ctl.s_ready[tile]), steps & 1u, abort_flag, a.status);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after();
                uint32_t v[128];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k * 32 < ncols) tmem_ld32(t_s + k * 32, v + k * 32);
                tmem_ld_wait();
                if (Lay::OWN_P) {                             // the scores are in registers: the next ones may take their place
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(ctl.s_read[tile]));
                }
                const int lim = vis - j * PT_KEYS;
                if (vis_all < (j + 1) * PT_KEYS) {            // hidden keys, and columns that were not formed
#pragma unroll
                    for (int e = 0; e < 128; ++e) v[e] = e < lim ? v[e] : 0xFF800000u;
                }
                float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k * 32 < ncols)
#pragma unroll
                        for (int e = 0; e < 32; ++e) t[e & 3] = fmaxf(t[e & 3], __uint_as_float(v[k * 32 + e]));
                const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
                if (j == 0) {
                    m = top;
                } else if (__any_sync(0xFFFFFFFFu, top > m + lag)) {
                    // what is there comes down to the new maximum, once the product before has been added
                    const float up = fmaxf(m, top), f = up == m ? 1.f : ex2f((m - up) * c);
                    m = up;
                    l *= f;
                    ok = mbar_wait(bar(ctl.pv_done[tile]), (steps - 1) & 1u, abort_flag, a.status);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        uint32_t o[16];
                        tmem_ld16(t_o + k * 16, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st16(t_o + k * 16, o);
                    }
                }
                if (Lay::OWN_P && steps > 0) {                // the product before has read its probabilities
                    ok = mbar_wait(bar(ctl.pv_done[tile]), (steps - 1) & 1u, abort_flag, a.status);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
                }
                const float mc = m == -INFINITY ? 0.f : -m * c;              // a row that sees nothing: all terms 0
                const uint64_t mc2 = pk2(mc, mc);
                uint64_t sum0 = pk2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k * 32 < ncols) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float x, y;
                            upk2(fma2(pk2(__uint_as_float(v[k * 32 + e]), __uint_as_float(v[k * 32 + e + 1])), c2, mc2), x, y);
                            x = ex2f(x);
                            y = ex2f(y);
                            if (e & 2) sum1 = add2(sum1, pk2(x, y));
                            else sum0 = add2(sum0, pk2(x, y));
                            pk[e >> 1] = pack_bf16(x, y);
                        }
                        tmem_st16(t_p + k * 16, pk);
                    }
                float s0, s1;
                upk2(add2(sum0, sum1), s0, s1);
                l += s0 + s1;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ctl.p_ready[tile]));
            }
            if (!ok) break;
            // Read by the output warps before o_read is signalled.  A buffer comes up again SUMS tiles later: scores of a tile are formed after
            // the product of the tile before it (own P: of the one before that) was issued, which waited for o_read of the tile before that.
            ctl.sums[sums % Lay::SUMS][tile][row] = l;
            ++sums;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(ctl.l_ready[tile]));
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------------ output
        regs_down<PT_REGS_OUT>();
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int row_tok = row / a.group, head = row % a.group;
        uint32_t done[2] = {0, 0};
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            PtUnit u;
            ok = take_unit(n, u);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            if (lane == 0) mbar_arrive(bar(ctl.unit_empty[n % PT_UNITS]));
            if (u.blocks0 < 0) break;
#pragma unroll
            for (int tile = 0; tile < 2; ++tile) {
                const int blocks = tile ? u.blocks1 : u.blocks0, tok = u.tok0 + tile * TT + row_tok;
                const bool real = row_tok < TT && tok < u.nq;
                bf16* to = (bf16*)a.out + (long long)(u.q0 + tok) * a.out_stride + (u.kv_head * a.group + head) * D;
                float inv = 0.f;
                if (blocks > 0) {
                    ok = mbar_wait(bar(ctl.l_ready[tile]), done[tile] & 1u, abort_flag, a.status);
                    ok = ok && mbar_wait(bar(ctl.o_ready[tile]), done[tile] & 1u, abort_flag, a.status);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    const float l = ctl.sums[done[tile] % Lay::SUMS][tile][row];
                    inv = l == 0.f ? 0.f : 1.f / l;
                    ++done[tile];
                }
                const uint32_t t_o = tmem + lanes + Lay::o_col(tile);
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    uint32_t o[32];
                    if (blocks > 0) {
                        tmem_ld32(t_o + k * 32, o);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0u;
                    }
                    if (real)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint32_t w[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                w[e] = pack_bf16(__uint_as_float(o[q * 16 + 2 * e]) * inv, __uint_as_float(o[q * 16 + 2 * e + 1]) * inv);
                            *reinterpret_cast<uint4*>(to + k * 32 + q * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                            *reinterpret_cast<uint4*>(to + k * 32 + q * 16 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                }
                if (blocks > 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(ctl.o_read[tile]));
                }
            }
        }
    } else {
        regs_down<PT_REGS_ISSUE>();
        if (warp == 12) {
            if (elect_one()) {
                // -------------------------------------------------------------- MMA issue
                // Steps: key block j of a unit, for the tiles that have it.  kv: ring position of the step's K block (V follows it).
                struct Step { PtUnit u; int j, blocks; uint32_t kv, q[2]; };
                const uint32_t idesc_pv = instr_desc_b_mn(D);
                uint32_t units = 0, kv_next = 0, q_next = 0;
                uint32_t s_count[2] = {0, 0}, p_count[2] = {0, 0}, o_count[2] = {0, 0};
                bool ok = true, more = true;
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
                    s.q[0] = s.q[1] = 0;
                    if (s.u.blocks0 > 0) s.q[0] = q_next++;
                    if (s.u.blocks1 > 0) s.q[1] = q_next++;
                    return true;
                };
                auto has = [&](const Step& s, int i) { return s.j < (i ? s.u.blocks1 : s.u.blocks0); };
                // the last of a step's tiles to use its K and V blocks
                auto last_tile = [&](const Step& s) { return has(s, 1) ? 1 : 0; };
                auto issue_s = [&](const Step& s, int i) {
                    if (Lay::OWN_P) {                         // the tile's scores before must have been read
                        ok = mbar_wait(bar(ctl.s_read[i]), (s_count[i] & 1u) ^ 1u, abort_flag, a.status);
                        if (!ok) return;
                    }
                    ++s_count[i];
                    const int q_slot = (int)(s.q[i] % Lay::Q_SLOTS), k_slot = (int)(s.kv % Lay::KV_SLOTS);
                    if (s.j == 0) ok = mbar_wait(bar(ctl.q_full[q_slot]), (s.q[i] / Lay::Q_SLOTS) & 1u, abort_flag, a.status);
                    ok = ok && mbar_wait(bar(ctl.kv_full[k_slot]), (s.kv / Lay::KV_SLOTS) & 1u, abort_flag, a.status);
                    if (!ok) return;
                    tc_fence_after();
                    const uint32_t idesc = instr_desc(round16(block_keys(s.u, i, s.j, TT, a.causal)));
                    const uint64_t dq = smem_desc(q_s(q_slot), 128), dk = smem_desc(kv_s(k_slot), 128);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t at = (uint64_t)((k / 4) * (16384 >> 4) + 2 * (k % 4));
                        umma_bf16(tmem + Lay::s_col(i), dq + at, dk + at, idesc, k > 0);
                    }
                    umma_commit(bar(ctl.s_ready[i]));
                    if (i == last_tile(s)) umma_commit(bar(ctl.kv_empty[k_slot]));
                    if (s.j + 1 == (i ? s.u.blocks1 : s.u.blocks0)) umma_commit(bar(ctl.q_empty[q_slot]));
                };
                auto issue_pv = [&](const Step& s, int i) {
                    const int blocks = i ? s.u.blocks1 : s.u.blocks0;
                    const uint32_t at = s.kv + 1;
                    const int v_slot = (int)(at % Lay::KV_SLOTS);
                    ok = mbar_wait(bar(ctl.p_ready[i]), p_count[i] & 1u, abort_flag, a.status);
                    ++p_count[i];
                    ok = ok && mbar_wait(bar(ctl.kv_full[v_slot]), (at / Lay::KV_SLOTS) & 1u, abort_flag, a.status);
                    // the tile's output before has been read
                    if (ok && s.j == 0) {
                        ok = mbar_wait(bar(ctl.o_read[i]), (o_count[i] & 1u) ^ 1u, abort_flag, a.status);
                        ++o_count[i];
                    }
                    if (!ok) return;
                    tc_fence_after();
                    const int pieces = round16(block_keys(s.u, i, s.j, TT, a.causal)) / 16;
                    const uint64_t dv = v_desc<D>(kv_s(v_slot));
                    for (int k = 0; k < pieces; ++k)
                        umma_bf16_ts(tmem + Lay::o_col(i), tmem + Lay::p_col(i) + 8 * k, dv + 128 * k, idesc_pv, (s.j > 0 || k > 0) ? 1u : 0u);
                    umma_commit(bar(ctl.pv_done[i]));
                    if (i == last_tile(s)) umma_commit(bar(ctl.kv_empty[v_slot]));
                    if (s.j + 1 == blocks) umma_commit(bar(ctl.o_ready[i]));
                };
                Step cur, next;
                more = advance(cur, true);
                if (more) {
                    for (int i = 0; i < 2 && ok; ++i)
                        if (has(cur, i)) issue_s(cur, i);
                }
                while (more && ok) {
                    next = cur;
                    more = advance(next, false);
                    if (!ok) break;
                    if (Lay::OWN_P) {
                        for (int i = 0; i < 2 && ok; ++i)
                            if (more && has(next, i)) issue_s(next, i);
                    }
                    for (int i = 0; i < 2 && ok; ++i) {
                        if (has(cur, i)) issue_pv(cur, i);
                        if (!Lay::OWN_P && ok && more && has(next, i)) issue_s(next, i);
                    }
                    cur = next;
                }
            }
        } else if (warp == 13) {
            // ------------------------------------------------------------------ units and loads
            dep_wait();                                       // everything else follows from what is read here
            const int n_seqs = a.n_seqs, per_unit = 2 * TT;
            auto units_of = [&](int s) {
                if (s >= n_seqs) return 0;
                return (packed_segment(a, s).nq + per_unit - 1) / per_unit;
            };
            int most = 0;
            for (int s = lane; s < n_seqs; s += 32) most = max(most, units_of(s));
            most = __reduce_max_sync(0xFFFFFFFFu, most);
            // Walk: level by level from `most` - 1 down, in a level the sequences that reach it, in a sequence the K/V heads.  `left` counts from
            // the start of the current 32 sequences at the current level.
            int level = most - 1, block = 0, mine = units_of(lane);
            long long left = blockIdx.x;
            uint32_t units = 0, kv = 0, q = 0, tails = 0;
            bool ok = true;
            while (ok) {
                uint32_t set = 0;
                while (level >= 0) {
                    set = __ballot_sync(0xFFFFFFFFu, mine > level);
                    const long long here = (long long)__popc(set) * a.kv_heads;
                    if (left < here) break;
                    left -= here;
                    block += 32;
                    if (block >= n_seqs) { block = 0; --level; }
                    if (n_seqs > 32) mine = units_of(block + lane);
                }
                PtUnit u = {0, 0, 0, 0, 0, 0, -1, -1};
                if (level >= 0) {
                    int nth = (int)(left / a.kv_heads);
                    for (; nth > 0; --nth) set &= set - 1;
                    const Segment g = packed_segment(a, block + __ffs((int)set) - 1);
                    u.q0 = g.q0; u.nq = g.nq; u.k0 = g.k0; u.nk = g.nk;
                    u.tok0 = level * per_unit;
                    u.kv_head = (int)(left % a.kv_heads);
                    u.blocks0 = tile_blocks(g, u.tok0, TT, a.causal);
                    u.blocks1 = tile_blocks(g, u.tok0 + TT, TT, a.causal);
                    left += gridDim.x;
                }
                const int at = (int)(units % PT_UNITS);
                ok = mbar_wait(bar(ctl.unit_empty[at]), ((units / PT_UNITS) & 1u) ^ 1u, abort_flag, a.status);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                if (lane == 0) {
                    int4* p = reinterpret_cast<int4*>(&ctl.units[at]);
                    p[0] = make_int4(u.q0, u.nq, u.k0, u.nk);
                    p[1] = make_int4(u.tok0, u.kv_head, u.blocks0, u.blocks1);
                    mbar_arrive(bar(ctl.unit_full[at]));
                }
                __syncwarp();
                ++units;
                if (u.blocks0 < 0) break;
                const int blocks = max(u.blocks0, u.blocks1);
                const bool tail = has_tail(u);
                if (elect_one()) {
                    auto load_q = [&](int i) {
                        const int slot = (int)(q % Lay::Q_SLOTS);
                        ok = ok && mbar_wait(bar(ctl.q_empty[slot]), ((q / Lay::Q_SLOTS) & 1u) ^ 1u, abort_flag, a.status);
                        if (!ok) return;
                        mbar_expect_tx(bar(ctl.q_full[slot]), (uint32_t)(TT * a.group * D * 2));
                        for (int x = 0; x < D / 64; ++x)
                            tma_load_3d(q_s(slot) + x * 16384, &tm_q, x * 64, u.kv_head * a.group, u.q0 + u.tok0 + i * TT, bar(ctl.q_full[slot]));
                        ++q;
                    };
                    auto load_kv = [&](const CUtensorMap* tm, int j, unsigned long long* full) {
                        const int slot = (int)(kv % Lay::KV_SLOTS);
                        ok = ok && mbar_wait(bar(ctl.kv_empty[slot]), ((kv / Lay::KV_SLOTS) & 1u) ^ 1u, abort_flag, a.status);
                        if (!ok) return;
                        const uint32_t on = full ? bar(*full) : bar(ctl.kv_full[slot]);
                        mbar_expect_tx(on, (uint32_t)Lay::SLOT);
                        for (int x = 0; x < D / 64; ++x) tma_load_3d(kv_s(slot) + x * 16384, tm, x * 64, u.kv_head, u.k0 + j * PT_KEYS, on);
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
                q = __reduce_max_sync(0xFFFFFFFFu, q);
            }
        } else if (warp == 14) {
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
                ok = mbar_wait(bar(ctl.tail[tails % PT_TAILS]), (tails / PT_TAILS) & 1u, abort_flag, a.status);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                ++tails;
                const int first = u.nk - (blocks - 1) * PT_KEYS, rows = round16(first) - first;
                for (int i = lane; i < rows * D / 8; i += 32) {              // whole rows, so their swizzle does not matter
                    const int r = first + i / (D / 8), c = i % (D / 8);
                    st_shared_v4(kv_s(slot) + (uint32_t)((c / 8) * 16384 + r * 128 + (c % 8) * 16), make_uint4(0, 0, 0, 0));
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
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int D>
cudaError_t launch_tc(const Launch& L, const PackedArgs& a, int n_sms) {
    PtArgs args;
    args.a = a;
    args.tile_tokens = PT_ROWS / a.group;
    CUtensorMap tm_q, tm_k, tm_v;
    if (!tm_encode_3d(&tm_q, a.q, D, a.heads, a.q_rows, D * 2, (uint64_t)a.q_stride * 2, 64, a.group, args.tile_tokens, 128) ||
        !tm_encode_3d(&tm_k, a.k, D, a.kv_heads, a.kv_rows, D * 2, (uint64_t)a.k_stride * 2, 64, 1, PT_KEYS, 128) ||
        !tm_encode_3d(&tm_v, a.v, D, a.kv_heads, a.kv_rows, D * 2, (uint64_t)a.v_stride * 2, 64, 1, PT_KEYS, 128))
        return cudaErrorInvalidValue;
    static SmemGrant grant;
    if (cudaError_t e = grant.ensure(attention_packed_tc_kernel<D>, (int)pt_smem<D>()); e != cudaSuccess) return e;
    const long long units = (a.q_rows / (2 * args.tile_tokens) + (long long)a.n_seqs) * a.kv_heads;      // at most
    ProfScope ps(L, KC_ATTENTION);
    cudaError_t e = launch_overlapped(L, attention_packed_tc_kernel<D>, dim3((unsigned)std::min<long long>(units, n_sms)), PT_THREADS, pt_smem<D>(), 1, tm_q, tm_k,
                                      tm_v, args);
    BUMP(L);
    return e;
}

}  // namespace

cudaError_t launch_packed_tc(const Launch& L, const PackedArgs& a, int head_dim, int n_sms) {
    return head_dim == 64 ? launch_tc<64>(L, a, n_sms) : launch_tc<128>(L, a, n_sms);
}
