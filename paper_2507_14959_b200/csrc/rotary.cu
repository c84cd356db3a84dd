// Rotation of queries and keys by position, with or without a norm for each head in front of it (pm_rope, pm_qk_norm_rope).
//
//     u = x * gamma / sqrt(mean(x^2) + eps)   or   (x - mean) * gamma / sqrt(var + eps) + beta   or   x        (per head)
//     (a, b) -> (a cos t - b sin t, a sin t + b cos t)   for each pair (a, b) of u,  t = position * frequency of the pair
//
// Positions are whole numbers, so an angle is needed modulo one turn only: a frequency is held as the 64-bit fraction of a
// turn per position, and the wrapped 64-bit product with the position is the angle's fraction of a turn, to 2^-33 turns
// at any 32-bit position (a 32-bit product of position and frequency is off by 0.06 rad at position 10^6).  It is rounded to
// 32 bits, and the nearest quarter turn comes off before it becomes a float: at most an eighth of a turn is left, whose 24 bits are good
// to 2^-28 turns, or 2^-24 of what is left (of a whole turn they would be good to 2^-26, which is more than the rounding of a sine in 32 bits).
// Sine and cosine of the rest change places and signs with the quarter.
//
// Every element is read and written once.  A thread holds 16 elements of a head as 16-byte pieces (two of bf16, four of fp32) that lie
// side by side with the neighbouring threads', so that each load and store of a warp covers whole lines: with half layout the pairs of the
// rotated part, or a quarter or half of the rest; interleaved, a quarter or half of the head from its place on.  A warp takes a row: LP lanes
// a head, 32 / LP heads at once.  The lanes of the same place share the work on its eight angles and pass them on by shuffles; they
// are used for all heads of the row.
#include <math.h>

#include <algorithm>

#include "f32x2.cuh"
#include "tcgen05_ptx.cuh"

#define BUMP(L) do { if ((L).launches) ++*(L).launches; } while (0)

namespace {

constexpr int ROT_THREADS = 128;
constexpr int ROT_WARPS = ROT_THREADS / 32;
constexpr int ROT_RESIDENT = 4;                // CTAs of an SM
// Heads of a warp whose loads are issued together, ahead of the angles.  Twelve LayerNorm forms (fp32 from heads of 32 on, bf16 with heads wider than 64) keep 12 to 72
// bytes a thread in local memory for it: 0.4 % of the instructions of 50176 fp32 rows of 24 heads of 64 (110 us, 0.86 of the copy rate).
template <typename T, bool NORMS>
constexpr int ROT_BATCH = sizeof(T) == 4 ? 2 : NORMS ? 3 : 4;

struct RotArgs {
    const void *x[2];              // queries, keys (the rotation alone: one of them)
    void* y[2];
    long long x_stride[2], y_stride[2];      // elements between rows
    int heads[2];
    const float *gamma[2], *beta[2];
    int per_head;                  // gamma and beta of each head, else shared by all
    float eps, inv_dim;
    const int* positions;          // [rows, axes], or null: no rotation
    int rows, units, rot_units;    // units: 16-element pieces of a head; of the rotated part
    int steps;                     // warp iterations over the heads of a row
    int parts;                     // warps that share a row's iterations
    pm_rope_table table;
};

// A 16-byte piece as packed pairs, so that the arithmetic runs on two results per instruction (one at a time it takes twice the cycles of the
// floating-point unit).  Half layout: elements (0, 1), (2, 3) and so on.  Interleaved (IL): of every four elements (0, 2), then (1, 3), so that the two
// of a rotated pair stand at the same place of two packed ones.
template <typename T, bool IL> struct Piece;
template <bool IL> struct Piece<bf16, IL> {
    static constexpr int ELEMENTS = 8;
    uint4 r;
    __device__ __forceinline__ void load(const bf16* p) { r = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void unpack(uint64_t* v) const {              // a bf16 is the upper half of its 32-bit value
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const float a = __uint_as_float(w[k] << 16), b = __uint_as_float(w[k] & 0xFFFF0000u);
            const float c = __uint_as_float(w[k + 1] << 16), d = __uint_as_float(w[k + 1] & 0xFFFF0000u);
            v[k] = IL ? pk2(a, c) : pk2(a, b);
            v[k + 1] = IL ? pk2(b, d) : pk2(c, d);
        }
    }
    static __device__ __forceinline__ void store(bf16* p, const uint64_t* v) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            float a, b, c, d;
            upk2(v[k], a, b);
            upk2(v[k + 1], c, d);
            w[k] = IL ? pack_bf16(a, c) : pack_bf16(a, b);
            w[k + 1] = IL ? pack_bf16(b, d) : pack_bf16(c, d);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <bool IL> struct Piece<float, IL> {
    static constexpr int ELEMENTS = 4;
    float4 r;
    __device__ __forceinline__ void load(const float* p) { r = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void unpack(uint64_t* v) const {
        v[0] = IL ? pk2(r.x, r.z) : pk2(r.x, r.y);
        v[1] = IL ? pk2(r.y, r.w) : pk2(r.z, r.w);
    }
    static __device__ __forceinline__ void store(float* p, const uint64_t* v) {
        float a, b, c, d;
        upk2(v[0], a, b);
        upk2(v[1], c, d);
        *reinterpret_cast<float4*>(p) = IL ? make_float4(a, c, b, d) : make_float4(a, b, c, d);
    }
};
// the weights of a piece's N elements, packed alike
template <int N, bool IL>
__device__ __forceinline__ void load_weights(const float* p, uint64_t* v) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        Piece<float, IL> w;
        w.load(p + 4 * i);
        w.unpack(v + 2 * i);
    }
}
__device__ __forceinline__ float sum2(uint64_t x) {
    float a, b;
    upk2(x, a, b);
    return a + b;
}

enum { NORM_NONE = 0, NORM_RMS = 1, NORM_LAYER = 2 };

template <typename T, int NORM, int LP, bool IL>
__global__ void __launch_bounds__(ROT_THREADS, ROT_RESIDENT) rotate_kernel(const __grid_constant__ RotArgs a) {
    constexpr int HW = 32 / LP;                          // heads of a warp iteration
    constexpr int PPL = HW >= 8 ? 1 : 8 / HW;            // angles a lane works out
    constexpr int BATCH = ROT_BATCH<T, NORM != NORM_NONE>;
    constexpr int PE = Piece<T, IL>::ELEMENTS, PIECES = 16 / PE;
    const int lane = threadIdx.x & 31, u = lane % LP, slot = lane / LP;
    const bool used = u < a.units;
    const int dim = a.units * 16, rot = a.positions ? a.rot_units * 16 : 0;
    const int all = a.heads[0] + a.heads[1];
    const float amplitude = a.table.amplitude;
    // this thread's pieces: of the whole head, or with half layout of the rotated part or of the rest
    const bool split = !IL && rot > 0, front = u < a.rot_units;
    const int base = split && !front ? rot : 0, size = !split ? dim : front ? rot : dim - rot, place = split && !front ? u - a.rot_units : u;
    int at[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) at[k] = base + PE * place + k * (size / PIECES);
    // The thread's eight angles, c[x / 2] half x % 2.  Interleaved: of the pairs v[2 k], v[2 k + 1] in order.  Half layout: of v[0] to v[3], whose partners
    // are v[4] to v[7].  This lane works out PPL of them.
    bool turns[4];                                       // whether v[2 k], v[2 k + 1] are turned
#pragma unroll
    for (int k = 0; k < 4; ++k) turns[k] = used && base + PE * place + (4 * k / PE) * (size / PIECES) + 4 * k % PE < rot;
    unsigned long long step[PPL];
    int axis[PPL];
#pragma unroll
    for (int i = 0; i < PPL; ++i) {
        const int x = ((slot * PPL) & 7) + i, e = IL ? 2 * x : x;            // the pair's first element among the thread's sixteen
        const int element = base + PE * place + (e / PE) * (size / PIECES) + e % PE, pair = IL ? element / 2 : element;
        const bool turned = used && pair < rot / 2;
        step[i] = turned ? a.table.step[pair] : 0ull;
        axis[i] = a.table.axes == 2 && 4 * pair >= rot ? 1 : 0;
    }
    const long long tasks = (long long)a.rows * a.parts, stride = (long long)gridDim.x * ROT_WARPS;
    dep_release();
    dep_wait();
    for (long long task = (long long)blockIdx.x * ROT_WARPS + (threadIdx.x >> 5); task < tasks; task += stride) {
        const long long row = a.parts == 1 ? task : task / a.parts;
        const int part = a.parts == 1 ? 0 : (int)(task - row * a.parts);
        const int first = a.steps * part / a.parts, end = a.steps * (part + 1) / a.parts;
        const T* xr[2] = {(const T*)a.x[0] + row * a.x_stride[0], (const T*)a.x[1] + row * a.x_stride[1]};
        T* yr[2] = {(T*)a.y[0] + row * a.y_stride[0], (T*)a.y[1] + row * a.y_stride[1]};
        uint64_t c[4], s[4], ns[4];                      // cos, sin, -sin
        for (int it0 = first; it0 < end; it0 += BATCH) {
            Piece<T, IL> raw[BATCH][PIECES];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int head = (it0 + i) * HW + slot, w = head >= a.heads[0] ? 1 : 0, h = w ? head - a.heads[0] : head;
                const T* x = (w ? xr[1] : xr[0]) + h * dim;
#pragma unroll
                for (int k = 0; k < PIECES; ++k) {
                    raw[i][k] = Piece<T, IL>{};
                    if (used && head < all && it0 + i < end) raw[i][k].load(x + at[k]);
                }
            }
            if (it0 == first && rot > 0) {
                float mc[PPL], ms[PPL];
#pragma unroll
                for (int i = 0; i < PPL; ++i) {
                    const long long p = a.positions[row * a.table.axes + axis[i]];
                    const uint32_t turn = (uint32_t)(((unsigned long long)p * step[i] + 0x80000000ull) >> 32);     // of 2^32 to a turn
                    const uint32_t quarter = (turn + 0x20000000u) >> 30;
                    float sine, cosine;
                    sincospif((float)(int)(turn - (quarter << 30)) * 4.656612873077393e-10f, &sine, &cosine);     // 2^-31: in half turns
                    mc[i] = amplitude * (quarter & 1 ? sine : cosine);
                    ms[i] = amplitude * (quarter & 1 ? cosine : sine);
                    if ((quarter + 1) & 2) mc[i] = -mc[i];
                    if (quarter & 2) ms[i] = -ms[i];
                }
                float fc[8], fs[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int from = (i / PPL) * LP + u;
                    fc[i] = __shfl_sync(0xFFFFFFFFu, mc[i % PPL], from);
                    fs[i] = __shfl_sync(0xFFFFFFFFu, ms[i % PPL], from);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    c[k] = pk2(fc[2 * k], fc[2 * k + 1]);
                    s[k] = pk2(fs[2 * k], fs[2 * k + 1]);
                    ns[k] = s[k] ^ 0x8000000080000000ull;
                }
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (it0 + i >= end) break;
                const int head = (it0 + i) * HW + slot, w = head >= a.heads[0] ? 1 : 0, h = w ? head - a.heads[0] : head;
                const bool live = used && head < all;
                uint64_t v[8];
#pragma unroll
                for (int k = 0; k < PIECES; ++k) raw[i][k].unpack(v + k * PE / 2);
                if (NORM != NORM_NONE) {
                    uint64_t acc = 0ull;
                    if (NORM == NORM_LAYER) {
#pragma unroll
                        for (int k = 0; k < 8; k += 2) acc = add2(acc, add2(v[k], v[k + 1]));
                        float mean = sum2(acc);
#pragma unroll
                        for (int m = 1; m < LP; m <<= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, m);
                        mean = used ? -mean * a.inv_dim : 0.f;
                        const uint64_t m2 = pk2(mean, mean);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = add2(v[k], m2);
                        acc = 0ull;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) acc = fma2(v[k], v[k], acc);
                    float sum = sum2(acc);
#pragma unroll
                    for (int m = 1; m < LP; m <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, m);
                    const float inv = rsqrtf(fmaf(sum, a.inv_dim, a.eps));
                    if (live) {
                        const float* g = (w ? a.gamma[1] : a.gamma[0]) + (a.per_head ? h * dim : 0);
                        const uint64_t i2 = pk2(inv, inv);
                        uint64_t gw[8], bw[8] = {};
#pragma unroll
                        for (int k = 0; k < PIECES; ++k) load_weights<PE, IL>(g + at[k], gw + k * PE / 2);
                        if (NORM == NORM_LAYER) {
                            const float* b = w ? a.beta[1] : a.beta[0];
                            if (b) {
                                b += a.per_head ? h * dim : 0;
#pragma unroll
                                for (int k = 0; k < PIECES; ++k) load_weights<PE, IL>(b + at[k], bw + k * PE / 2);
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = NORM == NORM_LAYER ? fma2(v[k], mul2(gw[k], i2), bw[k]) : mul2(v[k], mul2(gw[k], i2));
                    }
                }
                auto turn = [](uint64_t& p, uint64_t& q, uint64_t c, uint64_t s, uint64_t ns) {
                    const uint64_t x = fma2(p, c, mul2(q, ns));
                    q = fma2(p, s, mul2(q, c));
                    p = x;
                };
                if (IL) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (turns[k]) turn(v[2 * k], v[2 * k + 1], c[k], s[k], ns[k]);
                } else if (turns[0]) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) turn(v[k], v[k + 4], c[k], s[k], ns[k]);
                }
                if (live) {
                    T* y = (w ? yr[1] : yr[0]) + h * dim;
#pragma unroll
                    for (int k = 0; k < PIECES; ++k) Piece<T, IL>::store(y + at[k], v + k * PE / 2);
                }
            }
        }
    }
}

template <typename T, int NORM, int LP>
cudaError_t rotate_launch(const Launch& L, RotArgs& a, int n_sms) {
    constexpr int HW = 32 / LP;
    a.steps = (a.heads[0] + a.heads[1] + HW - 1) / HW;
    // a row to a warp while that fills the GPU; fewer rows are cut along their heads
    const long long want = (long long)ROT_RESIDENT * ROT_WARPS * n_sms;
    a.parts = (int)std::min<long long>(a.steps, std::max<long long>(1, want / a.rows));
    const long long blocks = ((long long)a.rows * a.parts + ROT_WARPS - 1) / ROT_WARPS;
    const int grid = (int)std::min<long long>(blocks, (long long)ROT_RESIDENT * n_sms);
    ProfScope ps(L, KC_LAYERNORM);
    const cudaError_t e = a.table.interleaved && a.positions ? launch_overlapped(L, rotate_kernel<T, NORM, LP, true>, grid, ROT_THREADS, 0, 1, a)
                                                             : launch_overlapped(L, rotate_kernel<T, NORM, LP, false>, grid, ROT_THREADS, 0, 1, a);
    BUMP(L);
    return e;
}
template <typename T, int NORM>
cudaError_t rotate_lanes(const Launch& L, RotArgs& a, int n_sms) {
    if (a.units <= 1) return rotate_launch<T, NORM, 1>(L, a, n_sms);
    if (a.units <= 2) return rotate_launch<T, NORM, 2>(L, a, n_sms);
    if (a.units <= 4) return rotate_launch<T, NORM, 4>(L, a, n_sms);
    if (a.units <= 8) return rotate_launch<T, NORM, 8>(L, a, n_sms);
    return rotate_launch<T, NORM, 16>(L, a, n_sms);
}
template <typename T>
cudaError_t rotate_norm(const Launch& L, RotArgs& a, int norm, int n_sms) {
    switch (norm) {
        case NORM_RMS: return rotate_lanes<T, NORM_RMS>(L, a, n_sms);
        case NORM_LAYER: return rotate_lanes<T, NORM_LAYER>(L, a, n_sms);
        default: return rotate_lanes<T, NORM_NONE>(L, a, n_sms);
    }
}

bool table_ok(const pm_rope_table* t) {
    return t->head_dim > 0 && t->head_dim <= PM_ROPE_MAX_DIM && t->head_dim % 16 == 0 && t->rot_dim >= 0 && t->rot_dim % 16 == 0 &&
           t->rot_dim <= t->head_dim && (t->axes == 1 || t->axes == 2);
}
// rows of `heads` heads `stride` elements apart that a thread can take 16 bytes at a time
bool rows_ok(const void* p, long long stride, int heads, int dim, int dtype) {
    const int each = dtype == 0 ? 8 : 4;
    return p && ((uintptr_t)p & 15) == 0 && stride >= (long long)heads * dim && stride % each == 0;
}
int rotate(RotArgs& a, int norm, int dtype, void* cuda_stream) {
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int dev = 0, n_sms = 0;
    if (const int rc = stream_device(st, &dev); rc != PM_OK) return rc;
    if (consumed(cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return PM_ERR_CUDA;
    a.inv_dim = 1.f / (float)(a.units * 16);
    Launch L;
    L.st = st;
    const cudaError_t e = dtype == 0 ? rotate_norm<bf16>(L, a, norm, n_sms) : rotate_norm<float>(L, a, norm, n_sms);
    return e == cudaSuccess ? PM_OK : PM_ERR_CUDA;
}

}  // namespace

extern "C" {

int pm_rope_init(const pm_rope_config* cfg, pm_rope_table* out) {
    if (!cfg || !out) return PM_ERR_ARG;
    const int pairs = cfg->rot_dim / 2;
    if (cfg->head_dim <= 0 || cfg->head_dim % 16 || cfg->rot_dim <= 0 || cfg->rot_dim % 16 || cfg->rot_dim > cfg->head_dim ||
        (cfg->axes != 1 && cfg->axes != 2) || !(cfg->base > 0.0) || !isfinite(cfg->base) || !isfinite(cfg->amplitude))
        return PM_ERR_ARG;
    if (cfg->head_dim > PM_ROPE_MAX_DIM) return PM_ERR_CAPACITY;
    if (cfg->scaling < PM_ROPE_PLAIN || cfg->scaling > PM_ROPE_BANDS) return PM_ERR_ARG;
    if (cfg->scaling != PM_ROPE_PLAIN && (!(cfg->factor > 0.0) || !isfinite(cfg->factor))) return PM_ERR_ARG;
    if (cfg->scaling == PM_ROPE_BANDS && (!(cfg->original > 0.0) || !isfinite(cfg->original) || !(cfg->high_turns > cfg->low_turns) ||
                                          !isfinite(cfg->low_turns) || !isfinite(cfg->high_turns)))
        return PM_ERR_ARG;
    *out = pm_rope_table{};
    out->head_dim = cfg->head_dim; out->rot_dim = cfg->rot_dim;
    out->interleaved = cfg->interleaved != 0; out->axes = cfg->axes;
    out->amplitude = cfg->amplitude;
    const int each = pairs / cfg->axes;
    const long double two_pi = 6.283185307179586476925286766559L;
    long double base = cfg->base;
    if (cfg->scaling == PM_ROPE_NTK && each > 1) base *= powl((long double)cfg->factor, (long double)each / (each - 1));
    for (int i = 0; i < pairs; ++i) {
        long double f = powl(base, -(long double)(i % each) / each);
        if (cfg->scaling == PM_ROPE_LINEAR) f /= cfg->factor;
        if (cfg->scaling == PM_ROPE_BANDS) {
            const long double turns = (long double)cfg->original * f / two_pi;
            const long double keep = std::min(1.0L, std::max(0.0L, (turns - cfg->low_turns) / ((long double)cfg->high_turns - cfg->low_turns)));
            f *= keep + (1.0L - keep) / cfg->factor;
        }
        long double turn = f / two_pi;
        turn -= floorl(turn);                            // whole turns of a step do not matter: positions are whole numbers
        if (!(turn >= 0.0L && turn < 1.0L)) return PM_ERR_ARG;               // the frequencies overflowed
        // rounded half up; a fraction that rounds up to a whole turn is none
        const long double scaled = floorl(ldexpl(turn, 64) + 0.5L);
        out->step[i] = scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
    }
    return PM_OK;
}

int pm_rope(const void* x, long long x_stride, void* y, long long y_stride, const int32_t* positions, int rows, int heads,
            const pm_rope_table* table, int dtype, void* cuda_stream) {
    if (!table || !table_ok(table) || rows < 0 || heads <= 0 || (dtype != 0 && dtype != 1)) return PM_ERR_ARG;
    if (heads > PM_ROPE_MAX_HEADS) return PM_ERR_CAPACITY;
    if (rows == 0) return PM_OK;
    if (!positions || !rows_ok(x, x_stride, heads, table->head_dim, dtype) || !rows_ok(y, y_stride, heads, table->head_dim, dtype)) return PM_ERR_ARG;
    RotArgs a = {};
    a.x[0] = x; a.y[0] = y; a.x_stride[0] = x_stride; a.y_stride[0] = y_stride; a.heads[0] = heads;
    a.positions = positions; a.rows = rows;
    a.units = table->head_dim / 16; a.rot_units = table->rot_dim / 16;
    a.table = *table;
    return rotate(a, NORM_NONE, dtype, cuda_stream);
}

int pm_qk_norm_rope(const pm_qk_norm_rope_args* p, void* cuda_stream) {
    if (!p || p->rows < 0 || p->heads <= 0 || p->kv_heads < 0 || p->head_dim <= 0 || p->head_dim % 16 || (p->dtype != 0 && p->dtype != 1) ||
        (p->norm != PM_NORM_RMS && p->norm != PM_NORM_LAYER) || !(p->eps >= 0.f) || !isfinite(p->eps))
        return PM_ERR_ARG;
    if (p->head_dim > PM_ROPE_MAX_DIM || p->heads > PM_ROPE_MAX_HEADS || p->kv_heads > PM_ROPE_MAX_HEADS) return PM_ERR_CAPACITY;
    if (p->table && (!table_ok(p->table) || p->table->head_dim != p->head_dim || !p->positions)) return PM_ERR_ARG;
    if (p->norm == PM_NORM_RMS && (p->q_beta || p->k_beta)) return PM_ERR_ARG;
    if (p->rows == 0) return PM_OK;
    RotArgs a = {};
    const void* x[2] = {p->q, p->k};
    void* y[2] = {p->q_out, p->k_out};
    const long long xs[2] = {p->q_stride, p->k_stride}, ys[2] = {p->q_out_stride, p->k_out_stride};
    const int heads[2] = {p->heads, p->kv_heads};
    const float *gamma[2] = {p->q_gamma, p->k_gamma}, *beta[2] = {p->q_beta, p->k_beta};
    for (int w = 0; w < 2; ++w) {
        if (heads[w] == 0) continue;
        if (!rows_ok(x[w], xs[w], heads[w], p->head_dim, p->dtype) || !rows_ok(y[w], ys[w], heads[w], p->head_dim, p->dtype) || !gamma[w] ||
            ((uintptr_t)gamma[w] & 15) || ((uintptr_t)beta[w] & 15))
            return PM_ERR_ARG;
        a.x[w] = x[w]; a.y[w] = y[w]; a.x_stride[w] = xs[w]; a.y_stride[w] = ys[w]; a.heads[w] = heads[w];
        a.gamma[w] = gamma[w]; a.beta[w] = beta[w];
    }
    a.per_head = p->per_head != 0; a.eps = p->eps; a.rows = p->rows;
    a.units = p->head_dim / 16;
    if (p->table) {
        a.positions = p->positions;
        a.rot_units = p->table->rot_dim / 16;
        a.table = *p->table;
    } else {
        a.table.axes = 1;
    }
    return rotate(a, p->norm == PM_NORM_RMS ? NORM_RMS : NORM_LAYER, p->dtype, cuda_stream);
}

}  // extern "C"
