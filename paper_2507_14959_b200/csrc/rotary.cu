// Rotation of queries and keys by position, with or without a norm for each head in front of it (pm_rope, pm_qk_norm_rope).
//
//     u = x * gamma / sqrt(mean(x^2) + eps)   or   (x - mean) * gamma / sqrt(var + eps) + beta   or   x        (per head)
//     (a, b) -> (a cos t - b sin t, a sin t + b cos t)   for each pair (a, b) of u,  t = position * frequency of the pair
//
// Positions are whole numbers, so an angle is needed modulo one turn only: a frequency is held as the 64-bit fraction of a
// turn per position, and the wrapped 64-bit product with the position is the angle's fraction of a turn, exact to 2^-33 turns
// at any 32-bit position (a 32-bit product of position and frequency is off by 0.06 rad at position 10^6).  sincospi of that
// fraction needs no argument reduction.
//
// Bound by memory: every element is read and written once.  A thread holds 16 elements of a head -- the eight pairs
// whose angles they share -- as two 16-byte pieces (bf16): elements 8u.. and rot/2 + 8u.. (half layout) or 16u.. (interleaved,
// and what lies behind rot).  A warp takes a row: LP lanes a head, 32 / LP heads at once.  The lanes with the same u share
// the work on its eight angles and pass them on by shuffles; they are used for all heads of the row.
#include <math.h>

#include <algorithm>

#include "tcgen05_ptx.cuh"

#define BUMP(L) do { if ((L).launches) ++*(L).launches; } while (0)

namespace {

constexpr int ROT_THREADS = 128;
constexpr int ROT_WARPS = ROT_THREADS / 32;

struct RotArgs {
    const void *x[2];              // queries, keys (the rotation alone: one of them)
    void* y[2];
    long long x_stride[2], y_stride[2];      // elements between rows
    int heads[2];
    const float *gamma[2], *beta[2];
    int per_head;                  // gamma and beta of each head, else shared by all
    float eps;
    const int* positions;          // [rows, axes], or null: no rotation
    int rows, units, rot_units;    // units: 16-element pieces of a head; of the rotated part
    int steps;                     // warp iterations over the heads of a row
    int parts;                     // warps that share a row's iterations
    pm_rope_table table;
};

struct __align__(16) Bf16x8 { __nv_bfloat162 v[4]; };

__device__ __forceinline__ void load8(const bf16* p, float* v) {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {                       // a bf16 is the upper half of its 32-bit value
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float* v) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(bf16* p, const float* v) {
    Bf16x8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&o);
}
__device__ __forceinline__ void store8(float* p, const float* v) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

enum { NORM_NONE = 0, NORM_RMS = 1, NORM_LAYER = 2 };

template <typename T, int NORM, int LP>
__global__ void __launch_bounds__(ROT_THREADS) rotate_kernel(const __grid_constant__ RotArgs a) {
    constexpr int HW = 32 / LP;                          // heads of a warp iteration
    constexpr int PPL = HW >= 8 ? 1 : 8 / HW;            // angles a lane works out
    const int lane = threadIdx.x & 31, u = lane % LP, slot = lane / LP;
    const bool used = u < a.units, turns = u < a.rot_units && a.positions;
    const bool interleaved = a.table.interleaved != 0;
    // offsets of the two 8-element pieces in a head
    const int at0 = u >= a.rot_units || interleaved ? 16 * u : 8 * u;
    const int at1 = u >= a.rot_units || interleaved ? at0 + 8 : a.rot_units * 8 + 8 * u;
    const int dim = a.units * 16;
    const int all = a.heads[0] + a.heads[1];
    const float amplitude = a.table.amplitude;
    // this lane's angles: pair 8u + its own of the eight, on axis 0 or 1
    unsigned long long step[PPL];
    int axis[PPL];
    const int pairs = a.rot_units * 8, own = (slot * PPL) & 7;
#pragma unroll
    for (int i = 0; i < PPL; ++i) {
        const int p = 8 * u + own + i;
        step[i] = turns ? a.table.step[p] : 0ull;
        axis[i] = a.table.axes == 2 && 2 * p >= pairs ? 1 : 0;
    }
    const long long tasks = (long long)a.rows * a.parts, stride = (long long)gridDim.x * ROT_WARPS;
    dep_release();
    dep_wait();
    for (long long task = (long long)blockIdx.x * ROT_WARPS + (threadIdx.x >> 5); task < tasks; task += stride) {
        const long long row = a.parts == 1 ? task : task / a.parts;
        const int part = a.parts == 1 ? 0 : (int)(task - row * a.parts);
        float c[8], s[8];
        if (a.positions) {
            float mc[PPL], ms[PPL];
#pragma unroll
            for (int i = 0; i < PPL; ++i) {
                const long long p = a.positions[row * a.table.axes + axis[i]];
                const int turn = (int)(((unsigned long long)p * step[i]) >> 32);         // of 2^32 to a turn, signed
                sincospif((float)turn * 4.656612873077393e-10f, &ms[i], &mc[i]);         // 2^-31: in half turns
                mc[i] *= amplitude;
                ms[i] *= amplitude;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int from = (i / PPL) * LP + u;
                c[i] = __shfl_sync(0xFFFFFFFFu, mc[i % PPL], from);
                s[i] = __shfl_sync(0xFFFFFFFFu, ms[i % PPL], from);
            }
        }
        const int first = a.steps * part / a.parts, end = a.steps * (part + 1) / a.parts;
#pragma unroll 2
        for (int it = first; it < end; ++it) {
            const int head = it * HW + slot;
            const int w = head >= a.heads[0] ? 1 : 0, h = w ? head - a.heads[0] : head;
            const bool live = used && head < all;
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.f;
            if (live) {
                const T* x = (const T*)a.x[w] + row * a.x_stride[w] + (long long)h * dim;
                load8(x + at0, v);
                load8(x + at1, v + 8);
            }
            if (NORM != NORM_NONE) {
                float mean = 0.f, sum = 0.f;
                if (NORM == NORM_LAYER) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) mean += v[i];
#pragma unroll
                    for (int m = 1; m < LP; m <<= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, m);
                    mean /= (float)dim;
                    if (used)
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] -= mean;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = fmaf(v[i], v[i], sum);
#pragma unroll
                for (int m = 1; m < LP; m <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, m);
                const float inv = 1.f / sqrtf(sum / (float)dim + a.eps);
                if (live) {
                    const float* g = a.gamma[w] + (a.per_head ? h * dim : 0);
                    float t[8];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        load8(g + (k ? at1 : at0), t);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[8 * k + i] *= inv * t[i];
                    }
                    if (NORM == NORM_LAYER && a.beta[w]) {
                        const float* b = a.beta[w] + (a.per_head ? h * dim : 0);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            load8(b + (k ? at1 : at0), t);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[8 * k + i] += t[i];
                        }
                    }
                }
            }
            if (turns) {
                if (interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = v[2 * i], q = v[2 * i + 1];
                        v[2 * i] = p * c[i] - q * s[i];
                        v[2 * i + 1] = p * s[i] + q * c[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = v[i], q = v[8 + i];
                        v[i] = p * c[i] - q * s[i];
                        v[8 + i] = p * s[i] + q * c[i];
                    }
                }
            }
            if (live) {
                T* y = (T*)a.y[w] + row * a.y_stride[w] + (long long)h * dim;
                store8(y + at0, v);
                store8(y + at1, v + 8);
            }
        }
    }
}

template <typename T, int NORM, int LP>
cudaError_t rotate_launch(const Launch& L, RotArgs& a, int n_sms) {
    constexpr int HW = 32 / LP;
    a.steps = (a.heads[0] + a.heads[1] + HW - 1) / HW;
    // a row to a warp while that fills the GPU (sixteen warps a multiprocessor); fewer rows are cut along their heads
    const long long want = 16ll * n_sms;
    a.parts = (int)std::min<long long>(a.steps, std::max<long long>(1, want / a.rows));
    const long long blocks = ((long long)a.rows * a.parts + ROT_WARPS - 1) / ROT_WARPS;
    const int grid = (int)std::min<long long>(blocks, 16ll * n_sms);
    ProfScope ps(L, KC_LAYERNORM);
    const cudaError_t e = launch_overlapped(L, rotate_kernel<T, NORM, LP>, grid, ROT_THREADS, 0, 1, a);
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
    if (cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return PM_ERR_CUDA; }
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
