// Row layers: residual sum with dropout and root-mean-square norm (forward, backward, output in 8 bits), dropout.
//
// All of them read and write each element once and are bound by memory: 8,192 rows of 4,096 units, bf16, dropout, sum and norm 52 us (268 MB, 5.2 TB/s,
// as a copy of that size), its gradients 76 us (336 MB, 4.4 TB/s; 5 us of it the sum over the rows for the gain); output in e4m3
// (16,384 rows) 107 us (472 MB, 4.4 TB/s); dropout of 4,099 rows of 16,381 units, bf16, 58 us (4.6 TB/s).  A row is held in registers between its loads and
// its stores by 64, 256 or 1,024 threads, eight neighbouring units to a thread and vector (16 bytes of a 16-bit type; the
// group that shares a counter of the dropout generator); the sum of squares goes over the lanes of a wavefront and, for more
// than 64 threads, through LDS.
#include "layers.h"

#include <algorithm>

namespace rnng {
namespace {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
template <class T> struct Vec8 { typedef T type __attribute__((ext_vector_type(8))); };
typedef float f32x8 __attribute__((ext_vector_type(8)));

// n of eight elements (all, if n >= 8) in fp32, zeros behind them.  Rows may start at any element: the load is one of 16 or 32
// bytes at whatever alignment (global memory takes unaligned vectors).
// WHOLE: n >= 8 or n <= 0 (rows of a multiple of eight units).
template <bool WHOLE, class T>
__device__ __forceinline__ f32x8 load8(const T* p, int n) {
    f32x8 r = 0.0f;
    if (n >= 8) {
        typename Vec8<T>::type v;
        __builtin_memcpy(&v, p, sizeof(v));
        r = __builtin_convertvector(v, f32x8);
    } else if (!WHOLE) {
        for (int i = 0; i < 8; ++i) if (i < n) r[i] = (float)p[i];
    }
    return r;
}
template <bool WHOLE, class T>
__device__ __forceinline__ void store8(T* p, f32x8 x, int n) {
    const typename Vec8<T>::type v = __builtin_convertvector(x, typename Vec8<T>::type);
    if (n >= 8) __builtin_memcpy(p, &v, sizeof(v));
    else if (!WHOLE) for (int i = 0; i < 8; ++i) if (i < n) p[i] = v[i];
}

// Philox4x32, seven rounds (the fewest that its authors found to pass all tests of randomness): eight 16-bit numbers for group g.
__device__ __forceinline__ void philox(uint64_t g, uint64_t offset, uint64_t seed, unsigned (&c)[4]) {
    c[0] = (unsigned)g; c[1] = (unsigned)(g >> 32); c[2] = (unsigned)offset; c[3] = (unsigned)(offset >> 32);
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
        c[0] = (unsigned)(b >> 32) ^ c[1] ^ k0; c[1] = (unsigned)b;
        c[2] = (unsigned)(a >> 32) ^ c[3] ^ k1; c[3] = (unsigned)a;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
}
// Kept elements times the factor, zeros in place of the others, whatever they held.
__device__ __forceinline__ f32x8 drop8(f32x8 x, uint64_t g, uint64_t offset, const DropoutArgs& d) {
    unsigned c[4];
    philox(g, offset, d.seed, c);
    f32x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned u = i & 1 ? c[i / 2] >> 16 : c[i / 2] & 0xFFFFu;
        r[i] = u >= d.cut ? x[i] * d.factor : 0.0f;
    }
    return r;
}
__device__ __forceinline__ uint64_t drop_offset(const DropoutArgs& d) { return d.offset + (d.cut && d.d_offset ? *d.d_offset : 0); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
// Over the TPR threads of a row.  `side` alternates from use to use: the one barrier keeps this use's writes apart from the reads of
// the one before last.
template <int TPR, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float (*part)[TPR > 64 ? TPR / 64 : 1], int& side) {
    v = MAX ? wave_max(v) : wave_sum(v);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) part[side][threadIdx.x / 64] = v;
        __syncthreads();
        float t = part[side][0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) t = MAX ? fmaxf(t, part[side][i]) : t + part[side][i];
        v = t;
        side ^= 1;
    }
    return v;
}

template <class T, int TPR, int NV, bool E4M3, bool WHOLE>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) add_norm_kernel(AddNormArgs a) {
    __shared__ float part[2][TPR > 64 ? TPR / 64 : 1];
    int side = 0;
    constexpr int RPB = TPR >= 256 ? 1 : 256 / TPR;
    const int lane = threadIdx.x % TPR, dim = a.dim;
    const int groups = (dim + 7) / 8;
    const uint64_t offset = drop_offset(a.drop);
    for (int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; r < a.rows; r += (int64_t)gridDim.x * RPB) {
        const T* x = (const T*)a.x.p + r * a.x.ld;
        f32x8 h[NV], res[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) h[v] = load8<WHOLE>(x + (v * TPR + lane) * 8, dim - (v * TPR + lane) * 8);
        if (a.residual.p) {
            const T* q = (const T*)a.residual.p + r * a.residual.ld;
#pragma unroll
            for (int v = 0; v < NV; ++v) res[v] = load8<WHOLE>(q + (v * TPR + lane) * 8, dim - (v * TPR + lane) * 8);
        }
        if (a.drop.cut)
#pragma unroll
            for (int v = 0; v < NV; ++v) h[v] = drop8(h[v], (uint64_t)r * groups + v * TPR + lane, offset, a.drop);
        if (a.residual.p)
#pragma unroll
            for (int v = 0; v < NV; ++v) h[v] += res[v];
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(h[v][i], h[v][i], sum);
        if (a.h.p)
#pragma unroll
            for (int v = 0; v < NV; ++v) store8<WHOLE>((T*)a.h.p + r * a.h.ld + (v * TPR + lane) * 8, h[v], dim - (v * TPR + lane) * 8);
        const float rstd = 1.0f / sqrtf(row_reduce<TPR, false>(sum, part, side) / (float)dim + a.eps);
        if (a.rstd && lane == 0) a.rstd[r] = rstd;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = (v * TPR + lane) * 8;
            h[v] *= rstd;
            if (a.gain) h[v] *= load8<WHOLE>(a.gain + at, dim - at);
        }
        if constexpr (!E4M3) {
#pragma unroll
            for (int v = 0; v < NV; ++v) store8<WHOLE>((T*)a.y.p + r * a.y.ld + (v * TPR + lane) * 8, h[v], dim - (v * TPR + lane) * 8);
        } else {
            float most[NV], all = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                most[v] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) most[v] = fmaxf(most[v], fabsf(h[v][i]));
                all = fmaxf(all, most[v]);
            }
            if (a.group == 0) all = row_reduce<TPR, true>(all, part, side);
            const int blocks = a.group ? (dim + 127) / 128 : 1;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int at = (v * TPR + lane) * 8;
                float m = all;
                if (a.group) {      // 128 units: 16 neighbouring lanes
                    m = most[v];
#pragma unroll
                    for (int k = 8; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
                }
                float scale = m / 448.0f;
                if (!(scale > 0.0f)) scale = 1.0f;
                if (at < dim && (a.group ? lane % 16 == 0 : at == 0)) a.scales[r * blocks + (a.group ? at / 128 : 0)] = scale;
                // (a scale whose reciprocal is beyond fp32: divided)
                const float inv = 1.0f / scale;
                f32x8 q;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = scale > 1e-37f ? h[v][i] * inv : h[v][i] / scale;
                    q[i] = u != u ? u : fminf(fmaxf(u, -448.0f), 448.0f);
                }
                int w[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k], q[4 * k + 1], 0, false);
                    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k + 2], q[4 * k + 3], w[k], true);
                }
                unsigned char* y = (unsigned char*)a.y.p + r * a.y.ld + at;
                if (dim - at >= 8) __builtin_memcpy(y, w, 8);
                else if (!WHOLE) for (int i = 0; i < 8; ++i) if (at + i < dim) y[i] = (unsigned char)(w[i / 4] >> (8 * (i % 4)));
            }
        }
    }
}

template <class T, int TPR, int NV, bool WHOLE>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) add_norm_grad_kernel(AddNormGradArgs a) {
    constexpr int RPB = TPR >= 256 ? 1 : 256 / TPR;
    __shared__ float part[2][TPR > 64 ? TPR / 64 : 1];
    __shared__ float columns[RPB > 1 ? (RPB - 1) * TPR * NV * 8 : 1];
    int side = 0;
    const int lane = threadIdx.x % TPR, dim = a.dim;
    const int groups = (dim + 7) / 8;
    const uint64_t offset = drop_offset(a.drop);
    f32x8 dg[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) dg[v] = 0.0f;
    for (int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; r < a.rows; r += (int64_t)gridDim.x * RPB) {
        f32x8 dy[NV], n[NV], dh[NV];
        const float rstd = a.rstd[r];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = (v * TPR + lane) * 8;
            dy[v] = load8<WHOLE>((const T*)a.dy.p + r * a.dy.ld + at, dim - at);
            n[v] = load8<WHOLE>((const T*)a.h.p + r * a.h.ld + at, dim - at);
        }
        if (a.dh.p)
#pragma unroll
            for (int v = 0; v < NV; ++v) dh[v] = load8<WHOLE>((const T*)a.dh.p + r * a.dh.ld + (v * TPR + lane) * 8, dim - (v * TPR + lane) * 8);
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = (v * TPR + lane) * 8;
            n[v] *= rstd;
            dg[v] += dy[v] * n[v];
            if (a.gain) dy[v] *= load8<WHOLE>(a.gain + at, dim - at);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(dy[v][i], n[v][i], sum);
        }
        const float mean = row_reduce<TPR, false>(sum, part, side) / (float)dim;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = (v * TPR + lane) * 8;
            f32x8 s = rstd * (dy[v] - n[v] * mean);
            if (a.dh.p) s += dh[v];
            if (a.dresidual.p) store8<WHOLE>((T*)a.dresidual.p + r * a.dresidual.ld + at, s, dim - at);
            if (a.dx.p) {
                if (a.drop.cut) s = drop8(s, (uint64_t)r * groups + v * TPR + lane, offset, a.drop);
                store8<WHOLE>((T*)a.dx.p + r * a.dx.ld + at, s, dim - at);
            }
        }
    }
    if (!a.dgain) return;
    if constexpr (RPB > 1) {      // the wavefronts' sums, added in order by the first
        const int w = threadIdx.x / TPR;
        if (w > 0)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) columns[(((w - 1) * NV + v) * 8 + i) * TPR + lane] = dg[v][i];
        __syncthreads();
        if (w > 0) return;
        for (int u = 0; u < RPB - 1; ++u)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) dg[v][i] += columns[((u * NV + v) * 8 + i) * TPR + lane];
    }
    float* out = gridDim.x == 1 ? a.dgain : a.partial + (int64_t)blockIdx.x * dim;
#pragma unroll
    for (int v = 0; v < NV; ++v) store8<WHOLE>(out + (v * TPR + lane) * 8, dg[v], dim - (v * TPR + lane) * 8);
}

// out[c] = sum of `rows` rows of `partial`, in one order: 32 runs of rows for each of 32 columns, a run in eight sums (eight loads in
// flight), then the runs.
__global__ void __launch_bounds__(1024) sum_rows_kernel(const float* partial, float* out, int rows, int dim) {
    __shared__ float part[32][33];
    const int x = threadIdx.x % 32, c = blockIdx.x * 32 + x, run = threadIdx.x / 32;
    const float* p = partial + min(c, dim - 1);
    float s[8] = {};
    int r = run;
    for (; r + 7 * 32 < rows; r += 8 * 32) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[(int64_t)(r + 32 * i) * dim];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += v[i];
    }
    for (; r < rows; r += 32) s[0] += p[(int64_t)r * dim];
    part[run][x] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    if (run > 0 || c >= dim) return;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += part[i][x];
    out[c] = sum;
}

__global__ void __launch_bounds__(256) zero_kernel(float* p, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0.0f;
}

__global__ void count_kernel(int64_t* p, int64_t add, bool fresh) { *p = (fresh ? 0 : *p) + add; }

// A thread takes groups of eight units, four of them in flight.
template <class T, bool WHOLE>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutRowsArgs a) {
    constexpr int U = 4;
    const unsigned groups = ((unsigned)a.dim + 7) / 8;
    const uint64_t total = (uint64_t)a.rows * groups, offset = drop_offset(a.drop);
    const int64_t first_row = a.first_row + (a.d_first_row ? *a.d_first_row : 0);
    for (uint64_t base = (uint64_t)blockIdx.x * (256 * U); base < total; base += (uint64_t)gridDim.x * (256 * U)) {
        f32x8 x[U];
        int64_t row[U]; int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t g = base + u * 256 + threadIdx.x;
            at[u] = a.dim;
            if (g >= total) continue;
            row[u] = total >> 32 ? (int64_t)(g / groups) : (int64_t)((unsigned)g / groups);
            at[u] = (int)(g - (uint64_t)row[u] * groups) * 8;
            x[u] = load8<WHOLE>((const T*)a.x.p + row[u] * a.x.ld + at[u], a.dim - at[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at[u] >= a.dim) continue;
            f32x8 y = x[u];
            if (a.drop.cut) y = drop8(y, (uint64_t)(row[u] + first_row) * groups + at[u] / 8, offset, a.drop);
            store8<WHOLE>((T*)a.y.p + row[u] * a.y.ld + at[u], y, a.dim - at[u]);
        }
    }
}

// Threads to a row and vectors to a thread, by the row's width: as few threads as keep up to 2 vectors (16 units) each, so that a row's loads are
// all in flight and its tensors fit the registers.  Forward / backward with all tensors, bf16, 2^26 units, us: 1,024 units 100 / 113 (256 threads, 1
// vector: 130 / 184); 2,048 units 100 / 120 (64 threads, 4 vectors: 108 / 279); 8,192 units 103 / 132 (256 threads, 4 vectors: 116 / 288).
template <class F>
hipError_t by_width(int dim, F f) {
    if (dim <= 512) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (dim <= 1024) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (dim <= 2048) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    if (dim <= 4096) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    if (dim <= 8192) return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
    return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}
static_assert(NORM_MAX_DIM == 1024 * 2 * 8, "the widest row");
template <class F>
hipError_t by_type(int dtype, F f) {
    if (dtype == DT_F32) return f((float*)nullptr);
    if (dtype == DT_BF16) return f((bf16_t*)nullptr);
    return f((f16_t*)nullptr);
}
constexpr int64_t MOST_BLOCKS = 1 << 20;      // (a grid's threads stay below 2^32)
int rows_per_block(int dim) { return dim <= 1024 ? 4 : 1; }

}  // namespace

hipError_t launch_add_norm(int dtype, const AddNormArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return by_type(dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        return by_width(a.dim, [&](auto tpr, auto nv) {
            constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, RPB = TPR >= 256 ? 1 : 256 / TPR;
            const unsigned blocks = (unsigned)std::min<int64_t>(MOST_BLOCKS, (a.rows + RPB - 1) / RPB);
            const bool whole = a.dim % 8 == 0;
            auto* kernel = a.scales ? (whole ? add_norm_kernel<T, TPR, NV, true, true> : add_norm_kernel<T, TPR, NV, true, false>)
                                    : (whole ? add_norm_kernel<T, TPR, NV, false, true> : add_norm_kernel<T, TPR, NV, false, false>);
            kernel<<<blocks, TPR > 256 ? TPR : 256, 0, s>>>(a);
            return hipGetLastError();
        });
    });
}

// Blocks of the gradient kernel, each with a row of partial sums of dgain (0: no rows; 1: dgain is stored whole).
int norm_grad_blocks(int64_t rows, int dim) {
    const int64_t blocks = (rows + rows_per_block(dim) - 1) / rows_per_block(dim);
    return (int)std::min<int64_t>(blocks, std::min<int64_t>(1024, std::max<int64_t>(1, (1 << 24) / dim)));
}

hipError_t launch_add_norm_grad(int dtype, const AddNormGradArgs& a, hipStream_t s) {
    if (a.rows == 0) {
        if (a.dgain) zero_kernel<<<(a.dim + 255) / 256, 256, 0, s>>>(a.dgain, a.dim);
        return hipGetLastError();
    }
    hipError_t e = by_type(dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        return by_width(a.dim, [&](auto tpr, auto nv) {
            constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
            auto* kernel = a.dim % 8 == 0 ? add_norm_grad_kernel<T, TPR, NV, true> : add_norm_grad_kernel<T, TPR, NV, false>;
            kernel<<<(unsigned)a.blocks, TPR > 256 ? TPR : 256, 0, s>>>(a);
            return hipGetLastError();
        });
    });
    if (e == hipSuccess && a.dgain && a.blocks > 1) {
        sum_rows_kernel<<<(a.dim + 31) / 32, 1024, 0, s>>>(a.partial, a.dgain, a.blocks, a.dim);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_count(int64_t* p, int64_t add, bool fresh, hipStream_t s) {
    count_kernel<<<1, 1, 0, s>>>(p, add, fresh);
    return hipGetLastError();
}

hipError_t launch_dropout(int dtype, const DropoutRowsArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int64_t total = a.rows * (((int64_t)a.dim + 7) / 8);
    return by_type(dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        auto* kernel = a.dim % 8 == 0 ? dropout_kernel<T, true> : dropout_kernel<T, false>;
        kernel<<<(unsigned)std::min<int64_t>(MOST_BLOCKS, (total + 1023) / 1024), 256, 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace rnng
