// Linear attention with a decay for each head (the operator that layers.h writes down).
#include "layers.h"

#include <algorithm>

namespace rnng {
namespace {

typedef __bf16 bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 0 >= log decay; a positive one counts as 0 (and so does NaN).  exp is 0 from about -104 on, so the bound below changes no value, and
// 0 times it is 0 (0 times -inf is not).
__device__ __forceinline__ float log_decay_of(const AttnCall& c, int h) { return fmaxf(fminf(c.log_decay[h], 0.0f), -1000.0f); }
__device__ __forceinline__ int length_of(const AttnCall& c, int n) { return c.lengths ? min(max(c.lengths[n], 0), c.T) : c.T; }

// ---------------------------------------------------------------------------------------------
// Frame by frame.  A workgroup keeps 64 columns of one head's state in registers: 16 lanes of 4 columns, 16 of these side by side
// with the rows r = lane group + 16 x.  For single frames it reads and writes the state once and is bound by that.
// ---------------------------------------------------------------------------------------------
struct StepOps { AttnOp op[3]; };

template <class T, int NR>
__global__ void __launch_bounds__(256) attention_steps_kernel(AttnCall c, StepOps ops, int slices) {
    const AttnOp& a = ops.op[blockIdx.y];
    const int n = blockIdx.x / slices / c.heads, h = blockIdx.x / slices % c.heads;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16, col = (blockIdx.x % slices) * 64 + tx * 4;
    if ((blockIdx.x % slices) * 64 >= a.dv) return;      // (operators of one launch may differ in dv)
    __shared__ float sum[2][4][64];
    const int L = length_of(c, n);
    const float g = expf(log_decay_of(c, h));
    const int64_t s0 = ((int64_t)n * c.heads + h) * a.dk * a.dv;
    const bool wide = a.sj == 1 && a.dv % 4 == 0;        // (a row's quads are whole then, and aligned if the state is)
    const bool aligned = wide && (((uintptr_t)a.s_in | (uintptr_t)a.s_out) & 15) == 0;
    f32x4 S[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int i = ty + 16 * r;
        S[r] = 0.0f;
        if (!a.s_in || i >= a.dk || col >= a.dv) continue;
        const float* p = a.s_in + s0 + i * a.si + col * a.sj;
        if (aligned) S[r] = *(const f32x4*)p;
        else for (int j = 0; j < 4; ++j) if (col + j < a.dv) S[r][j] = p[j * a.sj];
    }
    const T* qp = (const T*)a.q.p + n * a.q.sn + (h / a.q.group) * a.q.sh;
    const T* kp = (const T*)a.k.p + n * a.k.sn + (h / a.k.group) * a.k.sh;
    const T* vp = (const T*)a.v.p + n * a.v.sn + (h / a.v.group) * a.v.sh;
    for (int i = 0; i < L; ++i) {
        const int t = a.reverse ? L - 1 - i : i;
        float q[NR], k[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = ty + 16 * r;
            q[r] = a.o.p && row < a.dk ? (float)qp[t * a.q.st + row] : 0.0f;
            k[r] = row < a.dk ? (float)kp[t * a.k.st + row] * a.update : 0.0f;
        }
        f32x4 v = 0.0f, o = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) if (col + j < a.dv) v[j] = (float)vp[t * a.v.st + col + j];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            if (a.early) S[r] *= g;
#pragma unroll
            for (int j = 0; j < 4; ++j) { S[r][j] = fmaf(k[r], v[j], S[r][j]); o[j] = fmaf(q[r], S[r][j], o[j]); }
            if (!a.early) S[r] *= g;
        }
        if (!a.o.p) continue;
        // over the lane groups of a wavefront, then over the four wavefronts
#pragma unroll
        for (int j = 0; j < 4; ++j) { o[j] += __shfl_xor(o[j], 16); o[j] += __shfl_xor(o[j], 32); }
        float (*part)[64] = sum[i & 1];                  // (the next frame writes the other half: one barrier a frame)
        if (ty % 4 == 0) *(f32x4*)&part[ty / 4][tx * 4] = o;
        __syncthreads();
        const int j = (blockIdx.x % slices) * 64 + threadIdx.x;
        if (threadIdx.x < 64 && j < a.dv) {
            const float x = a.out * (part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x]);
            const int64_t at = t * a.o.st + n * a.o.sn + h * a.o.sh + j;
            if (a.o_f32) ((float*)a.o.p)[at] = x;
            else ((T*)a.o.p)[at] = (T)x;
        }
    }
    if (!a.s_out) return;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int i = ty + 16 * r;
        if (i >= a.dk || col >= a.dv) continue;
        float* p = a.s_out + s0 + i * a.si + col * a.sj;
        if (aligned) *(f32x4*)p = S[r];
        else for (int j = 0; j < 4; ++j) if (col + j < a.dv) p[j * a.sj] = S[r][j];
    }
}

template <class T>
__global__ void __launch_bounds__(256) attention_sum_heads_kernel(AttnCall c, const float* part, AttnOut out, int d, int group) {
    const int kv_heads = c.heads / group;
    const int64_t total = (int64_t)c.T * c.N * kv_heads * d;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
        const int i = (int)(x % d);
        const int64_t row = x / d, frame = row / kv_heads;
        const int h = (int)(row % kv_heads), n = (int)(frame % c.N);
        const int64_t t = frame / c.N;
        if (t >= length_of(c, n)) continue;
        float s = 0.0f;
        for (int u = 0; u < group; ++u) s += part[(frame * c.heads + h * group + u) * d + i];
        ((T*)out.p)[t * out.st + n * out.sn + h * out.sh + i] = (T)s;
    }
}

}  // namespace

hipError_t launch_attention_steps(const AttnCall& c, const AttnOp* ops, int n_ops, hipStream_t s) {
    StepOps so;
    int dk = 0, dv = 0;
    for (int i = 0; i < n_ops; ++i) { so.op[i] = ops[i]; dk = std::max(dk, ops[i].dk); dv = std::max(dv, ops[i].dv); }
    const int slices = (dv + 63) / 64;
    const dim3 grid((unsigned)c.N * c.heads * slices, (unsigned)n_ops);
    auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (dk <= 64) attention_steps_kernel<T, 4><<<grid, 256, 0, s>>>(c, so, slices);
        else if (dk <= 128) attention_steps_kernel<T, 8><<<grid, 256, 0, s>>>(c, so, slices);
        else attention_steps_kernel<T, 16><<<grid, 256, 0, s>>>(c, so, slices);
        return hipGetLastError();
    };
    return c.dtype == DT_F32 ? go((float*)nullptr) : go((bf16_t*)nullptr);
}

hipError_t launch_attention_sum_heads(const AttnCall& c, const float* part, const AttnOut& out, int d, int group, hipStream_t s) {
    const int64_t total = (int64_t)c.T * c.N * (c.heads / group) * d;
    const unsigned blocks = (unsigned)std::min<int64_t>(1 << 20, (total + 255) / 256);
    if (c.dtype == DT_F32) attention_sum_heads_kernel<float><<<blocks, 256, 0, s>>>(c, part, out, d, group);
    else attention_sum_heads_kernel<bf16_t><<<blocks, 256, 0, s>>>(c, part, out, d, group);
    return hipGetLastError();
}

}  // namespace rnng
