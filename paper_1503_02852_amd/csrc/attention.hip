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

// ---------------------------------------------------------------------------------------------
// In chunks of C frames.  With g = exp(log decay), i and j frames of a chunk and S the state before it:
//     o_i = out (g^(i + early) S^T q_i + update sum_{j <= i} g^(i - j) (q_i . k_j) v_j)
//     S  <- g^rows S + update sum_j g^(rows - j - early) k_j v_j^T
// A workgroup has BV = 64 NT columns of one head's state, 16 NT to each of its four wavefronts, and walks over the chunks (of a
// segment, if the frames are split).  Everything but the decays is matrix products on 16 x 16 tiles:
//     scores  K Q^T, the tiles j <= i shared out over the wavefronts, decayed and handed on through LDS
//     output  transposed, [columns][frames]: S^T Q^T, scaled by a frame's power of g, plus V^T P^T: a lane then has 4 NT neighbouring
//             columns of one frame to store
//     state   K^T V', V' = V times the frames' powers of g
// A state tile stays in the accumulator layout (a lane has one column and 4 neighbouring rows of it), which is the layout of a
// product's first operand over those rows: the state never leaves the registers, and q is read in the rows' order.  The operands that run
// along frames (V, K^T) come out of LDS through the transposing read.
// fp32 takes the matrix cores' fp32 products.  bf16 takes its inputs as they are; what is computed is split: scores and state into two
// parts of 8 bits (2^-17 of each is lost, against the 2^-9 of the result's own rounding), V' into PARTS: three keep all 24 bits of a
// state that is handed on.  (One part each would double the error of a result in bf16.)
// ---------------------------------------------------------------------------------------------
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct ChunkOps {
    AttnOp op[3];
    float* seg_state[3];      // [segment][stream, head][dk][dv]: what a segment adds to the state, then the state before it
    int n_ops, slices, n_seg, seg_len;
    unsigned works;
};

// Four frames (rows) x 16 columns of 16-bit values: lane l of 16 gives the place of four columns 4 (l % 4) of row l / 4 and receives column
// l of the four rows.
__device__ __forceinline__ s16x4 lds_transposed(const bf16_t* p) {
    typedef __attribute__((address_space(3))) s16x4 lds_t;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)p);
}
__device__ __forceinline__ bf16x8 join(s16x4 a, s16x4 b) {
    union { s16x4 h[2]; bf16x8 v; } u;
    u.h[0] = a; u.h[1] = b;
    return u.v;
}
__device__ __forceinline__ bf16x8 split(f32x8& x) {      // the leading 8 bits; the rest stays in x
    const bf16x8 hi = __builtin_convertvector(x, bf16x8);
    x -= __builtin_convertvector(hi, f32x8);
    return hi;
}

// 16 bytes of a row from unit `at` on, zeros from unit `dim` on.
template <class T>
__device__ __forceinline__ u32x4 load16(const T* row, int at, int dim, bool there) {
    constexpr int E = 16 / sizeof(T);
    u32x4 r = 0u;
    if (!there || at >= dim) return r;
    if (at + E <= dim) { __builtin_memcpy(&r, row + at, 16); return r; }
    for (int i = 0; i < E - 1; ++i) {
        if (at + i >= dim) continue;
        if constexpr (sizeof(T) == 4) r[i] = __builtin_bit_cast(unsigned, row[at + i]);
        else r[i / 2] |= (unsigned)__builtin_bit_cast(unsigned short, row[at + i]) << (16 * (i % 2));
    }
    return r;
}

template <class T, int DK> constexpr int chunk_frames() { return sizeof(T) == 4 || DK > 128 ? 32 : 64; }

// A tile of C frames x D units on its way from memory to LDS, in registers.
template <class T, int C, int D>
struct Tile {
    static constexpr int E = 16 / sizeof(T), PIECES = C * D / E / 256, PITCH = D + (sizeof(T) == 4 ? 4 : 8);
    static_assert(C * D / E % 256 == 0, "tile");
    u32x4 r[PIECES];
    __device__ __forceinline__ void load(const AttnTensor& a, int n, int h, int first, int rows, int unit, int dim, bool reverse, int L) {
        const T* base = (const T*)a.p + n * a.sn + (h / a.group) * a.sh;
#pragma unroll
        for (int x = 0; x < PIECES; ++x) {
            const int p = x * 256 + threadIdx.x, row = p / (D / E), at = unit + p % (D / E) * E;
            const int i = first + row, t = reverse ? L - 1 - i : i;
            r[x] = load16(base + t * a.st, at, dim, row < rows);
        }
    }
    __device__ __forceinline__ void store(T* lds) const {
#pragma unroll
        for (int x = 0; x < PIECES; ++x) {
            const int p = x * 256 + threadIdx.x;
            *(u32x4*)(lds + p / (D / E) * PITCH + p % (D / E) * E) = r[x];
        }
    }
};

template <class T, int DK, int NT, int PARTS, bool STATE>
__global__ void __launch_bounds__(256, 2) attention_chunks_kernel(AttnCall c, ChunkOps ops) {
    constexpr int C = chunk_frames<T, DK>(), BV = 64 * NT, IT = C / 16, AT = DK / 16;
    constexpr bool F32 = sizeof(T) == 4;
    typedef Tile<T, C, DK> TileK;
    typedef Tile<T, C, BV> TileV;
    constexpr int PP = C + (F32 ? 4 : 8);                                  // pitch of the scores
    __shared__ alignas(16) T lds_q[STATE ? 1 : C * TileK::PITCH];
    __shared__ alignas(16) T lds_k[C * TileK::PITCH];
    __shared__ alignas(16) T lds_v[C * TileV::PITCH];
    __shared__ alignas(16) T lds_p[STATE ? 1 : (F32 ? 1 : 2) * C * PP];
    __shared__ float power[C + 1], power_low[C + 1], weight[2 * C];       // g^i and what its rounding left; update g^(C - j - early), zeros

    // Workgroups go to the eight XCDs in turn; neighbours in the list of works (slices of a head, gradients of it, heads that share keys) read the same
    // tensors and are put on one.
    const unsigned each = (ops.works + 7) / 8;
    unsigned w = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (blockIdx.x / 8 >= each || w >= ops.works) return;
    const int slice = w % ops.slices; w /= ops.slices;
    const int which = w % ops.n_ops; w /= ops.n_ops;
    const int h = w % c.heads; w /= c.heads;
    const int n = w % c.N, seg = w / c.N;
    const AttnOp& a = ops.op[which];
    const int col0 = slice * BV;
    if (col0 >= a.dv) return;
    const int L = length_of(c, n), begin = seg * ops.seg_len, end = min(L, begin + ops.seg_len);
    if (begin >= end && (STATE || seg > 0)) return;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16, m = lane % 16;
    // the lane's columns: as a result's column, and the first of 4 NT neighbouring ones of an output
    const int my_col = 16 * NT * wave + (NT == 2 ? 8 * (m / 4) + m % 4 : m), out_col = col0 + 16 * NT * wave + 4 * NT * g;

    const float ld = log_decay_of(c, h);
    if (threadIdx.x <= C) {
        const double p = exp((double)ld * (int)threadIdx.x);
        power[threadIdx.x] = (float)p;
        power_low[threadIdx.x] = (float)(p - (float)p);
    }
    if (threadIdx.x < 2 * C) weight[threadIdx.x] = threadIdx.x < C ? a.update * expf(ld * (C - (int)threadIdx.x - (a.early ? 1 : 0))) : 0.0f;

    f32x4 S[AT][NT];
    const int64_t nh = (int64_t)n * c.heads + h, heads = (int64_t)c.N * c.heads, size = (int64_t)a.dk * a.dv;
    {
        const bool seg_state = !STATE && ops.n_seg > 1;
        const float* from = STATE ? nullptr : seg_state ? ops.seg_state[which] + (seg * heads + nh) * size : a.s_in ? a.s_in + nh * size : nullptr;
        const int64_t si = seg_state ? a.dv : a.si, sj = seg_state ? 1 : a.sj;
#pragma unroll
        for (int t = 0; t < AT; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * t + 4 * g + r, j = col0 + my_col + 4 * nt;
                    S[t][nt][r] = from && i < a.dk && j < a.dv ? from[i * si + j * sj] : 0.0f;
                }
    }
    TileK tq, tk;
    TileV tv;
    auto load = [&](int first) {
        const int rows = end - first;
        if constexpr (!STATE) tq.load(a.q, n, h, first, rows, 0, a.dk, a.reverse, L);
        tk.load(a.k, n, h, first, rows, 0, a.dk, a.reverse, L);
        tv.load(a.v, n, h, first, rows, col0, a.dv, a.reverse, L);
    };
    load(begin);
    const float both = a.out * a.update;
    for (int first = begin; first < end; first += C) {
        const int rows = min(C, end - first);
        __syncthreads();                       // the last chunk's tiles have been read (and, first, the tables are there)
        if constexpr (!STATE) tq.store(lds_q);
        tk.store(lds_k);
        tv.store(lds_v);
        __syncthreads();
        if (first + C < end) load(first + C);
        if constexpr (!STATE) {
            f32x4 acc[IT][NT];
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[it][nt] = 0.0f;
            if (a.o.p) {
                // scores of the tiles (16 frames i, 16 frames j) that the products below read: j up to the end of i's pair of tiles
#pragma unroll
                for (int x = 0; x < (IT == 4 ? 3 : 1); ++x) {
                    const int e = wave + 4 * x, it = e < 4 ? e / 2 : 2 + (e - 4) / 4, jt = e < 4 ? e % 2 : e % 4;
                    f32x4 s = 0.0f;
                    if (jt <= it) {
                        if constexpr (F32) {
#pragma unroll
                            for (int t = 0; t < AT; ++t) {
                                const f32x4 k = *(const f32x4*)(lds_k + (16 * jt + m) * TileK::PITCH + 16 * t + 4 * g);
                                const f32x4 q = *(const f32x4*)(lds_q + (16 * it + m) * TileK::PITCH + 16 * t + 4 * g);
#pragma unroll
                                for (int r = 0; r < 4; ++r) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[r], q[r], s, 0, 0, 0);
                            }
                        } else {
#pragma unroll
                            for (int t = 0; t < DK / 32; ++t)
                                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)(lds_k + (16 * jt + m) * TileK::PITCH + 32 * t + 8 * g),
                                                                            *(const bf16x8*)(lds_q + (16 * it + m) * TileK::PITCH + 32 * t + 8 * g), s, 0, 0, 0);
                        }
                    }
                    const int i = 16 * it + m, j = 16 * jt + 4 * g;
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[r] = i >= j + r ? s[r] * (both * power[i >= j + r ? i - j - r : 0]) : 0.0f;
                    if constexpr (F32) *(f32x4*)(lds_p + i * PP + j) = s;
                    else {
                        const bf16x4 hi = __builtin_convertvector(s, bf16x4);
                        *(bf16x4*)(lds_p + i * PP + j) = hi;
                        *(bf16x4*)(lds_p + (C + i) * PP + j) = __builtin_convertvector(s - __builtin_convertvector(hi, f32x4), bf16x4);
                    }
                }
                // the state's part
                if constexpr (F32) {
#pragma unroll
                    for (int t = 0; t < AT; ++t)
#pragma unroll
                        for (int it = 0; it < IT; ++it) {
                            const f32x4 q = *(const f32x4*)(lds_q + (16 * it + m) * TileK::PITCH + 16 * t + 4 * g);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) acc[it][nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(S[t][nt][r], q[r], acc[it][nt], 0, 0, 0);
                        }
                } else {
#pragma unroll
                    for (int t = 0; t < DK / 32; ++t) {
                        bf16x8 hi[NT], lo[NT];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            f32x8 s = __builtin_shufflevector(S[2 * t][nt], S[2 * t + 1][nt], 0, 1, 2, 3, 4, 5, 6, 7);
                            hi[nt] = split(s);
                            lo[nt] = __builtin_convertvector(s, bf16x8);
                        }
#pragma unroll
                        for (int it = 0; it < IT; ++it) {
                            const bf16_t* q = lds_q + (16 * it + m) * TileK::PITCH + 32 * t + 4 * g;
                            const bf16x8 qf = join(*(const s16x4*)q, *(const s16x4*)(q + 16));
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                acc[it][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi[nt], qf, acc[it][nt], 0, 0, 0);
                                acc[it][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo[nt], qf, acc[it][nt], 0, 0, 0);
                            }
                        }
                    }
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const float x = a.out * power[16 * it + m + (a.early ? 1 : 0)];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) acc[it][nt] *= x;
                }
            }
            __syncthreads();                   // the scores are there
            if (a.o.p) {
                if constexpr (F32) {
#pragma unroll
                    for (int jt = 0; jt < IT; ++jt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float v[NT];
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) v[nt] = lds_v[(16 * jt + 4 * g + r) * TileV::PITCH + my_col + 4 * nt];
#pragma unroll
                            for (int it = jt; it < IT; ++it) {
                                const float p = lds_p[(16 * it + m) * PP + 16 * jt + 4 * g + r];
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) acc[it][nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[nt], p, acc[it][nt], 0, 0, 0);
                            }
                        }
                } else {
#pragma unroll
                    for (int s = 0; s < C / 32; ++s) {
                        bf16x8 v[NT];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const bf16_t* p = lds_v + (32 * s + 8 * g + m / 4) * TileV::PITCH + 16 * NT * wave + 4 * NT * (m % 4) + 4 * nt;
                            v[nt] = join(lds_transposed(p), lds_transposed(p + 4 * TileV::PITCH));
                        }
#pragma unroll
                        for (int it = 2 * s; it < IT; ++it) {
                            const bf16_t* p = lds_p + (16 * it + m) * PP + 32 * s + 8 * g;
                            const bf16x8 hi = *(const bf16x8*)p, lo = *(const bf16x8*)(p + C * PP);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                acc[it][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[nt], hi, acc[it][nt], 0, 0, 0);
                                acc[it][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[nt], lo, acc[it][nt], 0, 0, 0);
                            }
                        }
                    }
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int i = 16 * it + m;
                    if (i >= rows || out_col >= a.dv) continue;
                    const int t = a.reverse ? L - 1 - first - i : first + i;
                    const int64_t at = t * a.o.st + n * a.o.sn + h * a.o.sh + out_col;
                    typedef float out_f32 __attribute__((ext_vector_type(4 * NT)));
                    typedef T out_t __attribute__((ext_vector_type(4 * NT)));
                    out_f32 x;
#pragma unroll
                    for (int u = 0; u < 4 * NT; ++u) x[u] = acc[it][u / 4][u % 4];
                    const out_t y = __builtin_convertvector(x, out_t);
                    if (out_col + 4 * NT <= a.dv) {
                        if (a.o_f32) __builtin_memcpy((float*)a.o.p + at, &x, sizeof(x));
                        else __builtin_memcpy((T*)a.o.p + at, &y, sizeof(y));
                    } else {
#pragma unroll
                        for (int u = 0; u < 4 * NT; ++u)
                            if (out_col + u < a.dv) { if (a.o_f32) ((float*)a.o.p)[at + u] = x[u]; else ((T*)a.o.p)[at + u] = y[u]; }
                    }
                }
            }
        }
        // the state after the chunk
        const float ph = power[rows], pl = power_low[rows];
#pragma unroll
        for (int t = 0; t < AT; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][nt][r] = fmaf(S[t][nt][r], ph, S[t][nt][r] * pl);
        const float* wt = weight + C - rows;
        if constexpr (F32) {
#pragma unroll
            for (int jt = 0; jt < IT; ++jt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jt + 4 * g + r;
                    float v[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) v[nt] = lds_v[j * TileV::PITCH + my_col + 4 * nt] * wt[j];
#pragma unroll
                    for (int t = 0; t < AT; ++t) {
                        const float k = lds_k[j * TileK::PITCH + 16 * t + m];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) S[t][nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k, v[nt], S[t][nt], 0, 0, 0);
                    }
                }
        } else {
#pragma unroll
            for (int s = 0; s < C / 32; ++s) {
                bf16x8 v[NT][PARTS];
                f32x8 wv;
#pragma unroll
                for (int e = 0; e < 8; ++e) wv[e] = wt[32 * s + 8 * g + e];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const bf16_t* p = lds_v + (32 * s + 8 * g + m / 4) * TileV::PITCH + 16 * NT * wave + 4 * NT * (m % 4) + 4 * nt;
                    f32x8 x = __builtin_convertvector(join(lds_transposed(p), lds_transposed(p + 4 * TileV::PITCH)), f32x8) * wv;
#pragma unroll
                    for (int u = 0; u < PARTS; ++u) v[nt][u] = split(x);
                }
#pragma unroll
                for (int t = 0; t < AT; ++t) {
                    const bf16_t* p = lds_k + (32 * s + 8 * g + m / 4) * TileK::PITCH + 16 * t + 4 * (m % 4);
                    const bf16x8 k = join(lds_transposed(p), lds_transposed(p + 4 * TileK::PITCH));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int u = 0; u < PARTS; ++u) S[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, v[nt][u], S[t][nt], 0, 0, 0);
                }
            }
        }
    }
    float* to = STATE ? ops.seg_state[which] + (seg * heads + nh) * size : a.s_out && end == L ? a.s_out + nh * size : nullptr;
    if (!to) return;
    const int64_t si = STATE ? a.dv : a.si, sj = STATE ? 1 : a.sj;
#pragma unroll
    for (int t = 0; t < AT; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * g + r, j = col0 + my_col + 4 * nt;
                if (i < a.dk && j < a.dv) to[i * si + j * sj] = S[t][nt][r];
            }
}

// What the segments add to the state becomes the state before each, in place.
__global__ void __launch_bounds__(256) attention_segments_kernel(AttnCall c, ChunkOps ops) {
    const AttnOp& a = ops.op[blockIdx.z];
    const int64_t size = (int64_t)a.dk * a.dv, heads = (int64_t)c.N * c.heads, nh = blockIdx.y;
    const int x = blockIdx.x * 256 + threadIdx.x;
    if (x >= size) return;
    const int L = length_of(c, (int)(nh / c.heads));
    const double ld = log_decay_of(c, (int)(nh % c.heads));
    float S = a.s_in ? a.s_in[nh * size + x / a.dv * a.si + x % a.dv * a.sj] : 0.0f;
    const float whole = (float)exp(ld * ops.seg_len);
    float* p = ops.seg_state[blockIdx.z] + nh * size + x;
    for (int s = 0; s < ops.n_seg; ++s, p += heads * size) {
        const int rows = min(L - s * ops.seg_len, ops.seg_len);
        if (s > 0 && rows <= 0) return;
        const float add = s + 1 < ops.n_seg && rows > 0 ? *p : 0.0f;
        *p = S;
        S = fmaf(S, rows == ops.seg_len ? whole : (float)exp(ld * rows), add);
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

static hipError_t launch_attention_steps(const AttnCall& c, const AttnOp* ops, int n_ops, hipStream_t s) {
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

// Segments of the frames, so that the chip is filled (two workgroups to a compute unit) where streams and heads are few.
static void plan_segments(int T, int64_t works, int C, int& n_seg, int& seg_len) {
    const int64_t chunks = (T + C - 1) / C;
    int64_t n = works >= 256 ? 1 : std::min<int64_t>((512 + works - 1) / works, chunks / 4);
    n = std::max<int64_t>(n, 1);
    const int64_t per = (chunks + n - 1) / n;
    seg_len = (int)(per * C);
    n_seg = std::max<int>(1, (int)((chunks + per - 1) / per));
}
namespace {
struct ChunkShape { int DK, NT, C, slices; };
ChunkShape chunk_shape(int dtype, int dk, int dv) {
    ChunkShape s;
    s.DK = dk <= 64 ? 64 : dk <= 128 ? 128 : 256;
    s.NT = dv <= 64 || s.DK == 256 ? 1 : 2;      // (256 rows x 32 columns a wavefront would not fit its registers)
    s.C = dtype == DT_F32 || s.DK > 128 ? 32 : 64;
    s.slices = (dv + 64 * s.NT - 1) / (64 * s.NT);
    return s;
}
}  // namespace

int64_t attention_space(const AttnCall& c, const AttnOp* ops, int n_ops) {
    if (c.T <= ATTN_STEPS || n_ops == 0) return 0;
    int dk = 0, dv = 0;
    int64_t floats = 0;
    for (int i = 0; i < n_ops; ++i) { dk = std::max(dk, ops[i].dk); dv = std::max(dv, ops[i].dv); floats += ((int64_t)ops[i].dk * ops[i].dv * c.N * c.heads + 63) / 64 * 64; }
    const ChunkShape sh = chunk_shape(c.dtype, dk, dv);
    int n_seg, seg_len;
    plan_segments(c.T, (int64_t)c.N * c.heads * n_ops * sh.slices, sh.C, n_seg, seg_len);
    return n_seg > 1 ? n_seg * floats * 4 : 0;
}

hipError_t launch_attention(const AttnCall& c, const AttnOp* ops, int n_ops, float* space, hipStream_t s) {
    if (c.T <= ATTN_STEPS) return launch_attention_steps(c, ops, n_ops, s);
    ChunkOps co = {};
    int dk = 0, dv = 0;
    bool state = false;
    for (int i = 0; i < n_ops; ++i) { co.op[i] = ops[i]; dk = std::max(dk, ops[i].dk); dv = std::max(dv, ops[i].dv); state = state || ops[i].s_out; }
    const ChunkShape sh = chunk_shape(c.dtype, dk, dv);
    co.n_ops = n_ops; co.slices = sh.slices;
    plan_segments(c.T, (int64_t)c.N * c.heads * n_ops * sh.slices, sh.C, co.n_seg, co.seg_len);
    if (co.n_seg > 1)
        for (int i = 0; i < n_ops; ++i) {
            co.seg_state[i] = space;
            space += co.n_seg * (((int64_t)ops[i].dk * ops[i].dv * c.N * c.heads + 63) / 64 * 64);
        }
    auto launch = [&](auto kernel, int segments) {
        co.works = (unsigned)((int64_t)segments * c.N * c.heads * n_ops * sh.slices);
        kernel<<<(co.works + 7) / 8 * 8, 256, 0, s>>>(c, co);
        return hipGetLastError();
    };
    auto go = [&](auto* t, auto DKc, auto NTc) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int DK = decltype(DKc)::value, NT = decltype(NTc)::value;
        if (co.n_seg > 1) {
            hipError_t e = launch(attention_chunks_kernel<T, DK, NT, 3, true>, co.n_seg - 1);
            if (e != hipSuccess) return e;
            attention_segments_kernel<<<dim3((unsigned)((dk * dv + 255) / 256), (unsigned)(c.N * c.heads), (unsigned)n_ops), 256, 0, s>>>(c, co);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if constexpr (sizeof(T) == 2) if (!state) return launch(attention_chunks_kernel<T, DK, NT, 2, false>, co.n_seg);
        return launch(attention_chunks_kernel<T, DK, NT, 3, false>, co.n_seg);
    };
    auto by_width = [&](auto* t) {
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        if (sh.DK == 64) return sh.NT == 1 ? go(t, std::integral_constant<int, 64>(), One()) : go(t, std::integral_constant<int, 64>(), Two());
        if (sh.DK == 128) return sh.NT == 1 ? go(t, std::integral_constant<int, 128>(), One()) : go(t, std::integral_constant<int, 128>(), Two());
        return go(t, std::integral_constant<int, 256>(), One());
    };
    return c.dtype == DT_F32 ? by_width((float*)nullptr) : by_width((bf16_t*)nullptr);
}

hipError_t launch_attention_sum_heads(const AttnCall& c, const float* part, const AttnOut& out, int d, int group, hipStream_t s) {
    const int64_t total = (int64_t)c.T * c.N * (c.heads / group) * d;
    const unsigned blocks = (unsigned)std::min<int64_t>(1 << 20, (total + 255) / 256);
    if (c.dtype == DT_F32) attention_sum_heads_kernel<float><<<blocks, 256, 0, s>>>(c, part, out, d, group);
    else attention_sum_heads_kernel<bf16_t><<<blocks, 256, 0, s>>>(c, part, out, d, group);
    return hipGetLastError();
}

}  // namespace rnng
