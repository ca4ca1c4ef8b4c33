// Linear attention with a decay for each head (the operator that layers.h writes down).
#include "layers.h"

#include <algorithm>

namespace rnng {
namespace {

typedef __bf16 bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 0 >= log decay; a positive one counts as 0, NaN stays.  exp is 0 from about -104 on, so the bound below changes no value, and
// 0 times it is 0 (0 times -inf is not).
__device__ __forceinline__ float log_decay_of(const AttnCall& c, int h) {
    const float x = c.log_decay[h];
    return x != x ? x : fmaxf(fminf(x, 0.0f), -1000.0f);
}
__device__ __forceinline__ int length_of(const AttnCall& c, int n) { return c.lengths ? min(max(c.lengths[n], 0), c.T) : c.T; }

// ---------------------------------------------------------------------------------------------
// Frame by frame.  A workgroup keeps 64 columns of one head's state in registers: 16 lanes of 4 columns, 16 of these side by side
// with the rows r = lane group + 16 x.  For single frames it reads and writes the state once and is bound by that: 192 streams x 16 heads x
// 128 x 128 units 78 us (404 MB, 5.2 TB/s, as a copy).  Each further frame is a chain of its loads, sums over the rows and a barrier, 1.5 us.
// ---------------------------------------------------------------------------------------------
struct StepOps { AttnOp op[3]; };

// WIDE: rows of the state whose quads of columns are whole and aligned, four numbers to a load (64 streams x 16 heads x 128 x 128, one frame, 26 us;
// one number to a load, which transposed states need, 42).
template <class T, int NR, bool WIDE>
__global__ void __launch_bounds__(256) attention_steps_kernel(AttnCall c, StepOps ops, int slices) {
    const AttnOp& a = ops.op[blockIdx.y];
    const int n = blockIdx.x / slices / c.heads, h = blockIdx.x / slices % c.heads;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16, col0 = (blockIdx.x % slices) * 64, col = col0 + tx * 4;
    if (col0 >= a.dv) return;      // (operators of one launch may differ in dv)
    __shared__ float sum[2][4][64];
    const int L = length_of(c, n);
    const float g = expf(log_decay_of(c, h));
    const int64_t s0 = ((int64_t)n * c.heads + h) * a.dk * a.dv;
    const int si = (int)a.si, sj = (int)a.sj;
    f32x4 S[NR];
    // loads without conditions, all in flight together: places outside are read from the nearest inside and set to zero afterwards
    if (a.s_in) {
        const float* p = a.s_in + s0;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = min(ty + 16 * r, a.dk - 1) * si;
            if constexpr (WIDE) S[r] = *(const f32x4*)(p + row + min(col, a.dv - 4));
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) S[r][j] = p[row + min(col + j, a.dv - 1) * sj];
        }
    } else
#pragma unroll
        for (int r = 0; r < NR; ++r) S[r] = 0.0f;
    const T* qp = (const T*)a.q.p + n * a.q.sn + (h / a.q.group) * a.q.sh;
    const T* kp = (const T*)a.k.p + n * a.k.sn + (h / a.k.group) * a.k.sh;
    const T* vp = (const T*)a.v.p + n * a.v.sn + (h / a.v.group) * a.v.sh;
    T q[NR], k[NR], v[4];
    auto load = [&](int t) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = min(ty + 16 * r, a.dk - 1);
            if (a.o.p) q[r] = qp[t * a.q.st + row];
            k[r] = kp[t * a.k.st + row];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = vp[t * a.v.st + min(col + j, a.dv - 1)];
    };
    if (L > 0) load(a.reverse ? L - 1 : 0);
#pragma unroll
    for (int r = 0; r < NR; ++r) asm volatile("" : "+v"(S[r]));
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[r][j] = ty + 16 * r < a.dk && col + j < a.dv ? S[r][j] : 0.0f;
    for (int i = 0; i < L; ++i) {
        const int t = a.reverse ? L - 1 - i : i;
        float qf[NR], kf[NR];
        f32x4 vf, o = 0.0f;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const bool there = ty + 16 * r < a.dk;
            qf[r] = a.o.p && there ? (float)q[r] : 0.0f;
            kf[r] = there ? (float)k[r] * a.update : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) vf[j] = col + j < a.dv ? (float)v[j] : 0.0f;
        if (i + 1 < L) load(a.reverse ? t - 1 : t + 1);
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            if (a.early) S[r] *= g;
#pragma unroll
            for (int j = 0; j < 4; ++j) { S[r][j] = fmaf(kf[r], vf[j], S[r][j]); o[j] = fmaf(qf[r], S[r][j], o[j]); }
            if (!a.early) S[r] *= g;
        }
        if (!a.o.p) continue;
        // over the lane groups of a wavefront, then over the four wavefronts
#pragma unroll
        for (int j = 0; j < 4; ++j) { o[j] += __shfl_xor(o[j], 16); o[j] += __shfl_xor(o[j], 32); }
        float (*part)[64] = sum[i & 1];                  // (the next frame writes the other half: one barrier a frame)
        if (ty % 4 == 0) *(f32x4*)&part[ty / 4][tx * 4] = o;
        __syncthreads();
        const int j = col0 + threadIdx.x;
        if (threadIdx.x < 64 && j < a.dv) {
            const float x = a.out * (part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x]);
            const int64_t at = t * a.o.st + n * a.o.sn + h * a.o.sh + j;
            if (a.o_f32) ((float*)a.o.p)[at] = x;
            else ((T*)a.o.p)[at] = (T)x;
        }
    }
    if (!a.s_out) return;
    float* p = a.s_out + s0;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int i = ty + 16 * r;
        if (i >= a.dk || col >= a.dv) continue;
        if constexpr (WIDE) *(f32x4*)(p + i * si + col) = S[r];
        else for (int j = 0; j < 4; ++j) if (col + j < a.dv) p[i * si + (col + j) * sj] = S[r][j];
    }
}

// ---------------------------------------------------------------------------------------------
// In chunks of C frames.  With g = exp(log decay), i and j frames of a chunk and S the state before it:
//     o_i = out (g^(i + early) S^T q_i + update sum_{j <= i} g^(i - j) (q_i . k_j) v_j)
//     S  <- g^rows S + update sum_j g^(rows - j - early) k_j v_j^T
// A workgroup of W wavefronts has BV = 16 W columns of one head's state, 16 to a wavefront, and walks over the chunks (of a
// segment, if the frames are split).  Everything but the decays is matrix products on 16 x 16 tiles:
//     scores  K Q^T, the tiles j <= i shared out over the wavefronts, decayed and handed on through LDS
//     output  transposed, [columns][frames]: S^T Q^T, scaled by a frame's power of g, plus V^T P^T: a lane then has 4 neighbouring
//             columns of one frame to store
//     state   K^T V', V' = V times the frames' powers of g
// A state tile stays in the accumulator layout (a lane has one column and 4 neighbouring rows of it), which is the layout of a
// product's first operand over those rows: the state never leaves the registers.  The operands that run along frames (V, K^T) come out of
// LDS through the transposing read, which takes columns in fours from anywhere: state tiles 2 t and 2 t + 1 have the rows of which a lane
// reads eight neighbouring ones of q.
// fp32 takes the matrix cores' fp32 products.  bf16 takes its inputs as they are; what is computed goes to the matrix cores in several bf16 numbers
// whose sum it is.  V' in three, which keep all of its bits: the state is carried on in 32 bits, whether it is asked for or not.  Scores, and the
// state as an operand of the outputs, in OPERAND_PARTS = 2: 2^-16 of a term is lost at most (the upper eight bits are cut off, the rest is rounded to
// eight), which is what 256 of the fp32 additions that make a result (some 4 (dk + dv) + 8 a frame between) may take.  In one number 2^-9 of a term
// would be lost, which results whose terms cancel (keys and values around one, queries that sum up to nothing) do not stand.  In one / two / three,
// us, 2,048 frames x 8 streams x 16 heads x 128 x 128, forward: 132 / 134 / 141, backward: 221 / 251 / 271; 65,536 frames, 8 heads: 197 / 209 / 223.
// ---------------------------------------------------------------------------------------------
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Measured, 2,048 frames x 8 streams x 16 heads x 128 x 128 units, bf16: forward 134 us, backward 251 us (0.45 GB moved, 0.15 TFLOP on the matrix cores
// with the parts: a third of the memory's rate, half of the matrix cores').  With neither loads nor stores it takes 190 where it took 239; without the
// state's update 63 less than that (as many vector instructions for V' as matrix instructions), without the state's part of the outputs 46, without the
// scores 25, without their product with V 28: a workgroup's phases follow each other, and what a second one on the compute unit fills in is limited by
// the 384 workgroups there are for 256 compute units.  Half the LDS reads (32 columns to a wavefront), keys a chunk ahead and one barrier fewer changed
// nothing (with scores and state in one part).  fp32: forward 287 us, backward 616 us, 64 GFLOP at 0.74 of the fp32 matrix rate.
// (Figures of one list come from one run; where a call's tensors lie moves them by up to 5 %.)
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
// Infinities and NaN among a lane's numbers.  Set to zero if `clear`; returns whether there are any (all exponent bits set: one more carries into
// the sign's place).
__device__ __forceinline__ bool infinite(float x) { return !(fabsf(x) <= 3.402823466e38f); }
__device__ __forceinline__ bool infinite(bf16x8& x, bool clear) {
    union { bf16x8 v; unsigned u[4]; } w;
    w.v = x;
    unsigned any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned carry = ((w.u[i] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
        any |= carry;
        if (clear) w.u[i] &= ~((carry >> 15) * 0xFFFFu);
    }
    if (clear) x = w.v;
    return any != 0;
}
__device__ __forceinline__ bool infinite(f32x4& x, bool clear) {
    float none = 0.0f;      // times zero: NaN if there is one
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        none = fmaf(x[i], 0.0f, none);
        if (clear && infinite(x[i])) x[i] = 0.0f;
    }
    return none != 0.0f;
}
__device__ __forceinline__ bf16x8 join(s16x4 a, s16x4 b) {
    union { s16x4 h[2]; bf16x8 v; } u;
    u.h[0] = a; u.h[1] = b;
    return u.v;
}
// The upper halves of two numbers (their leading 8 bits, cut off) in one word; the rest stays in them, exactly.  (Cutting off takes five
// instructions for two numbers, rounding to nearest and converting back seven.)
__device__ __forceinline__ unsigned upper(float& x, float& y) {
    const unsigned a = __builtin_bit_cast(unsigned, x), b = __builtin_bit_cast(unsigned, y);
    x -= __builtin_bit_cast(float, a & 0xFFFF0000u);
    y -= __builtin_bit_cast(float, b & 0xFFFF0000u);
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
// Numbers in fp32 as the sum of N in bf16: eight of the 24 bits each, with three of them all.
constexpr int OPERAND_PARTS = 2;
template <int N, class F, class B>
__device__ __forceinline__ void split(F x, B (&part)[N]) {
    constexpr int PAIRS = sizeof(F) / 8;
#pragma unroll
    for (int p = 0; p < N - 1; ++p) {
        union { unsigned u[PAIRS]; B v; } r;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            float a = x[2 * i], b = x[2 * i + 1];
            r.u[i] = upper(a, b);
            x[2 * i] = a; x[2 * i + 1] = b;
        }
        part[p] = r.v;
    }
    part[N - 1] = __builtin_convertvector(x, B);
}

// Frames of a chunk: as many as leave LDS room for two workgroups.  (bf16, 128 units, with 64 / 32: forward 134 / 144, backward 251 / 268, 4,096
// frames of one stream 57 / 62, 16 streams forward 187 / 198 us.)
constexpr int chunk_frames(bool f32, int DK) { return f32 || DK > 128 ? 32 : 64; }

// Place of (frame, unit) of a tile of D units in LDS: the 16-byte pieces of a row are exchanged, so that neither 16 bytes of eight frames
// (operands that run along units) nor four neighbouring pieces of four frames (operands that run along frames) meet in a bank.
template <class T, int D>
__device__ __forceinline__ int place(int row, int col) {
    constexpr int E = 16 / sizeof(T);
    const int f = sizeof(T) == 4 ? row & 15 : D == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
    return row * D + ((col / E ^ f) * E) + col % E;
}

// A tile of C frames x D units, brought from memory to LDS by all THREADS.  Frames beyond the last one read the last again (their scores,
// weights and outputs are left out); what lies behind the units of a row stays zero from the start.
// DIRECT (rows of whole 16-byte pieces, all aligned to them): straight to LDS, 64 lanes x 16 bytes at once in the order of the lanes, a lane
// reading the piece that belongs in its place; s_waitcnt vmcnt(0) and a barrier make them visible.  Otherwise through registers, a row's last
// 16 bytes from where they end, rows of less than 16 bytes number by number.  (128 units, direct / through registers, us: bf16 forward 134 / 178, backward 251 / 392, fp32 backward 616 / 879.)
template <class T, int C, int D, int THREADS, bool DIRECT>
struct Tile {
    static constexpr int E = 16 / sizeof(T), ROW = D / E, ROWS = THREADS / ROW, PIECES = C / ROWS;      // pieces of a row; rows of a piece of all threads
    static_assert(THREADS % ROW == 0 && C % ROWS == 0, "tile");
    const T* base; int64_t step; int dim; bool narrow;
    __device__ __forceinline__ Tile(const AttnTensor& a, int n, int h, int unit, int d, bool reverse, int L, int begin) {
        dim = d - unit;      // units of this tile (may be more than D)
        narrow = d < E;
        step = reverse ? -a.st : a.st;
        base = (const T*)a.p + n * a.sn + (h / a.group) * a.sh + unit + (reverse ? (L - 1) * a.st : 0) + begin * step;
    }
    // the next chunk's first `rows` frames, rows > 0
    __device__ __forceinline__ void load(T* lds, int rows) {
        const int row = threadIdx.x / ROW, slot = threadIdx.x % ROW * E;
        if constexpr (DIRECT) {
            typedef const __attribute__((address_space(1))) void* global_t;
            typedef __attribute__((address_space(3))) void* lds_t;
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
            for (int x = 0; x < PIECES; ++x) {
                const int i = row + x * ROWS, at = place<T, D>(i, slot) - i * D;      // (exchanging twice gives back the piece)
                if (at < dim) __builtin_amdgcn_global_load_lds((global_t)(base + min(i, rows - 1) * step + at), (lds_t)(lds + x * ROWS * D + wave * 64 * E), 16, 0, 0);
            }
        } else if (narrow) {
            if (slot == 0)
                for (int e = 0; e < dim; ++e) {
                    T v[PIECES];
#pragma unroll
                    for (int x = 0; x < PIECES; ++x) v[x] = base[min(row + x * ROWS, rows - 1) * step + e];
#pragma unroll
                    for (int x = 0; x < PIECES; ++x) lds[place<T, D>(row + x * ROWS, e)] = v[x];
                }
        } else {
            u32x4 r[PIECES];
#pragma unroll
            for (int x = 0; x < PIECES; ++x) __builtin_memcpy(&r[x], base + min(row + x * ROWS, rows - 1) * step + min(slot, dim - E), 16);
            const int shift = max(slot + E - dim, 0);      // the row's last units stand at the end of what was read
            typedef std::conditional_t<sizeof(T) == 4, unsigned, unsigned short> word;
#pragma unroll
            for (int x = 0; x < PIECES; ++x) {
                if (shift == 0) *(u32x4*)(lds + place<T, D>(row + x * ROWS, slot)) = r[x];
                else if (slot < dim)
                    for (int e = 0; e < E; ++e) {
                        word v;
                        if constexpr (sizeof(T) == 4) v = r[x][e];
                        else v = (word)(r[x][e / 2] >> (16 * (e % 2)));
                        if (e >= shift) *(word*)(lds + place<T, D>(row + x * ROWS, slot + e - shift)) = v;
                    }
            }
        }
        base += C * step;
    }
};
template <class T>
__device__ __forceinline__ void clear_lds(T* p, int count) {      // a multiple of 16 bytes
    for (int i = threadIdx.x; i < count * (int)sizeof(T) / 16; i += blockDim.x) ((u32x4*)p)[i] = 0u;
}

// Wavefronts of a SIMD that the registers are cut for: as many as LDS has room for, as long as the state fits them.
// (fp32, 128 units: 4 would spill; rows that go through registers need more of them.)
constexpr int chunk_waves(bool f32, int DK, bool direct) { return !direct || DK > 128 || (f32 && DK > 64) ? 2 : 4; }

template <class T, int DK, int W, bool DIRECT, bool STATE>
__global__ void __launch_bounds__(64 * W, (chunk_waves(sizeof(T) == 4, DK, DIRECT))) attention_chunks_kernel(AttnCall c, ChunkOps ops) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int C = chunk_frames(F32, DK), BV = 16 * W, IT = C / 16, AT = DK / 16;
    typedef Tile<T, C, DK, 64 * W, DIRECT> TileK;
    typedef Tile<T, C, BV, 64 * W, DIRECT> TileV;
    __shared__ alignas(256) T lds_q[STATE ? 8 : C * DK];
    constexpr int BUFS = STATE ? 2 : 1;                                               // (the state alone: no room is needed for q and the scores)
    __shared__ alignas(256) T lds_ks[BUFS * C * DK];
    __shared__ alignas(256) T lds_vs[BUFS * C * BV];
    __shared__ alignas(256) T lds_p[STATE ? 8 : F32 ? C * (C + 4) : OPERAND_PARTS * C * C];       // scores [i][j]; bf16: their parts one behind the other
    __shared__ float chunk_decay;
    __shared__ double exact_decay, carry;                                             // g^C; what the roundings of chunk_decay have left so far: the next makes up for it
    __shared__ float power[16 + C + 1], weight[2 * C];                                // g^i from 16 on (what is before it goes to masked scores only); update g^(C - j - early), zeros
    // place of score (i, j); bf16: pieces of 16 bytes exchanged as in the tiles
    auto score_at = [](int i, int j) { return F32 ? i * (C + 4) + j : C == 64 ? i * C + ((j >> 3 ^ (i >> 1 & 7)) << 3) + (j & 7) : i * C + ((j >> 3 ^ (i >> 2 & 3)) << 3) + (j & 7); };

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
    const int my_col = col0 + 16 * wave + m, out_col = col0 + 16 * wave + 4 * g;      // the lane's column; the first of the four it has of an output
    const bool busy = col0 + 16 * wave < a.dv;                                        // of a wavefront; the others help with the tiles and scores

    TileK tq(a.q, n, h, 0, a.dk, a.reverse, L, begin), tk(a.k, n, h, 0, a.dk, a.reverse, L, begin);
    TileV tv(a.v, n, h, col0, a.dv, a.reverse, L, begin);
    if constexpr (!STATE) clear_lds(lds_q, C * DK);
    clear_lds(lds_ks, BUFS * C * DK);
    clear_lds(lds_vs, BUFS * C * BV);
    __syncthreads();
    const T* lds_k = lds_ks;
    const T* lds_v = lds_vs;
    if (begin < end) {
        if constexpr (!STATE) if (a.o.p) tq.load(lds_q, end - begin);                 // (without outputs there may be no q)
        tk.load(lds_ks, end - begin);
        tv.load(lds_vs, end - begin);
    }
    if constexpr (!STATE) clear_lds(lds_p, F32 ? C * (C + 4) : OPERAND_PARTS * C * C);                // (tiles above the diagonal stay zero)
    const float ld = log_decay_of(c, h), both = a.out * a.update;
    if (threadIdx.x <= C + 16) power[threadIdx.x] = threadIdx.x < 16 ? 0.0f : threadIdx.x == 16 ? 1.0f : (float)exp((double)ld * ((int)threadIdx.x - 16));
    if (threadIdx.x == C) { exact_decay = exp((double)ld * C); carry = 1.0; }
    if (threadIdx.x < 2 * C) weight[threadIdx.x] = threadIdx.x < C ? a.update * expf(ld * (C - (int)threadIdx.x - (a.early ? 1 : 0))) : 0.0f;

    // state tile t: rows row_of(t) + r of this lane
    auto row_of = [](int t, int g) { return F32 ? 16 * t + 4 * g : 32 * (t / 2) + 8 * g + 4 * (t % 2); };
    f32x4 S[AT];
    const int64_t nh = (int64_t)n * c.heads + h, heads = (int64_t)c.N * c.heads, size = (int64_t)a.dk * a.dv;
#pragma unroll
    for (int t = 0; t < AT; ++t) S[t] = 0.0f;
    if constexpr (!STATE) {
        // the state before
        const float* from = ops.n_seg > 1 ? ops.seg_state[which] + (seg * heads + nh) * size : a.s_in ? a.s_in + nh * size : nullptr;
        if (from) {
            const int si = ops.n_seg > 1 ? a.dv : (int)a.si, col = min(my_col, a.dv - 1) * (ops.n_seg > 1 ? 1 : (int)a.sj);
            int group = g;
            asm volatile("" : "+v"(group));
            // (loads first, a quarter of them at a time: left to itself the compiler moves each under its condition and waits for it there)
#pragma unroll
            for (int t0 = 0; t0 < AT; t0 += AT / 4) {
#pragma unroll
                for (int t = t0; t < t0 + AT / 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[t][r] = from[min(row_of(t, group) + r, a.dk - 1) * si + col];
#pragma unroll
                for (int t = t0; t < t0 + AT / 4; ++t) asm volatile("" : "+v"(S[t]));
#pragma unroll
                for (int t = t0; t < t0 + AT / 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[t][r] = row_of(t, group) + r < a.dk && my_col < a.dv ? S[t][r] : 0.0f;
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    // operands of 32 units of 16 frames; of 32 frames 32 s + 8 g + e, four columns each
    auto along = [&](const T* tile, int row16, int t) { return *(const bf16x8*)(tile + row16 * 16 * DK + (place<T, DK>(m, 8 * g) ^ (32 * t))); };
    auto along4 = [&](const T* tile, int row16, int t) { return *(const f32x4*)(tile + row16 * 16 * DK + (place<T, DK>(m, 4 * g) ^ (16 * t))); };      // fp32: of 16 units
    auto v_frames = [&](int s) {
        const bf16_t* p = (const bf16_t*)lds_v + 32 * s * BV;
        return join(lds_transposed(p + place<T, BV>(8 * g + m / 4, 16 * wave + 4 * (m % 4))), lds_transposed(p + place<T, BV>(8 * g + 4 + m / 4, 16 * wave + 4 * (m % 4))));
    };
    auto k_frames = [&](int s, int t) {
        const bf16_t* p = (const bf16_t*)lds_k + 32 * s * DK + 4 * (t % 2);
        return join(lds_transposed(p + (place<T, DK>(8 * g + m / 4, 8 * (m % 4)) ^ (32 * (t / 2)))), lds_transposed(p + (place<T, DK>(8 * g + 4 + m / 4, 8 * (m % 4)) ^ (32 * (t / 2)))));
    };
    for (int first = begin; first < end; first += C) {
        const int rows = min(C, end - first);
        f32x4 acc[STATE ? 1 : IT];
        if (threadIdx.x == 0) {
            const double p = exact_decay * carry;
            chunk_decay = (float)p;
            carry = exact_decay > 1e-30 ? p / chunk_decay : 1.0;
        }
        // 1. the state's part of the outputs (q is there; k and v are on their way)
        if constexpr (!STATE) if (a.o.p && busy) {
#pragma unroll
            for (int it = 0; it < IT; ++it) acc[it] = 0.0f;
            if constexpr (F32) {
#pragma unroll
                for (int t = 0; t < AT; ++t) {
                    f32x4 qf[IT];
#pragma unroll
                    for (int it = 0; it < IT; ++it) qf[it] = along4(lds_q, it, t);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int it = 0; it < IT; ++it) acc[it] = __builtin_amdgcn_mfma_f32_16x16x4f32(S[t][r], qf[it][r], acc[it], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int t = 0; t < DK / 32; ++t) {
                    bf16x8 qf[IT];
#pragma unroll
                    for (int it = 0; it < IT; ++it) qf[it] = along(lds_q, it, t);
                    const f32x8 s = __builtin_shufflevector(S[2 * t], S[2 * t + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                    bf16x8 sf[OPERAND_PARTS];
                    split(s, sf);
#pragma unroll
                    for (int u = 0; u < OPERAND_PARTS; ++u)
#pragma unroll
                        for (int it = 0; it < IT; ++it) acc[it] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf[u], qf[it], acc[it], 0, 0, 0);
                }
            }
#pragma unroll
            for (int it = 0; it < IT; ++it) acc[it] *= a.out * power[16 + 16 * it + m + (a.early ? 1 : 0)];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                       // k and v are there
        if constexpr (STATE) {
            const int other = (first - begin) / C & 1 ^ 1;
            lds_k = lds_ks + (other ^ 1) * C * DK;
            lds_v = lds_vs + (other ^ 1) * C * BV;
            if (first + C < end) {
                tk.load(lds_ks + other * C * DK, end - first - C);
                tv.load(lds_vs + other * C * BV, end - first - C);
            }
        }
        // 2. scores of the tiles (it, jt), jt <= it
        if constexpr (!STATE) if (a.o.p) {
#pragma unroll
            for (int x = 0; x < (IT * (IT + 1) / 2 + W - 1) / W; ++x) {
                const int e = wave + W * x, it = e < 1 ? 0 : e < 3 ? 1 : e < 6 ? 2 : 3, jt = e - it * (it + 1) / 2;
                if (e >= IT * (IT + 1) / 2) break;
                f32x4 s = 0.0f;
                if constexpr (F32) {
#pragma unroll
                    for (int t = 0; t < AT; ++t) {
                        const f32x4 kf = along4(lds_k, jt, t), qf = along4(lds_q, it, t);
#pragma unroll
                        for (int r = 0; r < 4; ++r) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[r], qf[r], s, 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < DK / 32; ++t) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(along(lds_k, jt, t), along(lds_q, it, t), s, 0, 0, 0);
                }
                const int lag = 16 * (it - jt) + m - 4 * g;
                const float* f = power + 16 + lag;
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = (lag >= r ? s[r] : 0.0f) * (both * f[-r]);
                T* p = lds_p + score_at(16 * it + m, 16 * jt + 4 * g);
                if constexpr (F32) *(f32x4*)p = s;
                else {
                    bf16x4 part[OPERAND_PARTS];
                    split(s, part);
#pragma unroll
                    for (int u = 0; u < OPERAND_PARTS; ++u) *(bf16x4*)(p + u * C * C) = part[u];
                }
            }
            __syncthreads();                   // the scores are there, q has been read
            if (first + C < end) tq.load(lds_q, end - first - C);
            // 3. the chunk's own part of the outputs.  The products take zero times a later frame's v, which is NaN if that is infinite or NaN: such
            // numbers of v are left out of them and added to the frames that they belong to, one by one.
            if (busy) {
                bool apart = false;
                if constexpr (F32) {
#pragma unroll
                    for (int jt = 0; jt < IT; ++jt) {
                        f32x4 v, pf[IT];
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = lds_v[(16 * jt + r) * BV + (place<T, BV>(4 * g, 16 * wave + m) ^ 4 * r)];
#pragma unroll
                        for (int it = jt; it < IT; ++it) pf[it] = *(const f32x4*)(lds_p + score_at(16 * it + m, 16 * jt + 4 * g));
                        if (__any(infinite(v, false))) { infinite(v, true); apart = true; }
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int it = jt; it < IT; ++it) acc[it] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r], pf[it][r], acc[it], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < C / 32; ++s) {
                        bf16x8 v = v_frames(s);
#pragma unroll
                        for (int u = 0; u < OPERAND_PARTS; ++u) {
                            bf16x8 pf[IT];
#pragma unroll
                            for (int it = 2 * s; it < IT; ++it) pf[it] = *(const bf16x8*)(lds_p + u * C * C + score_at(16 * it + m, 32 * s + 8 * g));
                            if (u == 0 && __any(infinite(v, false))) { infinite(v, true); apart = true; }
#pragma unroll
                            for (int it = 2 * s; it < IT; ++it) acc[it] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[it], acc[it], 0, 0, 0);
                        }
                    }
                }
                if (apart) {
                    int frame = m, column = 16 * wave + 4 * g;
                    asm volatile("" : "+v"(frame), "+v"(column));      // (places are worked out here: kept through the chunks, they would not fit the registers)
#pragma unroll 1
                    for (int j = 0; j < rows; ++j)
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const float x = (float)lds_v[place<T, BV>(j, column + u)];
                            if (!infinite(x)) continue;
#pragma unroll
                            for (int it = 0; it < IT; ++it) {
                                const T* p = lds_p + score_at(16 * it + frame, j);
                                float score = (float)p[0];
                                if constexpr (!F32)
#pragma unroll
                                    for (int y = 1; y < OPERAND_PARTS; ++y) score += (float)p[y * C * C];
                                if (j <= 16 * it + frame) acc[it][u] = fmaf(score, x, acc[it][u]);
                            }
                        }
                }
                const int64_t step = a.reverse ? -a.o.st : a.o.st;
                const int64_t at = (int64_t)(a.reverse ? L - 1 - first - m : first + m) * a.o.st + n * a.o.sn + h * a.o.sh + out_col;
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    if (16 * it + m >= rows || out_col >= a.dv) continue;
                    typedef T out_t __attribute__((ext_vector_type(4)));
                    const out_t y = __builtin_convertvector(acc[it], out_t);
                    float* of = (float*)a.o.p + at + 16 * it * step;
                    T* ot = (T*)a.o.p + at + 16 * it * step;
                    if (DIRECT || out_col + 4 <= a.dv) {
                        if (a.o_f32) __builtin_memcpy(of, &acc[it], sizeof(acc[it]));
                        else __builtin_memcpy(ot, &y, sizeof(y));
                    } else {
#pragma unroll
                        for (int u = 0; u < 3; ++u)
                            if (out_col + u < a.dv) { if (a.o_f32) of[u] = acc[it][u]; else ot[u] = y[u]; }
                    }
                }
            }
        }
        // 4. the state after the chunk
        const float decay = rows == C ? chunk_decay : power[16 + rows];
        const float* wt = weight + C - rows;
        if (busy) {
#pragma unroll
            for (int t = 0; t < AT; ++t) S[t] *= decay;
            if constexpr (F32) {
                int at = place<T, DK>(4 * g, m);       // of frame 4 g, unit m; the others' places differ from it in constant bits of the piece
                asm volatile("" : "+v"(at));           // (worked out in every chunk: kept, they would not fit the registers)
#pragma unroll
                for (int jt = 0; jt < IT; ++jt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = 16 * jt + 4 * g + r;
                        const float v = lds_v[(16 * jt + r) * BV + (place<T, BV>(4 * g, 16 * wave + m) ^ 4 * r)] * wt[j];
#pragma unroll
                        for (int t = 0; t < AT; ++t) S[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(lds_k[(16 * jt + r) * DK + (at ^ (4 * t ^ r) * 4)], v, S[t], 0, 0, 0);
                    }
            } else {
#pragma unroll
                for (int s = 0; s < C / 32; ++s) {
                    f32x8 x = __builtin_convertvector(v_frames(s), f32x8);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= wt[32 * s + 8 * g + e];
                    bf16x8 v[3];
                    split(x, v);
#pragma unroll
                    for (int t = 0; t < AT; t += 2) {
                        const bf16x8 k[2] = {k_frames(s, t), k_frames(s, t + 1)};
#pragma unroll
                        for (int p = 0; p < 3; ++p)
#pragma unroll
                            for (int u = 0; u < 2; ++u) S[t + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[u], v[p], S[t + u], 0, 0, 0);
                    }
                }
            }
        }
        if constexpr (!STATE) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                       // the next q is there; k, v and the scores have been read
        if constexpr (!STATE)
            if (first + C < end) {
                tk.load(lds_ks, end - first - C);
                tv.load(lds_vs, end - first - C);
            }
    }
    float* to = STATE ? ops.seg_state[which] + (seg * heads + nh) * size : a.s_out && end == L ? a.s_out + nh * size : nullptr;
    if (!to || my_col >= a.dv) return;
    const int si = STATE ? a.dv : (int)a.si, sj = (STATE ? 1 : (int)a.sj) * my_col;
    int group = g;
    asm volatile("" : "+v"(group));            // (the rows' addresses are worked out here again, not kept through the loop)
#pragma unroll
    for (int t = 0; t < AT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = row_of(t, group) + r;
            if (i < a.dk) to[i * si + sj] = S[t][r];
        }
}

// What the segments add to the state becomes the state before each, in place; U segments are read ahead.
template <int U>
__global__ void __launch_bounds__(256) attention_segments_kernel(AttnCall c, ChunkOps ops) {
    const AttnOp& a = ops.op[blockIdx.z];
    const int64_t size = (int64_t)a.dk * a.dv, heads = (int64_t)c.N * c.heads, nh = blockIdx.y;
    const int x = blockIdx.x * 256 + threadIdx.x;
    if (x >= size) return;
    const int L = length_of(c, (int)(nh / c.heads));
    const double ld = log_decay_of(c, (int)(nh % c.heads));
    const int used = max(1, (L + ops.seg_len - 1) / ops.seg_len);      // segments that hold frames; all but the last of them are whole
    double S = a.s_in ? a.s_in[nh * size + x / a.dv * a.si + x % a.dv * a.sj] : 0.0;
    const double whole = exp(ld * ops.seg_len);
    float* p = ops.seg_state[blockIdx.z] + nh * size + x;
    for (int first = 0; first < used; first += U) {
        float add[U];
#pragma unroll
        for (int u = 0; u < U; ++u) add[u] = p[min(first + u, ops.n_seg - 2) * heads * size];      // (behind the last: any)
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u < used) {
                p[(first + u) * heads * size] = (float)S;
                S = S * whole + add[u];
            }
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
    bool wide = true;
    for (int i = 0; i < n_ops; ++i) {
        const AttnOp& a = so.op[i] = ops[i];
        dk = std::max(dk, a.dk); dv = std::max(dv, a.dv);
        wide = wide && a.sj == 1 && a.dv % 4 == 0 && ((reinterpret_cast<uintptr_t>(a.s_in) | reinterpret_cast<uintptr_t>(a.s_out)) & 15) == 0;
    }
    const int slices = (dv + 63) / 64;
    const dim3 grid((unsigned)c.N * c.heads * slices, (unsigned)n_ops);
    auto start = [&](auto* t, auto rows) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int NR = decltype(rows)::value;
        auto* kernel = wide ? attention_steps_kernel<T, NR, true> : attention_steps_kernel<T, NR, false>;
        kernel<<<grid, 256, 0, s>>>(c, so, slices);
        return hipGetLastError();
    };
    auto go = [&](auto* t) {
        if (dk <= 64) return start(t, std::integral_constant<int, 4>());
        if (dk <= 128) return start(t, std::integral_constant<int, 8>());
        return start(t, std::integral_constant<int, 16>());
    };
    return c.dtype == DT_F32 ? go((float*)nullptr) : go((bf16_t*)nullptr);
}

// Segments of the frames, so that the chip is filled (two workgroups to a compute unit) where streams and heads are few: each adds its frames up to a
// state of its own, a scan makes these the states in front of the segments, and the outputs of all are worked out at once.  That reads k and v twice.
// Whole / in segments, us, heads of 128 x 128 in bf16: 4,096 frames, 16 heads 294 / 57; 65,536 frames, 8 heads 4536 / 209; 2,048 frames x 8 streams x 16
// heads forward (128 workgroups) 157 / 134; backward (384) 251 / 314: from 256 on they stay whole.  For 256, 512, 1,024 workgroups: 57, 57, 57; 245, 209, 226;
// 143, 134, 165.  Segments of at least 2, 4, 8 chunks: 62, 57, 76 (4,096 frames).
static int64_t most_segments(int T, int64_t works, int C) {      // (grows with T: room for a window's is room for a part's)
    const int64_t chunks = (T + C - 1) / C;
    return std::max<int64_t>(1, works >= 256 || works == 0 ? 1 : std::min<int64_t>((512 + works - 1) / works, chunks / 4));
}
static void plan_segments(int T, int64_t works, int C, int& n_seg, int& seg_len) {
    const int64_t chunks = (T + C - 1) / C, n = most_segments(T, works, C);
    const int64_t per = (chunks + n - 1) / n;
    seg_len = (int)(per * C);
    n_seg = std::max<int>(1, (int)((chunks + per - 1) / per));
}
namespace {
struct ChunkShape { int DK, W, C, slices; };
ChunkShape chunk_shape(int dtype, int dk, int dv) {
    ChunkShape s;
    s.DK = dk <= 64 ? 64 : dk <= 128 ? 128 : 256;
    // Columns of a workgroup: 64, or 128 (half as many reads of q and k, scores worked out once; fewer workgroups on a compute unit, which hide each
    // other's waits less).  128 / 64 columns, us, 2,048 frames x 8 streams x 16 heads, forward and backward: bf16 128 x 128 units 133 / 130, 244 / 293,
    // 256 x 256 287 / 288, 771 / 718; fp32 64 x 128 185 / 194, 688 / 607 (4,096 frames, one stream 256 / 291), 128 x 128 332 / 287, 828 / 615,
    // 128 x 256 414 / 444, 2221 / 2340, 256 x 256 758 / 800, 2246 / 2358.
    const bool half = dv <= 64 || (dtype == DT_F32 ? s.DK == 128 && dv <= 128 : s.DK == 256);
    s.W = half ? 4 : 8;
    s.C = chunk_frames(dtype == DT_F32, s.DK);
    s.slices = (dv + 16 * s.W - 1) / (16 * s.W);
    return s;
}
}  // namespace

// Few frames go one after another.
static bool by_frames(const AttnCall& c, const AttnOp& a) {
    const bool narrow = std::min(a.dk, a.dv) * (c.dtype == DT_F32 ? 4 : 2) < 16;
    return c.T <= (narrow ? ATTN_STEPS_NARROW : ATTN_STEPS);
}

int64_t attention_space(const AttnCall& c, const AttnOp* ops, int n_ops) {
    if (n_ops == 0 || by_frames(c, ops[0])) return 0;
    int dk = 0, dv = 0;
    int64_t floats = 0;
    for (int i = 0; i < n_ops; ++i) { dk = std::max(dk, ops[i].dk); dv = std::max(dv, ops[i].dv); floats += ((int64_t)ops[i].dk * ops[i].dv * c.N * c.heads + 63) / 64 * 64; }
    const ChunkShape sh = chunk_shape(c.dtype, dk, dv);
    const int64_t n_seg = most_segments(c.T, (int64_t)c.N * c.heads * n_ops * sh.slices, sh.C);
    return n_seg > 1 ? n_seg * floats * 4 : 0;
}

hipError_t launch_attention(const AttnCall& c, const AttnOp* ops, int n_ops, float* space, hipStream_t s) {
    if (by_frames(c, ops[0])) return launch_attention_steps(c, ops, n_ops, s);
    ChunkOps co = {};
    int dk = 0, dv = 0;
    const int E = c.dtype == DT_F32 ? 4 : 8;      // units of 16 bytes
    bool direct = true;
    for (int i = 0; i < n_ops; ++i) {
        const AttnOp& a = co.op[i] = ops[i];
        dk = std::max(dk, a.dk); dv = std::max(dv, a.dv);
        direct = direct && a.dk % E == 0 && a.dv % E == 0;
        for (const AttnTensor* x : {&a.q, &a.k, &a.v})
            direct = direct && reinterpret_cast<uintptr_t>(x->p) % 16 == 0 && x->st % E == 0 && x->sn % E == 0 && x->sh % E == 0;
    }
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
        kernel<<<(co.works + 7) / 8 * 8, 64 * sh.W, 0, s>>>(c, co);
        return hipGetLastError();
    };
    auto start = [&](auto* t, auto DKc, auto Wc, auto directc) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int DK = decltype(DKc)::value, W = decltype(Wc)::value;
        constexpr bool DIRECT = decltype(directc)::value;
        if (co.n_seg > 1) {
            hipError_t e = launch(attention_chunks_kernel<T, DK, W, DIRECT, true>, co.n_seg - 1);
            if (e != hipSuccess) return e;
            auto* join = co.n_seg <= 4 ? attention_segments_kernel<4> : attention_segments_kernel<8>;
            join<<<dim3((unsigned)((dk * dv + 255) / 256), (unsigned)(c.N * c.heads), (unsigned)n_ops), 256, 0, s>>>(c, co);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        return launch(attention_chunks_kernel<T, DK, W, DIRECT, false>, co.n_seg);
    };
    auto by_slice = [&](auto* t, auto DKc) {
        const std::integral_constant<int, 4> four;
        const std::integral_constant<int, 8> eight;
        if (sh.W == 4) return direct ? start(t, DKc, four, std::true_type()) : start(t, DKc, four, std::false_type());
        return direct ? start(t, DKc, eight, std::true_type()) : start(t, DKc, eight, std::false_type());
    };
    auto by_width = [&](auto* t) {
        if (sh.DK == 64) return by_slice(t, std::integral_constant<int, 64>());
        if (sh.DK == 128) return by_slice(t, std::integral_constant<int, 128>());
        return by_slice(t, std::integral_constant<int, 256>());
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
