// Launch wrappers of the layers that need no step loop (rows.hip, attention.hip), and the error text that
// the C entry points share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

namespace rnng {

int set_error(int code, const std::string& msg);      // rnn_last_error's message on this thread; returns code
int set_hip_error(hipError_t e, const char* what);

enum { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };         // = enum rnn_dtype

// Rows of `dim` units of one type; ld: elements from a row to the next one.
struct RowTensor { void* p; int64_t ld; };

// Dropout of a call: an element is kept if its 16-bit number is at least `cut` (0: no dropout).
struct DropoutArgs { unsigned cut; float factor; uint64_t seed, offset; const uint64_t* d_offset; };
inline unsigned dropout_cut(double p) { return (unsigned)(p * 65536.0 + 0.5); }
inline DropoutArgs dropout_args(double p, uint64_t seed, uint64_t offset, const uint64_t* d_offset) {
    const unsigned cut = dropout_cut(p);
    return DropoutArgs{cut, cut < 65536 ? (float)(65536.0 / (65536 - cut)) : 0.0f, seed, offset, d_offset};
}

constexpr int NORM_MAX_DIM = 16384;
struct AddNormArgs {
    int64_t rows; int dim; float eps; DropoutArgs drop;
    RowTensor x, residual, h, y;                      // residual, h: p may be NULL
    const float* gain; float* rstd;
    float* scales; int group;                         // y in e4m3 with scales if scales != NULL
};
hipError_t launch_add_norm(int dtype, const AddNormArgs& a, hipStream_t s);
struct AddNormGradArgs {
    int64_t rows; int dim; DropoutArgs drop;
    RowTensor dy, dh, h, dx, dresidual;               // dh, dx, dresidual: p may be NULL
    const float* gain; const float* rstd; float* dgain; float* partial;
    int blocks;                                       // norm_grad_blocks: rows of `partial`
};
int norm_grad_blocks(int64_t rows, int dim);
hipError_t launch_add_norm_grad(int dtype, const AddNormGradArgs& a, hipStream_t s);
// The generator's number of row 0 is first_row + *d_first_row (NULL: 0).
struct DropoutRowsArgs { int64_t rows; int dim; DropoutArgs drop; RowTensor x, y; int64_t first_row; const int64_t* d_first_row; };
hipError_t launch_dropout(int dtype, const DropoutRowsArgs& a, hipStream_t s);
hipError_t launch_count(int64_t* p, int64_t add, bool fresh, hipStream_t s);      // *p = (fresh ? 0 : *p) + add

// ---- linear attention with a decay for each head --------------------------------------------
// One operator serves the forward pass and all of its gradients.  For stream n, head h and its L frames, with g = exp(log_decay[h]):
//     for i = 0 .. L - 1, frame t = i, or L - 1 - i if reverse:
//         early:  S <- g S
//         S <- S + update k(t) v(t)^T          o(t) = out S^T q(t)
//         else:   S <- g S
//   forward    q, k, v                     early, update 1, out scale             S: the state
//   dq         q := do, k := v, v := k     early, update 1, out scale             S: the state, transposed
//   dv         q := k,  k := q, v := do    reverse, update scale, out 1           S: dE/dS of the state after the frame
//   dk         q := v,  k := do, v := q    reverse, update scale, out 1           S: the same, transposed
struct AttnTensor { const void* p; int64_t st, sn, sh; int group; };      // head h of the operator reads head h / group
struct AttnOut { void* p; int64_t st, sn, sh; };
struct AttnOp {
    AttnTensor q, k, v;
    AttnOut o; bool o_f32;                            // p may be NULL; o_f32: stored in fp32 whatever the inputs' type
    const float* s_in; float* s_out;                  // element (i, j) of head (n, h) at (n * heads + h) * dk * dv + i * si + j * sj; either may be NULL
    int64_t si, sj;
    int dk, dv;                                       // units of q and k, of v and o
    float update, out;
    bool early, reverse;
};
struct AttnCall { int T, N, heads, dtype; const float* log_decay; const int32_t* lengths; };
constexpr int ATTN_MAX_DIM = 256;
// Windows of at most so many frames go frame by frame, longer ones in chunks.  Frame by frame / in chunks, us for T = 2, 4, 8 (in a graph):
// 64 streams x 16 heads x 128 x 128, bf16: 29 / 36, 37 / 35, 51 / 36;  64 x 64, bf16: 9.5 / 17.5, 12.5 / 17.7, 18.1 / 17.8;
// 64 x 8 heads x 128 x 128, fp32: 20 / 31, 25 / 31, 38 / 31;  one stream, 16 heads x 128 x 128, bf16: 6.7 / 10.4, 9.7 / 10.4, 16.0 / 10.4;
// backward, 16 x 16 heads x 128 x 128, bf16: 33 / 38, 41 / 38, 55 / 39.
constexpr int ATTN_STEPS = 4;
// Heads of less than 16 bytes (their tiles are loaded number by number), T = 6, 8, 16, 1,024: 64 streams x 16 heads x 4 x 4, bf16: 13.3 / 17.1, 16.2 / 17.0,
// 27 / 17.0, 1,352 / 143;  one stream: 9.1 / 9.2, 11.1 / 9.2, 19.3 / 9.2, 1,024 / 34;  64 x 16 heads x 3 x 3, fp32: 13.3 / 16.5, 15.9 / 16.5, 26 / 16.6, 1,257 / 287.
constexpr int ATTN_STEPS_NARROW = 8;
// Up to three operators side by side.  space: attention_space bytes.
int64_t attention_space(const AttnCall& c, const AttnOp* ops, int n_ops);
hipError_t launch_attention(const AttnCall& c, const AttnOp* ops, int n_ops, float* space, hipStream_t s);
// out (T, N, heads / group, d), of the inputs' type, = sum of `part` [T][N][heads][d] over the heads of a group.
hipError_t launch_attention_sum_heads(const AttnCall& c, const float* part, const AttnOut& out, int d, int group, hipStream_t s);

}  // namespace rnng
