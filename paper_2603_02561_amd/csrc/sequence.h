// Kernels' parameters and host-side launchers of the sequence operators (internal to the library): rotary positions,
// linear attention with a decay, layer norm.
#pragma once

#include "common.h"

namespace solar {

// Elements between users, rows and heads.
struct Strides {
    int64_t batch, row, head;
};

// One tensor of heads: head h of the operator reads (or writes) head h / share of it.
struct Heads {
    char* data;
    Strides s;      // in bytes
    int share;
};

__device__ __forceinline__ char* row_of(const Heads& t, int b, int64_t n, int h) {
    return t.data + b * t.s.batch + n * t.s.row + (int64_t)(h / t.share) * t.s.head;
}

// What a state keeps over n rows, g^n x.  Near 1 that is x + (g^n - 1) x, or the error of a rounded g^n would add up over thousands of
// steps; below a half g^n - 1 has lost bits that count, and it is g^n x: what is left of a large first state may be all there is.
struct Kept {
    float by;
    bool near;      // by is g^n - 1, else g^n
};
__device__ __forceinline__ Kept kept(float log_g, int n) {
    const float x = log_g * (float)n, m = expm1f(x);
    return {m < -0.5f ? expf(x) : m, !(m < -0.5f)};
}
__device__ __forceinline__ float keep(float x, Kept k) { return fmaf(x, k.by, k.near ? x : 0.f); }

// One walk over the rows of every user and head with a state S [D,D]:
//   forward   S = g S + k_t v_t^T,  o_t = o_scale S^T q_t          rows 0 .. len - 1
//   reverse   S += k_t v_t^T,  o_t = o_scale S^T q_t,  S = g S     rows len - 1 .. 0
// with kv_scale on every k_t v_t^T.  The gradients of the operator are walks with the tensors in other roles.
struct Walk {
    Heads q, k, v, o;               // o.data may be null: the last state alone
    const int32_t* lengths;
    const float* log_decay;         // [H]
    const float* state_in;          // [B,H,D,D], null: zeros
    float* state_out;               // [B,H,D,D] or null
    int B, N, H, D;
    float o_scale, kv_scale;
    bool reverse, in_turned;        // in_turned: state_in is read transposed
    bool bf16, o_float;             // o_float: o is float whatever the inputs are
    // the sequence is cut into nparts parts of part_rows rows, and each part into `pieces` pieces of a multiple of 64; parts and
    // part_moments are [B,H,nparts * pieces,D,D] work arrays, not used where nparts is 1
    int nparts, part_rows, pieces;
    float *parts, *part_moments;
    bool parts_turned;              // parts hold the states of this walk transposed
    // moment: also the derivative of o by log g, summed against `grad`, and that of the last state against `grad_state` (or null;
    // read transposed with in_turned)
    bool moment;
    Heads grad;
    const float* grad_state;
    double* moments;                // [B][H][nparts][moment_slices(D)] partial sums
};

// Walks that run side by side: users, rows, heads, types and parts are the same, and the states of the first (in `parts`) are
// those of all.
struct Walks {
    Walk walk[2];
    int count;
};

// decay.hip
// A forward walk row by row, for a few rows (N <= kDecayRows); nparts is not looked at.  Every row costs it a sum across the
// workgroup, the chunked form takes up to 32 or 64 rows at the price of one.  Six rows of 1024 states take 14.4 against 17.4 us at
// D = 64, 36.9 against 39.2 at 128, 116 against 140 at 256, eight rows 17.5 against 17.4, 42.2 against 39.4, 130 against 141; of four states
// 7.4 against 7.5 at D = 64 and 7.8 against 11.6 at 128, eight rows 8.9 against 7.5 and 9.5 against 11.6 (bf16).
constexpr int kDecayRows = 6;
hipError_t launch_decay_rows(const Walk& w, hipStream_t stream);
// dlog[h] = the sum of moments [B][H][slices] over users and slices
hipError_t launch_moment_sum(const double* moments, int B, int H, int slices, float* dlog, hipStream_t stream);
// out [.., Hkv, D] = the sum of in [B,N,H,D] over the H / Hkv heads that share one
hipError_t launch_share_sum(const float* in, int B, int N, int H, int Hkv, int D, const Heads& out, bool bf16,
                            hipStream_t stream);

// decay_chunk.hip
struct DecayParts {
    int parts, rows, pieces;
};
DecayParts decay_parts(int B, int N, int H, int D, int walks);
int moment_slices(int D);
hipError_t launch_decay_chunks(const Walks& ws, hipStream_t stream);

// rotary.hip
struct Rotary {
    Heads in[2], out[2];            // queries and keys; heads[1] = 0: queries alone
    int heads[2];
    const int32_t *lengths, *positions;
    const double* freq;             // [rot / 2] radians per position
    int B, N, D, rot;
    bool interleaved, inverse, bf16;
    float amplitude;
};
constexpr int kRotaryRows = 4;      // of a workgroup: 256 angles at 128 rotated columns, one a thread
hipError_t launch_rotary(const Rotary& r, hipStream_t stream);

// norm.hip
constexpr int kNormMaxD = 16384;
size_t norm_partial_floats(int rows, int groups, int d);
hipError_t launch_layer_norm(const void* in, const float* weight, const float* bias, int rows, int groups, int d,
                             float eps, bool in_bf16, bool out_bf16, void* out, float* mean, float* rstd,
                             hipStream_t stream);
hipError_t launch_layer_norm_backward(const void* in, const float* weight, const float* mean, const float* rstd,
                                      const void* dout, int rows, int groups, int d, bool in_bf16, bool dout_bf16,
                                      void* din, float* dweight, float* dbias, float* partials, hipStream_t stream);

}  // namespace solar
