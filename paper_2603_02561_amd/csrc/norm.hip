// Layer norm over groups of columns and its gradient.  A row of d elements:
//   y = (x - mu) rstd w + b,  rstd = 1 / sqrt(mean((x - mu)^2) + eps)
//   dx = rstd (a - mean(a) - xh mean(a xh)),  a = dy w,  xh = (x - mu) rstd;   dw = sum dy xh,  db = sum dy
//
// Bound by memory: x is read once and y written once; the gradient reads x and dy once and writes dx once.  A row stays
// in registers, so mean and variance are taken one after the other from the same values (no difference of two large
// sums).  Between 8 and 256 threads share a row, by its width; each such team walks over rows a whole number of groups
// apart, so that its weights, and its sums for dw and db, stay in registers.  The teams' sums go to the workspace and are
// added by a second kernel in a fixed order.
#include "sequence.h"

namespace solar {

namespace {

constexpr int kThreads = 256;

template <bool BF16>
struct Elem {
    using type = float;
};
template <>
struct Elem<true> {
    using type = __bf16;
};

// Columns of vector v, element e of thread t in a team of T: eight in a row where rows start on a vector (VEC), else
// neighbouring threads take neighbouring columns.
template <int T, bool VEC>
__device__ __forceinline__ int column(int t, int v, int e) {
    return VEC ? (v * T + t) * 8 + e : (v * 8 + e) * T + t;
}

// A team's part of one row; what lies past d is zero.
template <int T, int NV, bool VEC, bool BF16>
__device__ __forceinline__ void load_row(const void* base, size_t at, int d, int t, float (&x)[NV][8]) {
    using E = typename Elem<BF16>::type;
    const E* p = reinterpret_cast<const E*>(base) + at;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if constexpr (VEC) {
            const int c = column<T, VEC>(t, v, 0);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = 0.f;
            if (c < d) {
                if constexpr (BF16) {
                    const v4u u = *reinterpret_cast<const v4u*>(p + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[v][2 * e] = bf16_lo(u[e]);
                        x[v][2 * e + 1] = bf16_hi(u[e]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const v4f u = reinterpret_cast<const v4f*>(p + c)[j];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[v][4 * j + e] = u[e];
                    }
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = column<T, VEC>(t, v, e);
                x[v][e] = c < d ? (float)p[c] : 0.f;
            }
        }
    }
}

template <int T, int NV, bool VEC, bool BF16>
__device__ __forceinline__ void store_row(void* base, size_t at, int d, int t, const float (&x)[NV][8]) {
    using E = typename Elem<BF16>::type;
    E* p = reinterpret_cast<E*>(base) + at;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if constexpr (VEC) {
            const int c = column<T, VEC>(t, v, 0);
            if (c < d) {
                if constexpr (BF16) {
                    v8bf u;
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[e] = (__bf16)x[v][e];
                    *reinterpret_cast<v8bf*>(p + c) = u;
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        v4f u = {x[v][4 * j], x[v][4 * j + 1], x[v][4 * j + 2], x[v][4 * j + 3]};
                        reinterpret_cast<v4f*>(p + c)[j] = u;
                    }
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = column<T, VEC>(t, v, e);
                if (c < d) p[c] = (E)x[v][e];
            }
        }
    }
}

// Sums of K values over a team, in every thread of it.  `turn` alternates between the two halves of `part`, so that one
// barrier a call is enough.
template <int T, int K>
__device__ __forceinline__ void team_sum(float (&s)[K], float (*part)[4][K], int& turn) {
#pragma unroll
    for (int m = 1; m < (T < 64 ? T : 64); m <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] += __shfl_xor(s[k], m);
    if constexpr (T > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) part[turn][wave][k] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = part[turn][0][k] + part[turn][1][k] + part[turn][2][k] + part[turn][3][k];
        turn ^= 1;
    }
}

// `teams` teams, a multiple of `groups`, walk over `rows` rows of d elements (groups counted as rows).
template <int T, int NV, bool VEC, bool IN_BF16, bool OUT_BF16>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(const void* in, const float* __restrict__ weight,
                                                              const float* __restrict__ bias, size_t rows, int groups,
                                                              int teams, int d, float eps, void* out, float* mean,
                                                              float* rstd) {
    __shared__ float part[2][4][1];
    int turn = 0;
    const int t = threadIdx.x % T, team = blockIdx.x * (kThreads / T) + threadIdx.x / T;
    if (team >= teams) return;      // whole workgroups where a team is one
    const int group = team % groups;
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column<T, VEC>(t, v, e);
            w[v][e] = weight && c < d ? weight[(size_t)group * d + c] : 1.f;
            b[v][e] = bias && c < d ? bias[(size_t)group * d + c] : 0.f;
        }
    const float inv = 1.f / (float)d;
    for (size_t row = team; row < rows; row += teams) {
        float x[NV][8];
        load_row<T, NV, VEC, IN_BF16>(in, row * d, d, t, x);
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += x[v][e];
        team_sum<T, 1>(s, part, turn);
        const float mu = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[v][e] = column<T, VEC>(t, v, e) < d ? x[v][e] - mu : 0.f;
                s[0] = fmaf(x[v][e], x[v][e], s[0]);
            }
        team_sum<T, 1>(s, part, turn);
        const float rs = 1.f / sqrtf(s[0] * inv + eps);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = fmaf(x[v][e] * rs, w[v][e], b[v][e]);
        store_row<T, NV, VEC, OUT_BF16>(out, row * d, d, t, x);
        if (t == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = rs;
        }
    }
}

// partials [2][teams][d]: sums of dy xh and of dy of each team; null where neither is wanted
template <int T, int NV, bool VEC, bool IN_BF16, bool DOUT_BF16>
__global__ __launch_bounds__(kThreads) void layer_norm_backward_kernel(
    const void* in, const float* __restrict__ weight, const float* __restrict__ mean, const float* __restrict__ rstd,
    const void* dout, size_t rows, int groups, int teams, int d, void* din, float* partials) {
    __shared__ float part[2][4][2];
    int turn = 0;
    const int t = threadIdx.x % T, team = blockIdx.x * (kThreads / T) + threadIdx.x / T;
    if (team >= teams) return;
    const int group = team % groups;
    float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column<T, VEC>(t, v, e);
            w[v][e] = weight && c < d ? weight[(size_t)group * d + c] : 1.f;
            dw[v][e] = db[v][e] = 0.f;
        }
    const float inv = 1.f / (float)d;
    for (size_t row = team; row < rows; row += teams) {
        float x[NV][8], dy[NV][8];
        load_row<T, NV, VEC, IN_BF16>(in, row * d, d, t, x);
        load_row<T, NV, VEC, DOUT_BF16>(dout, row * d, d, t, dy);
        const float mu = mean[row], rs = rstd[row];
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // past d dy is zero, and a zero takes the place of what x would give there
                x[v][e] = column<T, VEC>(t, v, e) < d ? (x[v][e] - mu) * rs : 0.f;
                const float a = dy[v][e] * w[v][e];
                s[0] += a;
                s[1] = fmaf(a, x[v][e], s[1]);
                dw[v][e] = fmaf(dy[v][e], x[v][e], dw[v][e]);
                db[v][e] += dy[v][e];
            }
        team_sum<T, 2>(s, part, turn);
        const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = rs * (fmaf(dy[v][e], w[v][e], -m0) - x[v][e] * m1);
        store_row<T, NV, VEC, IN_BF16>(din, row * d, d, t, x);
    }
    if (partials) {
        store_row<T, NV, VEC, false>(partials, (size_t)team * d, d, t, dw);
        store_row<T, NV, VEC, false>(partials, ((size_t)teams + team) * d, d, t, db);
    }
}

// dweight and dbias [width] from [2][n][width]: 64 columns a workgroup, 16 of its threads down each
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* __restrict__ partials, int n, int width, float* dweight,
                                                        float* dbias) {
    __shared__ float sum[16][64];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6, c = blockIdx.x * 64 + x;
    float* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const float* p = partials + (size_t)blockIdx.y * n * width;
    float s = 0.f;
    if (c < width)
        for (int i = y; i < n; i += 16) s += p[(size_t)i * width + c];
    sum[y][x] = s;
    __syncthreads();
    if (y == 0 && c < width) {
        for (int i = 1; i < 16; ++i) s += sum[i][x];
        out[c] = s;
    }
}

// Threads a row, and vectors a thread: a row of up to 512 elements stays in a wave at one vector a thread.
struct Team {
    int threads, vectors;
};

Team team_for(int d) {
    if (d <= 64) return {8, 1};
    if (d <= 128) return {16, 1};
    if (d <= 256) return {32, 1};
    if (d <= 512) return {64, 1};
    if (d <= 1024) return {64, 2};
    if (d <= 2048) return {256, 1};
    if (d <= 4096) return {256, 2};
    if (d <= 8192) return {256, 4};
    return {256, 8};
}

// Teams: four workgroups for each compute unit, whole groups, no team without a row.
int teams_for(int rows, int groups, int d) {
    const int per_block = kThreads / team_for(d).threads;
    const size_t all = (size_t)rows * groups, want = (size_t)1024 * per_block;
    const size_t teams = (want + groups - 1) / groups * groups;
    return (int)(teams < all ? teams : all);
}

}  // namespace

size_t norm_partial_floats(int rows, int groups, int d) { return (size_t)2 * teams_for(rows, groups, d) * d; }

#define SOLAR_NORM_SHAPES(CALL)                                  \
    switch (tm.threads * 16 + tm.vectors) {                      \
        case 8 * 16 + 1: CALL(8, 1); break;                      \
        case 16 * 16 + 1: CALL(16, 1); break;                    \
        case 32 * 16 + 1: CALL(32, 1); break;                    \
        case 64 * 16 + 1: CALL(64, 1); break;                    \
        case 64 * 16 + 2: CALL(64, 2); break;                    \
        case 256 * 16 + 1: CALL(256, 1); break;                  \
        case 256 * 16 + 2: CALL(256, 2); break;                  \
        case 256 * 16 + 4: CALL(256, 4); break;                  \
        case 256 * 16 + 8: CALL(256, 8); break;                  \
        default: return hipErrorInvalidValue;                    \
    }

namespace {

template <bool VEC, bool A, bool B>
hipError_t forward(const void* in, const float* weight, const float* bias, int rows, int groups, int d, float eps,
                   void* out, float* mean, float* rstd, hipStream_t stream) {
    const Team tm = team_for(d);
    const int teams = teams_for(rows, groups, d);
    const dim3 grid(ceil_div(teams, kThreads / tm.threads)), block(kThreads);
#define SOLAR_CALL(T, NV)                                                                                        \
    hipLaunchKernelGGL((layer_norm_kernel<T, NV, VEC, A, B>), grid, block, 0, stream, in, weight, bias,          \
                       (size_t)rows * groups, groups, teams, d, eps, out, mean, rstd)
    SOLAR_NORM_SHAPES(SOLAR_CALL)
#undef SOLAR_CALL
    return hipGetLastError();
}

template <bool VEC, bool A, bool B>
hipError_t backward(const void* in, const float* weight, const float* mean, const float* rstd, const void* dout, int rows,
                    int groups, int d, void* din, float* partials, hipStream_t stream) {
    const Team tm = team_for(d);
    const int teams = teams_for(rows, groups, d);
    const dim3 grid(ceil_div(teams, kThreads / tm.threads)), block(kThreads);
#define SOLAR_CALL(T, NV)                                                                                          \
    hipLaunchKernelGGL((layer_norm_backward_kernel<T, NV, VEC, A, B>), grid, block, 0, stream, in, weight, mean, rstd, \
                       dout, (size_t)rows * groups, groups, teams, d, din, partials)
    SOLAR_NORM_SHAPES(SOLAR_CALL)
#undef SOLAR_CALL
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(const void* in, const float* weight, const float* bias, int rows, int groups, int d,
                             float eps, bool in_bf16, bool out_bf16, void* out, float* mean, float* rstd,
                             hipStream_t stream) {
#define SOLAR_NORM(V)                                                                                                 \
    (in_bf16 ? (out_bf16 ? forward<V, true, true>(in, weight, bias, rows, groups, d, eps, out, mean, rstd, stream)    \
                         : forward<V, true, false>(in, weight, bias, rows, groups, d, eps, out, mean, rstd, stream))  \
             : (out_bf16 ? forward<V, false, true>(in, weight, bias, rows, groups, d, eps, out, mean, rstd, stream)   \
                         : forward<V, false, false>(in, weight, bias, rows, groups, d, eps, out, mean, rstd, stream)))
    return d % 8 == 0 ? SOLAR_NORM(true) : SOLAR_NORM(false);
#undef SOLAR_NORM
}

hipError_t launch_layer_norm_backward(const void* in, const float* weight, const float* mean, const float* rstd,
                                      const void* dout, int rows, int groups, int d, bool in_bf16, bool dout_bf16,
                                      void* din, float* dweight, float* dbias, float* partials, hipStream_t stream) {
    float* part = dweight || dbias ? partials : nullptr;
    hipError_t e;
#define SOLAR_NORM(V)                                                                                            \
    (in_bf16 ? (dout_bf16 ? backward<V, true, true>(in, weight, mean, rstd, dout, rows, groups, d, din, part, stream)    \
                          : backward<V, true, false>(in, weight, mean, rstd, dout, rows, groups, d, din, part, stream))  \
             : (dout_bf16 ? backward<V, false, true>(in, weight, mean, rstd, dout, rows, groups, d, din, part, stream)   \
                          : backward<V, false, false>(in, weight, mean, rstd, dout, rows, groups, d, din, part, stream)))
    e = d % 8 == 0 ? SOLAR_NORM(true) : SOLAR_NORM(false);
#undef SOLAR_NORM
    if (e != hipSuccess || !part) return e;
    const int width = groups * d;
    hipLaunchKernelGGL(norm_sum_kernel, dim3(ceil_div(width, 64), 2), dim3(1024), 0, stream, partials,
                       teams_for(rows, groups, d) / groups, width, dweight, dbias);
    return hipGetLastError();
}

}  // namespace solar
