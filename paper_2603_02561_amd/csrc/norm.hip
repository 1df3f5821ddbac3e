// Layer norm over groups of columns and its gradient.  A row of d elements:
//   y = (x - mu) rstd w + b,  rstd = 1 / sqrt(mean((x - mu)^2) + eps)
//   dx = rstd (a - mean(a) - xh mean(a xh)),  a = dy w,  xh = (x - mu) rstd;   dw = sum dy xh,  db = sum dy
//
// Bound by memory: x is read once and y written once; the gradient reads x and dy once and writes dx once.  A row stays
// in registers, so mean and variance are taken one after the other from the same values (no difference of two large
// sums).  Between 8 and 1024 threads share a row, by its width; each such team walks over rows of one group, the next of them
// on its way, so that its weights, and its sums for dw and db, stay in registers.  The sums of a workgroup go to the workspace
// and are added by a second kernel in a fixed order.  65536 x 16 x 128 bf16 forward: 545 MB in 99 us (5.5 TB/s); gradient of
// 32768 x 4096 bf16: 806 MB in 147 us and 6 for the sums (5.2 TB/s).  A large copy reaches 5.1 here.
#include "sequence.h"

namespace solar {

namespace {

// Threads of a workgroup whose rows take T threads each.
constexpr int block_for(int T) { return T < 256 ? 256 : T; }

template <bool BF16>
struct Elem {
    using type = float;
};
template <>
struct Elem<true> {
    using type = __bf16;
};

// Column of vector v, element e of thread t in a team of T.
template <int T>
__device__ __forceinline__ int column(int t, int v, int e) {
    return (v * T + t) * 8 + e;
}

// A team's part of one row as it comes from memory; what lies past d is zero.  VEC: rows start on a vector and end with one.
// Otherwise the vectors lie wherever the row does (the memory takes that in one access too) and the last one is taken apart.
template <int T, int NV, bool VEC, bool BF16>
struct Row {
    static constexpr int VS = BF16 ? 1 : 2;     // 16-byte loads of eight elements
    v4u raw[NV][VS];

    __device__ __forceinline__ void load(const void* base, size_t at, int d, int t) {
        using E = typename Elem<BF16>::type;
        const E* p = reinterpret_cast<const E*>(base) + at;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = column<T>(t, v, 0);
#pragma unroll
            for (int j = 0; j < VS; ++j) raw[v][j] = v4u{0u, 0u, 0u, 0u};
            if constexpr (VEC) {
                if (c < d)
#pragma unroll
                    for (int j = 0; j < VS; ++j) raw[v][j] = reinterpret_cast<const v4u*>(p + c)[j];
            } else if (c + 8 <= d) {
                __builtin_memcpy(raw[v], __builtin_assume_aligned(p + c, sizeof(E)), sizeof(raw[v]));
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (c + e < d) {
                        if constexpr (BF16)
                            raw[v][0][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[c + e] << (16 * (e & 1));
                        else
                            raw[v][e / 4][e % 4] = __float_as_uint((float)p[c + e]);
                    }
            }
        }
    }
    __device__ __forceinline__ void get(float (&x)[NV][8]) const {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (BF16) x[v][e] = e & 1 ? bf16_hi(raw[v][0][e / 2]) : bf16_lo(raw[v][0][e / 2]);
                else x[v][e] = __uint_as_float(raw[v][e / 4][e % 4]);
            }
    }
};

template <int T, int NV, bool VEC, bool BF16>
__device__ __forceinline__ void store_row(void* base, size_t at, int d, int t, const float (&x)[NV][8]) {
    using E = typename Elem<BF16>::type;
    E* p = reinterpret_cast<E*>(base) + at;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = column<T>(t, v, 0);
        E u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = (E)x[v][e];
        if constexpr (VEC) {
            if (c < d) __builtin_memcpy(__builtin_assume_aligned(p + c, 16), u, sizeof(u));
        } else if (c + 8 <= d) {
            __builtin_memcpy(__builtin_assume_aligned(p + c, sizeof(E)), u, sizeof(u));
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (c + e < d) p[c + e] = u[e];
        }
    }
}

// Sums of K values over a team, in every thread of it.  `turn` alternates between the two halves of `part`, so that one
// barrier a call is enough.
template <int T, int K>
__device__ __forceinline__ void team_sum(float (&s)[K], float (*part)[16][K], int& turn) {
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
        for (int k = 0; k < K; ++k) {
            s[k] = part[turn][0][k];
#pragma unroll
            for (int y = 1; y < T / 64; ++y) s[k] += part[turn][y][k];
        }
        turn ^= 1;
    }
}

// `teams` teams, a multiple of `groups`, walk over `rows` rows of d elements (groups counted as rows).
template <int T, int NV, bool VEC, bool IN_BF16, bool OUT_BF16>
__global__ __launch_bounds__(block_for(T)) void layer_norm_kernel(const void* in, const float* __restrict__ weight,
                                                              const float* __restrict__ bias, size_t rows, int groups,
                                                              int teams, int d, float eps, void* out, float* mean,
                                                              float* rstd) {
    __shared__ float part[2][16][1];
    int turn = 0;
    const int t = threadIdx.x % T, team = blockIdx.x * (block_for(T) / T) + threadIdx.x / T;
    if (team >= teams) return;      // whole workgroups where a team is one
    const int group = team % groups;
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column<T>(t, v, e);
            w[v][e] = weight && c < d ? weight[(size_t)group * d + c] : 1.f;
            b[v][e] = bias && c < d ? bias[(size_t)group * d + c] : 0.f;
        }
    const float inv = 1.f / (float)d;
    Row<T, NV, VEC, IN_BF16> next;
    next.load(in, (size_t)team * d, d, t);
    for (size_t row = team; row < rows; row += teams) {
        float x[NV][8];
        next.get(x);
        if (row + teams < rows) next.load(in, (row + teams) * d, d, t);
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
                x[v][e] = column<T>(t, v, e) < d ? x[v][e] - mu : 0.f;
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

// A workgroup takes rows of one group, blockIdx.x % groups, its teams one each at a time.  partials [2][blocks / groups][groups]
// [d]: its sums of dy xh and of dy; null where neither is wanted.
template <int T, int NV, bool VEC, bool IN_BF16, bool DOUT_BF16>
__global__ __launch_bounds__(block_for(T)) void layer_norm_backward_kernel(
    const void* in, const float* __restrict__ weight, const float* __restrict__ mean, const float* __restrict__ rstd,
    const void* dout, size_t rows, int groups, int d, void* din, float* partials) {
    constexpr int TEAMS = block_for(T) / T;
    __shared__ float part[2][16][2];
    __shared__ float sums[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? T * NV * 8 : 1];
    int turn = 0;
    const int t = threadIdx.x % T, team = threadIdx.x / T;
    const int group = blockIdx.x % groups, block = blockIdx.x / groups, blocks = gridDim.x / groups;
    float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column<T>(t, v, e);
            w[v][e] = weight && c < d ? weight[(size_t)group * d + c] : 1.f;
            dw[v][e] = db[v][e] = 0.f;
        }
    const float inv = 1.f / (float)d;
    const size_t step = (size_t)blocks * TEAMS;
    size_t i = (size_t)block * TEAMS + team;
    Row<T, NV, VEC, IN_BF16> nx;
    Row<T, NV, VEC, DOUT_BF16> ny;
    float mu_next = 0.f, rs_next = 0.f;
    auto fetch = [&](size_t r) __attribute__((always_inline)) {
        const size_t row = r * groups + group;
        nx.load(in, row * d, d, t);
        ny.load(dout, row * d, d, t);
        mu_next = mean[row];
        rs_next = rstd[row];
    };
    if (i < rows) fetch(i);
    for (; i < rows; i += step) {
        float x[NV][8], dy[NV][8];
        nx.get(x);
        ny.get(dy);
        const float mu = mu_next, rs = rs_next;
        if (i + step < rows) fetch(i + step);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // past d dy is zero, and a zero takes the place of what x would give there
                x[v][e] = column<T>(t, v, e) < d ? (x[v][e] - mu) * rs : 0.f;
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
        store_row<T, NV, VEC, IN_BF16>(din, (i * groups + group) * d, d, t, x);
    }
    if (!partials) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* out = partials + (((size_t)which * blocks + block) * groups + group) * d;
        const float(&mine)[NV][8] = which ? db : dw;
        if constexpr (TEAMS == 1) {
            store_row<T, NV, VEC, false>(out, 0, d, t, mine);
        } else {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[team][column<T>(t, v, e)] = mine[v][e];
            __syncthreads();
            for (int c = threadIdx.x; c < d; c += block_for(T)) {
                float s = 0.f;
                for (int y = 0; y < TEAMS; ++y) s += sums[y][c];
                out[c] = s;
            }
        }
    }
}

// dweight and dbias [width] from [2][n][width]: 32 columns a workgroup, 32 of its threads down each
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* __restrict__ partials, int n, int width, float* dweight,
                                                        float* dbias) {
    __shared__ float sum[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const float* p = partials + (size_t)blockIdx.y * n * width;
    float s = 0.f;
    if (c < width)
        for (int i = y; i < n; i += 32) s += p[(size_t)i * width + c];
    sum[y][x] = s;
    __syncthreads();
    s = sum[x][y];              // column y of the workgroup, row x of the sums
#pragma unroll
    for (int m = 16; m; m >>= 1) s += __shfl_xor(s, m);
    if (x == 0 && blockIdx.x * 32 + y < width) out[blockIdx.x * 32 + y] = s;
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
    if (d <= 8192) return {512, 2};
    return {1024, 2};
}

// Teams of the forward pass: four workgroups for each compute unit, whole groups, no team without a row.
int teams_for(int rows, int groups, int d) {
    const int per_block = block_for(team_for(d).threads) / team_for(d).threads;
    const size_t all = (size_t)rows * groups, want = (size_t)1024 * per_block;
    const size_t teams = (want + groups - 1) / groups * groups;
    return (int)(teams < all ? teams : all);
}

// Workgroups of the gradient for each group: their sums for dw and db are written once each, so there are no more than keep
// the GPU busy (512 together: 32768 rows of 4096 take 156 us, with 1024 185, as three of them fit a compute unit), and none whose
// teams would have less than four rows.
int blocks_for(int rows, int groups, int d) {
    const int per_block = block_for(team_for(d).threads) / team_for(d).threads;
    const int want = ceil_div(512, groups), most = ceil_div(rows, 4 * per_block);
    return want < most ? want : most;
}

}  // namespace

size_t norm_partial_floats(int rows, int groups, int d) { return (size_t)2 * blocks_for(rows, groups, d) * groups * d; }

#define SOLAR_NORM_SHAPES(CALL)                                  \
    switch (tm.threads * 16 + tm.vectors) {                      \
        case 8 * 16 + 1: CALL(8, 1); break;                      \
        case 16 * 16 + 1: CALL(16, 1); break;                    \
        case 32 * 16 + 1: CALL(32, 1); break;                    \
        case 64 * 16 + 1: CALL(64, 1); break;                    \
        case 64 * 16 + 2: CALL(64, 2); break;                    \
        case 256 * 16 + 1: CALL(256, 1); break;                  \
        case 256 * 16 + 2: CALL(256, 2); break;                  \
        case 512 * 16 + 2: CALL(512, 2); break;                  \
        case 1024 * 16 + 2: CALL(1024, 2); break;                \
        default: return hipErrorInvalidValue;                    \
    }

namespace {

template <bool VEC, bool A, bool B>
hipError_t forward(const void* in, const float* weight, const float* bias, int rows, int groups, int d, float eps,
                   void* out, float* mean, float* rstd, hipStream_t stream) {
    const Team tm = team_for(d);
    const int teams = teams_for(rows, groups, d);
    const int threads = block_for(tm.threads);
    const dim3 grid(ceil_div(teams, threads / tm.threads)), block(threads);
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
    const dim3 grid((unsigned)blocks_for(rows, groups, d) * groups), block(block_for(tm.threads));
#define SOLAR_CALL(T, NV)                                                                                              \
    hipLaunchKernelGGL((layer_norm_backward_kernel<T, NV, VEC, A, B>), grid, block, 0, stream, in, weight, mean, rstd, \
                       dout, (size_t)rows, groups, d, din, partials)
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
    hipLaunchKernelGGL(norm_sum_kernel, dim3(ceil_div(width, 32), 2), dim3(1024), 0, stream, partials,
                       blocks_for(rows, groups, d), width, dweight, dbias);
    return hipGetLastError();
}

}  // namespace solar
