// Linear attention with a decay for each head, row by row: S_t = g S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t; the form for
// single tokens, bound by reading and writing the states.
//
// The state is cut into slices of 32 columns, one workgroup each: eight lanes hold four columns, 32 groups of lanes hold
// D / 32 rows each, in registers from the first row of the sequence to the last.  A row costs one sum over the groups
// (three steps across lanes, one through LDS).  2048 states of 128 x 128 a step: 268 MB read and written in 50 us, launch and
// all (5.4 TB/s; a large copy 5.1).
#include "sequence.h"

namespace solar {

namespace {

constexpr int kSlice = 32;      // columns of the state per workgroup
constexpr int kThreads = 256;

template <bool BF16>
__device__ __forceinline__ float load1(const char* p, int i) {
    if constexpr (BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
    else return reinterpret_cast<const float*>(p)[i];
}

// IN_PLACE: the last states go where the first are read from
template <int D, bool BF16, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void decay_rows_kernel(Walk w) {
    constexpr int RPT = D / 32;             // rows of the state per thread
    constexpr int NS = D / kSlice;
    __shared__ float part[2][4][kSlice];
    const int slice = blockIdx.x % NS, h = blockIdx.x / NS % w.H, b = blockIdx.x / NS / w.H;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = (tid >> 3) * RPT, col = slice * kSlice + 4 * (tid & 7);
    const Kept g = kept(w.log_decay[h], 1);
    const size_t at = ((size_t)b * w.H + h) * D * D;
    const int len = user_len(w.lengths, b, w.N);
    float S[RPT][4];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        v4f x = {0.f, 0.f, 0.f, 0.f};
        if (w.state_in) x = *reinterpret_cast<const v4f*>(w.state_in + at + (row0 + i) * D + col);
#pragma unroll
        for (int c = 0; c < 4; ++c) S[i][c] = x[c];
    }
    for (int t = 0; t < len; ++t) {
        const char *q = row_of(w.q, b, t, h), *k = row_of(w.k, b, t, h), *v = row_of(w.v, b, t, h);
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        float vv[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) vv[c] = load1<BF16>(v, col + c);
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const float kr = load1<BF16>(k, row0 + r), qr = load1<BF16>(q, row0 + r);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                S[r][c] = fmaf(kr, vv[c], keep(S[r][c], g));
                o[c] = fmaf(qr, S[r][c], o[c]);
            }
        }
        if (!w.o.data) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            o[c] += __shfl_xor(o[c], 8);
            o[c] += __shfl_xor(o[c], 16);
            o[c] += __shfl_xor(o[c], 32);
            if (lane < 8) part[t & 1][wave][4 * lane + c] = o[c];
        }
        __syncthreads();        // the other half of `part` is free again: everybody has read it before coming here
        if (tid < kSlice) {
            float s = 0.f;
#pragma unroll
            for (int y = 0; y < 4; ++y) s += part[t & 1][y][tid];
            s *= w.o_scale;
            const int c = slice * kSlice + tid;
            char* out = row_of(w.o, b, t, h);
            if constexpr (BF16) reinterpret_cast<__bf16*>(out)[c] = (__bf16)s;
            else reinterpret_cast<float*>(out)[c] = s;
        }
    }
    if (w.o.data && tid < kSlice) {
        for (int t = len; t < w.N; ++t) {
            char* out = row_of(w.o, b, t, h);
            const int c = slice * kSlice + tid;
            if constexpr (BF16) reinterpret_cast<__bf16*>(out)[c] = (__bf16)0.f;
            else reinterpret_cast<float*>(out)[c] = 0.f;
        }
    }
    if (w.state_out) {
        // To a place of its own past the caches, which then hold what is read (2048 states of 128 x 128, the same two buffers again: a step
        // 60 us -> 51; from one to the other and back at 67 MB and 134 MB of states 8 to 18 % longer instead).  In place the next
        // token finds the states where they are read from: 256 states of 256 x 256 23.9 -> 22.2 us, 512 47.7 -> 42.5, 2048 of 128 x 128
        // 44.4 -> 43.2; with 1.4 GB of other layers' states in between within 3 % either way, below 34 MB equal.
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const v4f x = {S[r][0], S[r][1], S[r][2], S[r][3]};
            v4f* const to = reinterpret_cast<v4f*>(w.state_out + at + (row0 + r) * D + col);
            if constexpr (IN_PLACE) *to = x;
            else __builtin_nontemporal_store(x, to);
        }
    }
}

template <int D, bool BF16>
void launch_rows(const Walk& w, hipStream_t stream) {
    const dim3 grid(w.B * w.H * (D / kSlice)), block(kThreads);
    if (w.state_out == w.state_in) hipLaunchKernelGGL((decay_rows_kernel<D, BF16, true>), grid, block, 0, stream, w);
    else hipLaunchKernelGGL((decay_rows_kernel<D, BF16, false>), grid, block, 0, stream, w);
}

__global__ __launch_bounds__(64) void moment_sum_kernel(const double* __restrict__ m, int B, int H, int slices, float* dlog) {
    const int h = blockIdx.x;
    double s = 0.;
    for (int i = threadIdx.x; i < B * slices; i += 64) s += m[((size_t)(i / slices) * H + h) * slices + i % slices];
    for (int x = 32; x; x >>= 1) s += __shfl_xor(s, x);
    if (threadIdx.x == 0) dlog[h] = (float)s;
}

// a thread takes four columns of one row and shared head
__global__ __launch_bounds__(256) void share_sum_kernel(const float* __restrict__ in, int B, int N, int H, int Hkv, int D,
                                                        Heads out, bool bf16) {
    const int share = H / Hkv, vecs = D / 4;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)B * N * Hkv * vecs) return;
    const int c = 4 * (int)(i % vecs), hk = (int)(i / vecs % Hkv);
    const size_t bn = i / vecs / Hkv;
    const float* p = in + (bn * H + (size_t)hk * share) * D + c;
    v4f s = *reinterpret_cast<const v4f*>(p);
    for (int j = 1; j < share; ++j) s += *reinterpret_cast<const v4f*>(p + (size_t)j * D);
    char* o = row_of(out, (int)(bn / N), (int64_t)(bn % N), hk);
    if (bf16) {
        typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
        v4bf r = {(__bf16)s[0], (__bf16)s[1], (__bf16)s[2], (__bf16)s[3]};
        *reinterpret_cast<v4bf*>(o + 2 * c) = r;
    } else {
        *reinterpret_cast<v4f*>(o + 4 * c) = s;
    }
}

}  // namespace

hipError_t launch_decay_rows(const Walk& w, hipStream_t stream) {
    switch (w.D) {
        case 64: w.bf16 ? launch_rows<64, true>(w, stream) : launch_rows<64, false>(w, stream); break;
        case 128: w.bf16 ? launch_rows<128, true>(w, stream) : launch_rows<128, false>(w, stream); break;
        case 256: w.bf16 ? launch_rows<256, true>(w, stream) : launch_rows<256, false>(w, stream); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_moment_sum(const double* moments, int B, int H, int slices, float* dlog, hipStream_t stream) {
    hipLaunchKernelGGL(moment_sum_kernel, dim3(H), dim3(64), 0, stream, moments, B, H, slices, dlog);
    return hipGetLastError();
}

hipError_t launch_share_sum(const float* in, int B, int N, int H, int Hkv, int D, const Heads& out, bool bf16,
                            hipStream_t stream) {
    const size_t n = (size_t)B * N * Hkv * (D / 4);
    hipLaunchKernelGGL(share_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, in, B, N, H, Hkv, D,
                       out, bf16);
    return hipGetLastError();
}

}  // namespace solar
