// Rotary positions: the pair (a, b) of columns i of a head at position p becomes
//   (m (a cos x - b sin x), m (a sin x + b cos x)),  x = p freq[i],
// with the pairs (i, i + rot/2) or (2 i, 2 i + 1) of the first rot columns; the others are copied.  The gradient is the
// same with -x (the matrix is m times a rotation).
//
// Bound by memory: every element is read and written once.  A workgroup takes a few rows: one thread per row and pair
// forms the angle, in turns and in double precision (a far position times a frequency loses its fraction in float: at
// p = 10^6 a float angle is off by 0.06), and all heads of Q and K then share the cosines and sines through LDS.
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

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

// eight consecutive elements at p
template <bool BF16>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
    if constexpr (BF16) {
        const v4u u = *reinterpret_cast<const v4u*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(u[i]);
            x[2 * i + 1] = bf16_hi(u[i]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const v4f u = reinterpret_cast<const v4f*>(p)[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * j + i] = u[i];
        }
    }
}

template <bool BF16>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
    if constexpr (BF16) {
        v8bf u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (__bf16)x[i];
        *reinterpret_cast<v8bf*>(p) = u;
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v4f u = {x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
            reinterpret_cast<v4f*>(p)[j] = u;
        }
    }
}

// VEC: whole vectors of eight columns lie in one half (or one run of pairs) of the rotated columns.  A unit is then two
// vectors of eight (half layout), one of them (interleaved), or one vector of columns that are copied; otherwise it is one
// pair, or one copied column.
template <bool BF16, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotary r, int tokens, bool copy) {
    using E = typename Elem<BF16>::type;
    constexpr int ES = BF16 ? 2 : 4;
    extern __shared__ __attribute__((aligned(16))) float2 turn[];       // [tokens][rot / 2] (m cos, m sin)
    const int pairs = r.rot / 2;
    const int64_t first = (int64_t)blockIdx.x * tokens, all = (int64_t)r.B * r.N;
    const int count = all - first < tokens ? (int)(all - first) : tokens;
    for (int i = threadIdx.x; i < count * pairs; i += kThreads) {
        const int64_t bn = first + i / pairs;
        const int n = (int)(bn % r.N);
        const int pos = r.positions ? r.positions[bn] : n;
        double x = (double)pos * (r.freq[i % pairs] * 0.15915494309189533577);
        x -= rint(x);
        float s, c;
        sincospif(2.f * (float)x, &s, &c);
        turn[i] = make_float2(r.amplitude * c, r.inverse ? -r.amplitude * s : r.amplitude * s);
    }
    __syncthreads();
    const int rot_units = VEC ? (INTERLEAVED ? r.rot / 8 : r.rot / 16) : pairs;
    const int copy_units = VEC ? (r.D - r.rot) / 8 : r.D - r.rot;
    const int units = rot_units + copy_units, heads = r.heads[0] + r.heads[1];
    const int per_token = units * heads;
    for (int i = threadIdx.x; i < count * per_token; i += kThreads) {
        const int tok = i / per_token, in_tok = i - tok * per_token;
        const int hh = in_tok / units, u = in_tok - hh * units;
        const int64_t bn = first + tok;
        const int b = (int)(bn / r.N), n = (int)(bn - (int64_t)b * r.N);
        const int which = hh >= r.heads[0];
        const int h = which ? hh - r.heads[0] : hh;
        const char* in = row_of(r.in[which], b, n, h);
        char* out = row_of(r.out[which], b, n, h);
        const bool valid = n < user_len(r.lengths, b, r.N);
        const float2* cs = turn + tok * pairs;
        if (u >= rot_units) {
            const int c = r.rot + (u - rot_units) * (VEC ? 8 : 1);
            if constexpr (VEC) {
                if (valid && !copy) continue;
#pragma unroll
                for (int j = 0; j < ES / 2; ++j) {
                    const v4u zero = {0u, 0u, 0u, 0u};
                    reinterpret_cast<v4u*>(out + c * ES)[j] = valid ? reinterpret_cast<const v4u*>(in + c * ES)[j] : zero;
                }
            } else {
                if (valid && !copy) continue;
                reinterpret_cast<E*>(out)[c] = valid ? reinterpret_cast<const E*>(in)[c] : (E)0.f;
            }
        } else if constexpr (!VEC) {
            const int ca = INTERLEAVED ? 2 * u : u, cb = INTERLEAVED ? 2 * u + 1 : u + pairs;
            float a = 0.f, d = 0.f;
            if (valid) {
                a = (float)reinterpret_cast<const E*>(in)[ca];
                d = (float)reinterpret_cast<const E*>(in)[cb];
                const float x = a * cs[u].x - d * cs[u].y;
                d = d * cs[u].x + a * cs[u].y;
                a = x;
            }
            reinterpret_cast<E*>(out)[ca] = (E)a;
            reinterpret_cast<E*>(out)[cb] = (E)d;
        } else if constexpr (INTERLEAVED) {
            float x[8], y[8];
            load8<BF16>(in + 8 * u * ES, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 t = cs[4 * u + j];
                y[2 * j] = valid ? x[2 * j] * t.x - x[2 * j + 1] * t.y : 0.f;
                y[2 * j + 1] = valid ? x[2 * j + 1] * t.x + x[2 * j] * t.y : 0.f;
            }
            store8<BF16>(out + 8 * u * ES, y);
        } else {
            float x[8], y[8];
            load8<BF16>(in + 8 * u * ES, x);
            load8<BF16>(in + (pairs + 8 * u) * ES, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 t = cs[8 * u + j];
                const float a = x[j], d = y[j];
                x[j] = valid ? a * t.x - d * t.y : 0.f;
                y[j] = valid ? d * t.x + a * t.y : 0.f;
            }
            store8<BF16>(out + 8 * u * ES, x);
            store8<BF16>(out + (pairs + 8 * u) * ES, y);
        }
    }
}

}  // namespace

hipError_t launch_rotary(const Rotary& r, hipStream_t stream) {
    const int pairs = r.rot / 2;
    // four rows a workgroup: 256 angles at 128 rotated columns, one a thread
    const int tokens = 4;
    const int64_t all = (int64_t)r.B * r.N;
    const dim3 grid((unsigned)((all + tokens - 1) / tokens)), block(kThreads);
    const size_t lds = sizeof(float2) * tokens * pairs;
    const bool vec = r.interleaved ? r.rot % 8 == 0 : r.rot % 16 == 0;
    const bool copy = r.in[0].data != r.out[0].data || (r.heads[1] && r.in[1].data != r.out[1].data);
#define SOLAR_ROTARY(BF, IL, V) hipLaunchKernelGGL((rotary_kernel<BF, IL, V>), grid, block, lds, stream, r, tokens, copy)
    if (r.bf16) {
        if (r.interleaved) { if (vec) SOLAR_ROTARY(true, true, true); else SOLAR_ROTARY(true, true, false); }
        else { if (vec) SOLAR_ROTARY(true, false, true); else SOLAR_ROTARY(true, false, false); }
    } else {
        if (r.interleaved) { if (vec) SOLAR_ROTARY(false, true, true); else SOLAR_ROTARY(false, true, false); }
        else { if (vec) SOLAR_ROTARY(false, false, true); else SOLAR_ROTARY(false, false, false); }
    }
#undef SOLAR_ROTARY
    return hipGetLastError();
}

}  // namespace solar
