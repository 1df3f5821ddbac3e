// Rotary positions: the pair (a, b) of columns i of a head at position p becomes
//   (m (a cos x - b sin x), m (a sin x + b cos x)),  x = p freq[i],
// with the pairs (i, i + rot/2) or (2 i, 2 i + 1) of the first rot columns; the others are copied.  The gradient is the
// same with -x (the matrix is m times a rotation).
//
// Bound by memory: every element is read and written once.  A workgroup takes a few rows: one thread per row and pair
// forms the angle, in turns and in double precision (a far position times a frequency loses its fraction in float: at
// p = 10^6 a float angle is off by 0.06), and all heads of Q and K then share the cosines and sines through LDS.  65536 rows of 40
// heads of 128 bf16 columns, 64 of them rotated: 1.34 GB in 247 to 265 us, 5.1 to 5.4 TB/s, the rate of a large copy.
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

// Eight consecutive elements at p; ALIGNED: at a multiple of 16 bytes, else wherever an element may be (the memory takes that in
// one access too).
template <bool BF16, bool ALIGNED>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
    constexpr int V = BF16 ? 1 : 2;
    v4u u[V];
    if constexpr (ALIGNED) {
#pragma unroll
        for (int j = 0; j < V; ++j) u[j] = reinterpret_cast<const v4u*>(p)[j];
    } else {
        __builtin_memcpy(u, __builtin_assume_aligned(p, BF16 ? 2 : 4), sizeof(u));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (BF16) x[i] = i & 1 ? bf16_hi(u[0][i / 2]) : bf16_lo(u[0][i / 2]);
        else x[i] = __uint_as_float(u[i / 4][i % 4]);
    }
}

template <bool BF16, bool ALIGNED>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
    if constexpr (BF16) {
        v8bf u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (__bf16)x[i];
        if constexpr (ALIGNED) *reinterpret_cast<v8bf*>(p) = u;
        else __builtin_memcpy(__builtin_assume_aligned(p, 2), &u, sizeof(u));
    } else {
        v4f u[2] = {{x[0], x[1], x[2], x[3]}, {x[4], x[5], x[6], x[7]}};
        if constexpr (ALIGNED) {
#pragma unroll
            for (int j = 0; j < 2; ++j) reinterpret_cast<v4f*>(p)[j] = u[j];
        } else {
            __builtin_memcpy(__builtin_assume_aligned(p, 4), u, sizeof(u));
        }
    }
}

// A head is cut into units, one for a thread at a time: eight pairs (half layout; their second columns start on a vector where
// EVEN) or four (interleaved), then the pairs that are left over, then the columns to copy: up to the next vector one by one,
// then by vectors.  Every unit reads its columns before it writes them, and no two share a column, so a call may be in place.
template <bool BF16, bool INTERLEAVED, bool EVEN>
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
    const int whole = INTERLEAVED ? r.rot / 8 : pairs / 8;              // units of vectors
    const int odd = INTERLEAVED ? r.rot % 8 / 2 : pairs % 8;            // pairs left over
    const int lone = (8 - r.rot % 8) % 8;                               // columns up to the next vector
    const int heads = r.heads[0] + r.heads[1];
    // all heads' pairs, then all heads' copied columns: the lanes of a wave do the same
    struct Place {
        const char* in;
        char* out;
        int tok, u;
        bool valid;
    };
    auto place = [&](int i, int units) __attribute__((always_inline)) {
        Place p;
        const int at = i / units;
        p.u = i - at * units;
        p.tok = at / heads;
        const int hh = at - p.tok * heads, which = hh >= r.heads[0], h = which ? hh - r.heads[0] : hh;
        const int64_t bn = first + p.tok;
        const int b = (int)(bn / r.N), n = (int)(bn - (int64_t)b * r.N);
        p.in = row_of(r.in[which], b, n, h);
        p.out = row_of(r.out[which], b, n, h);
        p.valid = n < user_len(r.lengths, b, r.N);
        return p;
    };
    const int turned = whole + odd, copied = lone + (r.D - r.rot - lone) / 8;
    for (int i = threadIdx.x; i < count * heads * turned; i += kThreads) {
        const Place at = place(i, turned);
        const float2* cs = turn + at.tok * pairs;
        const bool valid = at.valid;
        if (at.u < whole) {
            const int c = 8 * at.u;
            float x[8], y[8];
            if constexpr (INTERLEAVED) {
                load8<BF16, true>(at.in + c * ES, x);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 t = cs[c / 2 + j];
                    y[2 * j] = valid ? x[2 * j] * t.x - x[2 * j + 1] * t.y : 0.f;
                    y[2 * j + 1] = valid ? x[2 * j + 1] * t.x + x[2 * j] * t.y : 0.f;
                }
                store8<BF16, true>(at.out + c * ES, y);
            } else {
                load8<BF16, true>(at.in + c * ES, x);
                load8<BF16, EVEN>(at.in + (pairs + c) * ES, y);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 t = cs[c + j];
                    const float a = x[j], d = y[j];
                    x[j] = valid ? a * t.x - d * t.y : 0.f;
                    y[j] = valid ? d * t.x + a * t.y : 0.f;
                }
                store8<BF16, true>(at.out + c * ES, x);
                store8<BF16, EVEN>(at.out + (pairs + c) * ES, y);
            }
        } else {
            const int p = (INTERLEAVED ? 4 : 8) * whole + at.u - whole;
            const int ca = INTERLEAVED ? 2 * p : p, cb = INTERLEAVED ? 2 * p + 1 : p + pairs;
            float a = 0.f, d = 0.f;
            if (valid) {
                a = (float)reinterpret_cast<const E*>(at.in)[ca];
                d = (float)reinterpret_cast<const E*>(at.in)[cb];
                const float x = a * cs[p].x - d * cs[p].y;
                d = d * cs[p].x + a * cs[p].y;
                a = x;
            }
            reinterpret_cast<E*>(at.out)[ca] = (E)a;
            reinterpret_cast<E*>(at.out)[cb] = (E)d;
        }
    }
    if (!copy && !r.lengths) return;
    for (int i = threadIdx.x; i < count * heads * copied; i += kThreads) {
        const Place at = place(i, copied);
        if (at.valid && !copy) continue;
        if (at.u < lone) {
            const int c = r.rot + at.u;
            reinterpret_cast<E*>(at.out)[c] = at.valid ? reinterpret_cast<const E*>(at.in)[c] : (E)0.f;
        } else {
            const int c = r.rot + lone + (at.u - lone) * 8;
#pragma unroll
            for (int j = 0; j < ES / 2; ++j) {
                const v4u zero = {0u, 0u, 0u, 0u};
                reinterpret_cast<v4u*>(at.out + c * ES)[j] = at.valid ? reinterpret_cast<const v4u*>(at.in + c * ES)[j] : zero;
            }
        }
    }
}

}  // namespace

hipError_t launch_rotary(const Rotary& r, hipStream_t stream) {
    const int pairs = r.rot / 2;
    const int tokens = kRotaryRows;
    const int64_t all = (int64_t)r.B * r.N;
    const dim3 grid((unsigned)((all + tokens - 1) / tokens)), block(kThreads);
    const size_t lds = sizeof(float2) * tokens * pairs;
    const bool even = r.interleaved || r.rot % 16 == 0;
    auto same = [](const Heads& x, const Heads& y) {
        return x.data == y.data && x.s.batch == y.s.batch && x.s.row == y.s.row && x.s.head == y.s.head;
    };
    const bool copy = !same(r.in[0], r.out[0]) || (r.heads[1] && !same(r.in[1], r.out[1]));
#define SOLAR_ROTARY(BF, IL, V) hipLaunchKernelGGL((rotary_kernel<BF, IL, V>), grid, block, lds, stream, r, tokens, copy)
    if (r.bf16) {
        if (r.interleaved) SOLAR_ROTARY(true, true, true);
        else if (even) SOLAR_ROTARY(true, false, true);
        else SOLAR_ROTARY(true, false, false);
    } else {
        if (r.interleaved) SOLAR_ROTARY(false, true, true);
        else if (even) SOLAR_ROTARY(false, false, true);
        else SOLAR_ROTARY(false, false, false);
    }
#undef SOLAR_ROTARY
    return hipGetLastError();
}

}  // namespace solar
