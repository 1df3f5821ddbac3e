// Linear attention with a decay for each head, in chunks of C rows on the matrix unit.  With local rows i = 0 .. C-1 and
// the state S in front of them (sequence.h: pre = 1 forward, 0 in reverse):
//   O = diag(g^(i+pre)) Q S + ((Q K^T) o M) V,   M_ij = g^(i-j) for j <= i,  0 else
//   S <- g^C S + K^T diag(g^(C-pre-j)) V
// A workgroup holds W columns of S in registers, sixteen per wave, and walks over the rows of one part of
// one user's sequence for one head.  Everything is formed transposed (O^T = S^T Q^T + V^T P^T): a lane's entries of S, eight
// of one column, are then an operand of the matrix instruction as they stand, and so are K^T and V from the transposing LDS
// read; only P = Q K^T o M goes through LDS, each wave forming a share of it.
//
// Precision.  Sums and S are float.  The matrix unit takes bf16, so a float operand is cut into bf16 terms that add up to it:
// three (24 bits) where the sum stays float - the state - and for float inputs, whose products take the six pairs of terms
// above 2^-24; two (16 bits) for S and P where the result is rounded to bf16 anyway (2^-8).  g^C S is S + (g^C - 1) S, so that
// the error of a rounded g^C does not add up over the chunks.
#include "kernels.h"
#include "sequence.h"

namespace solar {

namespace {

constexpr int kJoinThreads = 256;

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

template <int D, bool BF16, bool MOMENT>
struct ChunkCfg {
    static constexpr int C = BF16 && D <= 128 && !MOMENT ? 64 : 32;     // rows of a chunk
    static constexpr int W = D < 128 ? D : 128;                         // columns of S per workgroup, 16 per wave
    static constexpr int kThreads = 4 * W;
    static constexpr int NT = BF16 ? 1 : 3;                             // terms of an input
    static constexpr int TP = BF16 && !MOMENT ? 2 : 3;                  // terms of P and S where they meet V and Q
    static constexpr int LP = C + 8;                                    // bf16 per row of P's images
    static constexpr int kQ = NT * C * D, kV = NT * C * W, kP = TP * C * LP;
    static constexpr size_t lds_bytes(bool out) { return 2 * (size_t)(kQ + kV + (out ? kQ + kP : 0)) + 4 * (4 * C + 3 + 16); }
    // Waves per SIMD that the registers are shared out for: two workgroups per compute unit where LDS has room for two and
    // 128 registers hold what a wave needs.
    static constexpr int waves(bool out) { return 2 * lds_bytes(out) <= 160 * 1024 && !(D == 256 || (MOMENT && D == 128)) ? W / 32 : W / 64; }
};

typedef float v8f __attribute__((ext_vector_type(8)));

// The float that a bf16 stands for, from pairs in a register: converted one by one the compiler takes every conversion twice.
__device__ __forceinline__ v8f widen(v8bf x) {
    const v4u u = __builtin_bit_cast(v4u, x);
    v8f f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = bf16_lo(u[e]);
        f[2 * e + 1] = bf16_hi(u[e]);
    }
    return f;
}

// x = the sum of its terms, to 8 bits each
template <int T>
__device__ __forceinline__ void split(v8f x, v8bf (&s)[T]) {
#pragma unroll
    for (int k = 0; k < T; ++k) {
        s[k] = __builtin_convertvector(x, v8bf);
        if (k + 1 < T) x -= widen(s[k]);
    }
}

__device__ __forceinline__ v4f mfma(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// c[n] + a[n] b[n] over the pairs of terms that matter, the small ones first; the products that follow one another are
// independent.  a or b is the same for all n.
template <int N, int TA, int TB>
__device__ __forceinline__ void products(const v8bf (&a)[TA], const v8bf (&b)[N][TB], v4f (&c)[N]) {
    constexpr int T = TA > TB ? TA : TB;
#pragma unroll
    for (int sum = T - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < TA; ++i)
            if (sum - i >= 0 && sum - i < TB)
#pragma unroll
                for (int n = 0; n < N; ++n) c[n] = mfma(a[i], b[n][sum - i], c[n]);
}

template <int N, int TA, int TB>
__device__ __forceinline__ void products(const v8bf (&a)[N][TA], const v8bf (&b)[TB], v4f (&c)[N]) {
    constexpr int T = TA > TB ? TA : TB;
#pragma unroll
    for (int sum = T - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < TA; ++i)
            if (sum - i >= 0 && sum - i < TB)
#pragma unroll
                for (int n = 0; n < N; ++n) c[n] = mfma(a[n][i], b[sum - i], c[n]);
}

template <int TA, int TB>
__device__ __forceinline__ v4f product(const v8bf (&a)[TA], const v8bf (&b)[TB], v4f c) {
    constexpr int T = TA > TB ? TA : TB;
#pragma unroll
    for (int sum = T - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < TA; ++i)
            if (sum - i >= 0 && sum - i < TB) c = mfma(a[i], b[sum - i], c);
    return c;
}

// The images of rows in LDS have no padding: chunks of eight elements lie in row `row` at the place (chunk ^ swizzle(row)).  Then
// neither the reads of one chunk from sixteen rows, nor the transposing reads of four rows, nor the stores of whole rows meet
// in a bank (a row is 32, 64 or 128 of the 64 banks long).
template <int COLS>
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (COLS == 64) return ((row >> 1 & 1) << 2) | (row >> 2 & 3);
    else return ((row & 3) << 2) | (row >> 2 & 3);
}

__device__ __forceinline__ v8bf lds8(const __bf16* p) { return *reinterpret_cast<const v8bf*>(p); }

// Transposing read of 16-bit elements from eight rows r .. r+7, r a multiple of 8, of an image: lane i of a group of 16 passes
// the address of four elements in row i/4 and receives element i%4 of the lanes i/4, 4 + i/4, 8 + i/4, 12 + i/4: rows 0..3 of
// "its" column.  at: the place of its four elements in row r + i/4; four rows on a chunk lies at its place ^ 1.
template <int COLS>
__device__ __forceinline__ v8bf lds_turned(const __bf16* img, uint32_t at) {
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s* lds_ptr;
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(img + at));
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(img + (at ^ 8) + 4 * COLS));
    typedef short v8s __attribute__((ext_vector_type(8)));
    const v8s r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(v8bf, r);
}

// Rows of one tensor, head and user in the order of the walk.  Addresses are a uniform base and a 32-bit offset per lane: row
// i of the chunk that starts at row `done` is at(done) + off(i), at() lying below all rows of the chunk.
template <int C>
struct Rows {
    const char* first;
    int64_t step;           // bytes
    uint32_t apart;         // |step| / 16, below 2^22 by the host's checks
    uint32_t turn;          // C - 1 where the walk goes down, else 0

    __device__ __forceinline__ static Rows make(const char* first, int64_t step) {
        return {first, step, (uint32_t)((step < 0 ? -step : step) / 16), step < 0 ? C - 1u : 0u};
    }
    __device__ __forceinline__ const char* at(int done) const { return first + done * step - (turn ? (int64_t)apart * 16 * (C - 1) : 0); }
    __device__ __forceinline__ uint32_t off(uint32_t i) const { return __umul24(i ^ turn, apart) << 4; }
};

// One thread's share of the rows of a chunk on their way from memory to LDS: vectors of eight elements.
template <int C, int COLS, int THREADS, bool BF16>
struct Fetch {
    static constexpr int PER = COLS / 8, N = C * PER / THREADS, VS = BF16 ? 1 : 2;
    v4u x[N][VS];

    // Row i is row done + i, or the last of the `count` rows where there are fewer: no branches, which would put the values
    // into scratch memory.
    __device__ __forceinline__ void load(const Rows<C>& r, int done, int count) {
        done = done < count ? done : count - 1;
        const char* p = r.at(done);
        const uint32_t last = count - 1 - done, tid = fresh_tid(), i0 = tid / PER, col = tid % PER * (VS * 16);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const uint32_t i = i0 + u * (THREADS / PER);
            const uint32_t at = r.off(i < last ? i : last) + col;
#pragma unroll
            for (int v = 0; v < VS; ++v) x[u][v] = *reinterpret_cast<const v4u*>(p + (at + v * 16));
        }
    }

    __device__ __forceinline__ void store(__bf16* img) const {
        const uint32_t tid = fresh_tid();
        const int i0 = tid / PER, c = tid % PER;
        // the rows of a thread are a multiple of 16 apart, so that its chunks have the same place in all of them
        static_assert(N == 1 || THREADS / PER % 16 == 0, "");
        __bf16* to = img + i0 * COLS + ((c ^ swizzle<COLS>(i0)) << 3);
#pragma unroll
        for (int u = 0; u < N; ++u, to += THREADS / PER * COLS) {
            if constexpr (BF16) {
                *reinterpret_cast<v4u*>(to) = x[u][0];
            } else {
                v8f f;
                v8bf s[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(x[u][e / 4][e % 4]);
                split<3>(f, s);
#pragma unroll
                for (int k = 0; k < 3; ++k) *reinterpret_cast<v8bf*>(to + k * C * COLS) = s[k];
            }
        }
    }

    // the rows from cnt on
    __device__ __forceinline__ static void clear(__bf16* img, int cnt) {
#pragma unroll 1
        for (int e = cnt * PER + threadIdx.x; e < C * PER; e += THREADS)
#pragma unroll
            for (int k = 0; k < (BF16 ? 1 : 3); ++k)
                *reinterpret_cast<v4u*>(img + k * C * COLS + (e << 3)) = v4u{0u, 0u, 0u, 0u};   // whole rows: no swizzle
    }
};

// kOut: outputs; kState: the state behind each part but the last, from a zero state, into w.parts; kMoment: the derivative of
// the outputs by log g, summed against their gradient; kMomentState: kState, and the derivative of these states; kLast: the
// state behind the last part, where nobody wants outputs.
enum { kOut, kState, kMoment, kMomentState, kLast };
constexpr bool is_moment(int mode) { return mode == kMoment || mode == kMomentState; }
constexpr bool is_out(int mode) { return mode == kOut || mode == kMoment; }

template <int D, bool BF16, int MODE>
__global__ __launch_bounds__((ChunkCfg<D, BF16, is_moment(MODE)>::kThreads), (ChunkCfg<D, BF16, is_moment(MODE)>::waves(is_out(MODE)))) void
decay_chunk_kernel(Walk w) {
    constexpr bool MOMENT = is_moment(MODE), OUT = is_out(MODE), STATES = MODE == kState || MODE == kMomentState;
    using F = ChunkCfg<D, BF16, MOMENT>;
    constexpr int C = F::C, W = F::W, THREADS = F::kThreads, NT = F::NT, TP = F::TP, LP = F::LP;
    constexpr int NW = THREADS / 64, NS = D / W, NJ = D / 32, NC = C / 16, NK = C / 32, ES = BF16 ? 2 : 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __bf16* const ki = reinterpret_cast<__bf16*>(lds);                  // [NT][C][D]
    __bf16* const vi = ki + F::kQ;                                      // [NT][C][W]
    __bf16* const qi = vi + F::kV;                                      // [NT][C][D]
    __bf16* const pi = qi + (OUT ? F::kQ : 0);                          // [TP][C][LP]: row t, column s
    float* const pw = reinterpret_cast<float*>(pi + (OUT ? F::kP : 0)); // o_scale g^n, n = 0 .. C
    float* const pk = pw + C + 1 + C;                                   // kv_scale g^n, n = -C .. C, zero below 0
    float* const po = pk + C + 1 + 16;                                  // o_scale kv_scale g^n, n = -16 .. C, zero below 0

    // Slices of one part and heads that share K and V run on one XCD (workgroups go to the eight in turn), where they
    // find each other's rows in its L2.
    const int share = w.k.share, nparts = MODE == kLast ? 1 : STATES ? w.nparts - 1 : w.nparts;
    const int turn = blockIdx.x >> 3, slice = turn % NS, k0 = turn / NS;
    const int64_t unit = (int64_t)(k0 / share * 8 + (blockIdx.x & 7)) * share + k0 % share;
    if (unit >= (int64_t)w.B * w.H * nparts) return;
    const int h = (int)(unit % w.H), b = (int)(unit / w.H / nparts);
    // in the order of the walk; the last part's state is nobody's start
    const int order = MODE == kLast ? w.nparts - 1 : (int)(unit / w.H % nparts), part = w.reverse ? w.nparts - 1 - order : order;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c16 = lane & 15, g4 = lane >> 4;
    const int len = user_len(w.lengths, b, w.N);
    const int row0 = part * w.part_rows;                                // may not overflow: part < nparts
    const int rows = w.N - row0 < w.part_rows ? w.N - row0 : w.part_rows;
    const int count = len - row0 < 0 ? 0 : (len - row0 < rows ? len - row0 : rows);
    const int pre = w.reverse ? 0 : 1;
    const float lg = w.log_decay[h];
    const int col0 = slice * W;                                         // this workgroup's columns of S
    const int mycol = col0 + wave * 16;                            // this wave's

    for (int n = tid; n <= C; n += THREADS) {
        const float x = n ? expf(lg * (float)n) : 1.f;                  // log g may be -infinity
        pw[n] = w.o_scale * x;
        pk[n] = w.kv_scale * x;
        po[n] = w.o_scale * w.kv_scale * x;
        if (n && n <= 16) po[-n] = 0.f;
        if (n) pk[-n] = 0.f;
    }

    if constexpr (OUT) {
        // P above the diagonal, as far as the 32 rows of V that a product takes reach: zero, and never written again
        for (int n = tid; n < TP * C * 2; n += THREADS) {
            const int t = n / 2 % C, k = n / 2 / C;
            if (!(t & 16)) *reinterpret_cast<v4u*>(pi + (k * C + t) * LP + (t & ~15) + 16 + 8 * (n & 1)) = v4u{0u, 0u, 0u, 0u};
        }
    }

    // S[j][a]: rows 32 j + 8 g4 + 4 a + (0..3), column mycol + c16
    v4f S[NJ][2], T[MOMENT ? NJ : 1][2];
    const size_t state_at = ((size_t)b * w.H + h) * D * D;
    const size_t part_at = (((size_t)b * w.H + h) * (w.nparts - 1) + (order - 1)) * D * D;   // order > 0 only
    const float* start = w.nparts == 1 || order == 0 ? (w.state_in ? w.state_in + state_at : nullptr) : w.parts + part_at;
    const bool turned = order == 0 && w.in_turned;
    if (STATES) start = nullptr;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 32 * j + 8 * g4 + 4 * a + i, col = mycol + c16;
                    S[j][a][i] = start ? start[turned ? (size_t)col * D + r : (size_t)r * D + col] : 0.f;
                    if constexpr (MOMENT)
                        T[j][a][i] = MODE == kMoment && order > 0 ? w.part_moments[part_at + (size_t)r * D + col] : 0.f;
                }

    const int64_t step = w.reverse ? -1 : 1;
    const int64_t first = w.reverse ? row0 + (int64_t)count - 1 : row0;
    const Rows<C> kr = Rows<C>::make(row_of(w.k, b, first, h), step * w.k.s.row);
    const Rows<C> vr = Rows<C>::make(row_of(w.v, b, first, h) + (size_t)col0 * ES, step * w.v.s.row);
    Rows<C> qr = kr, outr = kr;                                            // of q, and of o or the gradient
    if constexpr (OUT) qr = Rows<C>::make(row_of(w.q, b, first, h), step * w.q.s.row);
    if constexpr (MODE == kOut) outr = Rows<C>::make(row_of(w.o, b, first, h), step * w.o.s.row);
    if constexpr (MODE == kMoment) outr = Rows<C>::make(row_of(w.grad, b, first, h), step * w.grad.s.row);
    Fetch<C, D, THREADS, BF16> fq, fk;
    Fetch<C, W, THREADS, BF16> fv;
    auto fetch = [&](int done) __attribute__((always_inline)) {
        fk.load(kr, done, count);
        fv.load(vr, done, count);
        if constexpr (OUT) fq.load(qr, done, count);
    };
    if (count) fetch(0);
    // places in the images: chunk g4 of row c16; this lane's four elements of row 8 g4 + c16 / 4 for K^T (columns
    // 8 (c16 % 4) ..) and for V (this wave's columns, 4 (c16 % 4) ..)
    const int trow = 8 * g4 + (c16 >> 2);
    uint32_t row_at = c16 * D + ((g4 ^ swizzle<D>(c16)) << 3), kt_at = trow * D + (((c16 & 3) ^ swizzle<D>(trow)) << 3),
             v_at = trow * W + (((2 * wave + (c16 >> 1 & 1)) ^ swizzle<W>(trow)) << 3) + 4 * (c16 & 1);
    const float gfull = expm1f(lg * (float)C);
    double z = 0.;          // terms of either sign over thousands of rows

    for (int done = 0; done < count; done += C) {
        const int cnt = count - done < C ? count - done : C;
        // what follows from these is formed anew for every chunk, not kept in registers by the dozen
        asm volatile("" : "+v"(row_at), "+v"(kt_at), "+v"(v_at));
        const int ln = fresh_tid() & 63, c16 = ln & 15, g4 = ln >> 4;
        fk.store(ki);
        fv.store(vi);
        if constexpr (OUT) fq.store(qi);
        if (cnt < C) {
            __syncthreads();
            fk.clear(ki, cnt);
            fv.clear(vi, cnt);
            if constexpr (OUT) fq.clear(qi, cnt);
        }
        __syncthreads();

        v4f O[NC];
        // Q S, times g^(i+pre)
        auto from_state = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < NC; ++t) O[t] = v4f{0.f, 0.f, 0.f, 0.f};
            v4f R[NC];
            if constexpr (MOMENT)
#pragma unroll
                    for (int t = 0; t < NC; ++t) R[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                v8bf s[TP], m[TP];
                    v8f x;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = S[j][e / 4][e % 4];
                    split<TP>(x, s);
                    if constexpr (MOMENT) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = T[j][e / 4][e % 4];
                        split<TP>(x, m);
                    }
                v8bf q[NC][NT];
#pragma unroll
                for (int t = 0; t < NC; ++t)
#pragma unroll
                    for (int k = 0; k < NT; ++k) q[t][k] = lds8(qi + (k * C + 16 * t) * D + (row_at ^ j << 5));
                products(s, q, O);
                if constexpr (MOMENT) products(m, q, R);
                // or the operands of all steps are read at once, and registers spilled
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int t = 0; t < NC; ++t) {
                const int i = 16 * t + c16;
                const float x = pw[i + pre];
                    if constexpr (MOMENT) O[t] = (R[t] + (float)(i + 1) * O[t]) * x;
                    else O[t] *= x;
            }
        };

        if constexpr (OUT) {
            // P^T, rows s, columns t, in tiles of 16: those up to the diagonal go round the waves
            auto tile = [&](int sb, int tb) __attribute__((always_inline)) {
                v4f p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    v8bf a[NT], q[NT];
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        a[k] = lds8(ki + (k * C + 16 * sb) * D + (row_at ^ j << 5));
                        q[k] = lds8(qi + (k * C + 16 * tb) * D + (row_at ^ j << 5));
                    }
                    p = product<NT, NT>(a, q, p);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ago = 16 * (tb - sb) + c16 - 4 * g4 - i;
                    const float wgt = MOMENT ? po[ago] * (float)ago : po[ago];
                    p[i] = ago < 0 ? 0.f : p[i] * wgt;          // not 0 * p: rows after t may hold anything
                }
#pragma unroll
                for (int k = 0; k < TP; ++k) {
                    const v4bf term = __builtin_convertvector(p, v4bf);
                    *reinterpret_cast<v4bf*>(pi + (k * C + 16 * tb + c16) * LP + 16 * sb + 4 * g4) = term;
                    if (k + 1 < TP) {
                        const uint2 u = __builtin_bit_cast(uint2, term);
                        p -= v4f{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
                    }
                }
            };
#pragma unroll 1
            for (int n = wave; n < NC * (NC + 1) / 2; n += NW) {
                const int tb = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
                tile(n - tb * (tb + 1) / 2, tb);
            }
            from_state();
            __syncthreads();
        }

        // V's rows 32 kk + 8 g4 + (0..7) of this wave's columns
        auto column = [&](int kk, v8bf (&v)[NT]) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < NT; ++k)
                v[k] = lds_turned<W>(vi + (k * C + 32 * kk) * W, v_at);
        };
        if constexpr (OUT) {
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                v8bf v[NT];
                column(kk, v);
                // rows 32 kk of V meet the tiles of P from 2 kk on
                v8bf p[2][TP];
#pragma unroll
                for (int t2 = kk; t2 < NK; ++t2) {
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int k = 0; k < TP; ++k) p[y][k] = lds8(pi + (k * C + 32 * t2 + 16 * y + c16) * LP + 32 * kk + 8 * g4);
                    v4f o[2] = {O[2 * t2], O[2 * t2 + 1]};
                    products(v, p, o);
                    O[2 * t2] = o[0], O[2 * t2 + 1] = o[1];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // A row of V that is not finite reaches the rows before it here, as 0 * V.  Then the products are taken again with
            // zeros for such values, and a column that has met one by row t is NaN from there on: the same products count them.
            // The last tile meets all rows of V.
            float probe = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) probe = fmaf(O[NC - 1][i], 0.f, probe);
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_expect(__any(probe != 0.f), 0)) {
                from_state();
#pragma unroll
                for (int t = 0; t < NC; ++t) {
                        v4f met = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int kk = 0; kk <= t / 2; ++kk) {
                            v8bf v[NT], p[TP], bad, upto;
                            column(kk, v);
#pragma unroll
                            for (int k = 0; k < TP; ++k) p[k] = lds8(pi + (k * C + 16 * t + c16) * LP + 32 * kk + 8 * g4);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                bool fine = true;
#pragma unroll
                                for (int k = 0; k < NT; ++k) {
                                    const bool f = finite32((float)v[k][e]);
                                    fine = fine && f;
                                    if (!f) v[k][e] = (__bf16)0.f;
                                }
                                bad[e] = fine ? (__bf16)0.f : (__bf16)1.f;
                                upto[e] = 32 * kk + 8 * g4 + e <= 16 * t + c16 ? (__bf16)1.f : (__bf16)0.f;
                            }
                            O[t] = product<NT, TP>(v, p, O[t]);
                            met = mfma(bad, upto, met);
                            __builtin_amdgcn_sched_barrier(0);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (met[i] != 0.f) O[t][i] = __builtin_nanf("");
                }
            }
            float zc = 0.f;
            const char* const outp = outr.at(done);
#pragma unroll
            for (int t = 0; t < NC; ++t) {
                const int i = 16 * t + c16;
                const uint32_t at = outr.off(i) + (mycol + 4 * g4) * (BF16 && !(MODE == kOut && w.o_float) ? 2 : 4);
                if (i < cnt) {
                    const v4f x = O[t];
                    if constexpr (MODE == kMoment) {
                        v4f d;
                        if constexpr (BF16) {
                            const uint2 u = *reinterpret_cast<const uint2*>(outp + at);
                            d = v4f{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
                        } else {
                            d = *reinterpret_cast<const v4f*>(outp + at);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) zc = fmaf(x[e], d[e], zc);
                    } else {
                        char* p = const_cast<char*>(outp + at);
                        if (BF16 && !w.o_float) *reinterpret_cast<v4bf*>(p) = __builtin_convertvector(x, v4bf);
                        else *reinterpret_cast<v4f*>(p) = x;
                    }
                }
            }
            if constexpr (MODE == kMoment) z += zc;
        }

        // the next rows are on their way while S is updated, where registers are free for them
        fetch(done + C);

        // S <- g^cnt S + K^T diag(g^(cnt-pre-j)) V, and T <- g^cnt (T + cnt S) + ... with the weights' derivative
        const float gc = cnt == C ? gfull : expm1f(lg * (float)cnt);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (MOMENT) {
                            const float x = fmaf((float)cnt, S[j][a][i], T[j][a][i]);
                            T[j][a][i] = fmaf(x, gc, x);
                        }
                        S[j][a][i] = fmaf(S[j][a][i], gc, S[j][a][i]);
                    }
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            v8bf v[3], m[3];
                v8bf raw[NT];
                column(kk, raw);
                v8f x = widen(raw[NT - 1]), y;
#pragma unroll
                for (int k = NT - 2; k >= 0; --k) x += widen(raw[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int left = cnt - pre - (32 * kk + 8 * g4 + e);
                    x[e] *= pk[left];
                    if constexpr (MOMENT) y[e] = x[e] * (float)left;
                }
                split<3>(x, v);
                if constexpr (MOMENT) split<3>(y, m);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                v8bf kt[2][NT];
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int k = 0; k < NT; ++k)
                        kt[a][k] = lds_turned<D>(ki + (k * C + 32 * kk) * D + 4 * a, kt_at ^ j << 5);
                products(kt, v, S[j]);
                if constexpr (MOMENT) products(kt, m, T[j]);
                if (j & 1) __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();        // everybody is done with the images
    }

    if constexpr (MODE == kOut) {
        // rows of this part that are not valid
        const int es = BF16 && !w.o_float ? 2 : 4, vecs = W * es / 16;
        for (int i = tid; i < (rows - count) * vecs; i += THREADS) {
            char* p = row_of(w.o, b, row0 + count + i / vecs, h) + (size_t)col0 * es + i % vecs * 16;
            *reinterpret_cast<v4u*>(p) = v4u{0u, 0u, 0u, 0u};
        }
    }
    float* to = nullptr;
    if (STATES) to = w.parts + (((size_t)b * w.H + h) * (w.nparts - 1) + order) * D * D;
    else if (MODE != kMoment && order == w.nparts - 1 && w.state_out) to = w.state_out + state_at;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const size_t at = (size_t)(32 * j + 8 * g4 + 4 * a + i) * D + mycol + c16;
                    if (to) to[at] = S[j][a][i];
                    if constexpr (MODE == kMomentState)
                        w.part_moments[(((size_t)b * w.H + h) * (w.nparts - 1) + order) * D * D + at] = T[j][a][i];
                    if constexpr (MODE == kMoment)
                        if (order == w.nparts - 1 && w.grad_state) z += (double)w.grad_state[state_at + at] * T[j][a][i];
                }
    if constexpr (MODE == kMoment) {
#pragma unroll
        for (int m = 32; m; m >>= 1) z += __shfl_xor(z, m);
        __syncthreads();        // the images are done with, and a part without rows has not come by a barrier
        double* const sum = reinterpret_cast<double*>(lds);
        if (lane == 0) sum[wave] = z;
        __syncthreads();
        if (tid == 0) {
            for (int i = 1; i < NW; ++i) z += sum[i];
            w.moments[(((size_t)b * w.H + h) * w.nparts + part) * NS + slice] = z;
        }
    }
}

// parts[o] holds the state behind part o of the walk from a zero state; it becomes the state behind parts 0 .. o from
// state_in, which is the start of part o + 1.
template <bool MOMENT>
__global__ __launch_bounds__(kJoinThreads) void join_parts_kernel(Walk w) {
    const int DD = w.D * w.D;
    const size_t i = (size_t)blockIdx.x * kJoinThreads + threadIdx.x;   // an element of a state
    const int e = (int)(i % DD), h = (int)(i / DD % w.H), b = (int)(i / DD / w.H);
    const int len = user_len(w.lengths, b, w.N);
    const float lg = w.log_decay[h];
    const size_t bh = (size_t)b * w.H + h;
    float s = 0.f, t = 0.f;
    if (w.state_in) s = w.state_in[bh * DD + (w.in_turned ? (e % w.D) * w.D + e / w.D : e)];
    float* p = w.parts + bh * (w.nparts - 1) * DD + e;
    float* pm = MOMENT ? w.part_moments + bh * (w.nparts - 1) * DD + e : nullptr;
    for (int o = 0; o + 1 < w.nparts; ++o) {
        const int part = w.reverse ? w.nparts - 1 - o : o, row0 = part * w.part_rows;
        const int rows = w.N - row0 < w.part_rows ? w.N - row0 : w.part_rows;
        const int count = len - row0 < 0 ? 0 : (len - row0 < rows ? len - row0 : rows);
        const float g = expm1f(lg * (float)count), gc = count ? g : 0.f;      // log g may be -infinity
        if constexpr (MOMENT) {
            const float x = fmaf((float)count, s, t);
            t = fmaf(x, gc, x) + pm[(size_t)o * DD];
            pm[(size_t)o * DD] = t;
        }
        s = fmaf(s, gc, s) + p[(size_t)o * DD];
        p[(size_t)o * DD] = s;
    }
}

template <int D, bool BF16, int MODE>
hipError_t launch(const Walk& w, int parts, hipStream_t stream) {
    using F = ChunkCfg<D, BF16, is_moment(MODE)>;
    auto kern = decay_chunk_kernel<D, BF16, MODE>;
    constexpr size_t bytes = F::lds_bytes(is_out(MODE));
    hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), bytes);
    if (e != hipSuccess) return e;
    const int share = w.k.share;
    const int64_t groups = (int64_t)w.B * w.H * parts / share;
    const int64_t blocks = (groups + 7) / 8 * 8 * share * (D / F::W);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(F::kThreads), bytes, stream, w);
    return hipGetLastError();
}

template <int D, bool BF16>
hipError_t walk(const Walk& w, hipStream_t stream) {
    hipError_t e;
    if (w.nparts > 1) {
        e = w.moment ? launch<D, BF16, kMomentState>(w, w.nparts - 1, stream) : launch<D, BF16, kState>(w, w.nparts - 1, stream);
        if (e != hipSuccess) return e;
        const dim3 grid((unsigned)((size_t)w.B * w.H * D * D / kJoinThreads));
        if (w.moment) hipLaunchKernelGGL(join_parts_kernel<true>, grid, dim3(kJoinThreads), 0, stream, w);
        else hipLaunchKernelGGL(join_parts_kernel<false>, grid, dim3(kJoinThreads), 0, stream, w);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!w.moment && !w.o.data) return launch<D, BF16, kLast>(w, 1, stream);
    return w.moment ? launch<D, BF16, kMoment>(w, w.nparts, stream) : launch<D, BF16, kOut>(w, w.nparts, stream);
}

}  // namespace

hipError_t launch_decay_chunks(const Walk& w, hipStream_t stream) {
    switch (w.D) {
        case 64: return w.bf16 ? walk<64, true>(w, stream) : walk<64, false>(w, stream);
        case 128: return w.bf16 ? walk<128, true>(w, stream) : walk<128, false>(w, stream);
        case 256: return w.bf16 ? walk<256, true>(w, stream) : walk<256, false>(w, stream);
        default: return hipErrorInvalidValue;
    }
}

int moment_slices(int D) { return D < 128 ? 1 : D / 128; }

// Parts that a sequence is cut into.  Two workgroups of the kernel fit a compute unit, so 512 fill the GPU; every part but
// the last reads K and V once more, so there are no more than that takes, and none below eight chunks of 64 rows.
DecayParts decay_parts(int B, int N, int H, int D) {
    const int slices = moment_slices(D);
    const int64_t have = (int64_t)B * H * slices;
    int64_t n = (512 + have - 1) / have;
    const int64_t most = N / 512;
    if (n > most) n = most;
    if (n < 1) n = 1;
    const int rows = (int)((((int64_t)N + n - 1) / n + 63) / 64 * 64);
    return {ceil_div(N, rows), rows};
}

}  // namespace solar
