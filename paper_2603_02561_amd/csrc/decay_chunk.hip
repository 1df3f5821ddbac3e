// Linear attention with a decay for each head, in chunks of C rows on the matrix unit.  With local rows i = 0 .. C-1 and
// the state S in front of them (sequence.h: pre = 1 forward, 0 in reverse):
//   O = diag(g^(i+pre)) Q S + ((Q K^T) o M) V,   M_ij = g^(i-j) for j <= i,  0 else
//   S <- g^C S + K^T diag(g^(C-pre-j)) V
// A workgroup holds W columns of S in registers, a share per wave, and walks over the rows of one part of one user's sequence
// for one head.  Everything is formed transposed (O^T = S^T Q^T + V^T P^T): a lane's entries of S, eight
// of one column, are then an operand of the matrix instruction as they stand, and so are K^T and V from the transposing LDS
// read; only P = Q K^T o M goes through LDS, each wave forming a share of it.
//
// Precision.  Sums and S are float.  The matrix unit takes bf16, so a float operand is cut into bf16 terms that add up to it:
// three, which hold all 24 bits.  Products of two such operands (float inputs) take the six pairs of terms above 2^-24.  The error
// of a rounded g^C does not add up over the chunks, nor is a small one lost (Kept, sequence.h).
//
// What bounds it: not memory (64 users of 10000 rows at D = 128: 655 MB, 130 us at the rate of a copy; 226 to 235 us) but the
// instructions of a chunk and the waits between them.  Per wave and chunk there are 240 matrix instructions, 3840 cycles, and 1020 of the
// vector ALU, 4070, most of them the terms of S, P and the weighted V.  By the counters the matrix unit is busy 34 % of the time and the
// vector ALU 36 %, both at once only 6 %; LDS 32 %.  A wave spends 23 % of its time waiting for LDS, memory or the others: there are
// three barriers a chunk, between which the waves of a workgroup run the same phase, and two waves to a SIMD.  With log g's derivative
// there is one workgroup to a compute unit: matrix unit 27 %, vector ALU 32 %, both 5 %, and 53 % of a wave's time is waiting.
// In that form registers are spilled: 37 at D = 128 and 274 at 256, 63 and 540 for float rows; the others spill a few at D = 256 with
// float rows, and outside the usual path at 128.  S and P in two terms (16 bits) took 8 to 10 % less.  Tried without gain, with those: sixteen
// columns per wave with twice the waves (twice the reads of Q and K from LDS: 186 us against 188), loads issued earlier in the
// chunk, vector instructions between the matrix instructions by schedule groups (+3 %).
#include "kernels.h"
#include "sequence.h"

namespace solar {

namespace {

constexpr int kJoinThreads = 256;

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

template <int D, bool BF16, bool MOMENT>
struct ChunkCfg {
    static constexpr int C = BF16 && D <= 128 ? 64 : 32;                // rows of a chunk
    static constexpr int W = D == 64 || (MOMENT && D == 256) ? 64 : 128;    // columns of S per workgroup
    // Tiles of 16 columns per wave.  Every wave reads all of Q and K from LDS, so two tiles halve that: at D = 128 the registers
    // of two waves per SIMD hold them.
    static constexpr int NB = D == 128 && !MOMENT ? 2 : 1;
    static constexpr int kThreads = 4 * W / NB;
    static constexpr int NT = BF16 ? 1 : 3;                             // terms of an input
    static constexpr int TP = 3;                                        // terms of P and S where they meet V and Q
    static constexpr int LP = C + 8;                                    // bf16 per row of P's images
    static constexpr int kQ = NT * C * D, kV = NT * C * W, kP = (TP + (MOMENT ? 3 : 0)) * C * LP;
    static constexpr int kTables = 4 * C + 3 + 16;
    static constexpr size_t lds_bytes(bool out) { return 2 * (size_t)(kQ + kV + (out ? kQ + kP : 0)) + 4 * kTables; }
    // waves per SIMD that the registers are shared out for
    static constexpr int waves(bool out) { return MOMENT ? 2 : out ? (D == 64 ? 3 : 2) : (D == 128 ? 3 : 4); }
};

typedef float v8f __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// x minus one of a pair of bf16: in one instruction, and exact where that is x rounded or cut.  The pair (-1, 0) comes from a register:
// as an inline constant the instruction reads -1.0 as (0, -1).
__device__ __forceinline__ float minus(float x, v2bf pair, int which) {
    uint32_t one = which ? 0xbf800000u : 0x0000bf80u;
    asm("" : "+s"(one));
    return __builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(v2bf, one), x, false);
}

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

// The first terms of N floats: bf16 of which x - term is finite wherever x is, also above the largest bf16.  Against rows of
// bf16 (CUT) the upper half of x: what is left has 16 bits, two terms.  Float rows drop the smallest pairs of terms, which the cut
// would make larger: there it is x rounded, the largest bf16 at most (one instruction more: 12 ragged users of 3001 rows 71 -> 73 us).
template <bool CUT, int N>
__device__ __forceinline__ auto first_term(float __attribute__((ext_vector_type(N))) x) {
    typedef __bf16 bf __attribute__((ext_vector_type(N)));
    if constexpr (CUT) {
        uint32_t __attribute__((ext_vector_type(N / 2))) u;
#pragma unroll
        for (int e = 0; e < N / 2; ++e)
            u[e] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302u);
        return __builtin_bit_cast(bf, u);
    } else {
        constexpr float kTop = 3.38953139e38f;      // the largest bf16
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e], -kTop, kTop);
        return __builtin_convertvector(x, bf);
    }
}

// x = the sum of its terms, to 8 bits each.  A neighbour that is not finite makes both of a pair NaN.
template <bool CUT, int T>
__device__ __forceinline__ void split(v8f x, v8bf (&s)[T]) {
#pragma unroll
    for (int k = 0; k < T; ++k) {
        s[k] = k ? __builtin_convertvector(x, v8bf) : first_term<CUT, 8>(x);
        if (k + 1 < T)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = minus(x[e], v2bf{s[k][e & ~1], s[k][e | 1]}, e & 1);
    }
}

// The same where neighbours must not meet (columns of an input), or x is kept: the instruction above overwrites it.
template <bool CUT, int T>
__device__ __forceinline__ void split_apart(v8f x, v8bf (&s)[T]) {
#pragma unroll
    for (int k = 0; k < T; ++k) {
        s[k] = k ? __builtin_convertvector(x, v8bf) : first_term<CUT, 8>(x);
        if (k + 1 < T) x -= widen(s[k]);
    }
}

__device__ __forceinline__ v4f mfma(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// c[m][n] + a[m] b[n] over the pairs of terms that matter, the small ones first; products that follow one another are
// independent.
template <int M, int N, int TA, int TB>
__device__ __forceinline__ void products(const v8bf (&a)[M][TA], const v8bf (&b)[N][TB], v4f (&c)[M][N]) {
    constexpr int T = TA > TB ? TA : TB;
#pragma unroll
    for (int sum = T - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < TA; ++i)
            if (sum - i >= 0 && sum - i < TB)
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int n = 0; n < N; ++n) c[m][n] = mfma(a[m][i], b[n][sum - i], c[m][n]);
}

// The images of rows in LDS have no padding: chunks of eight elements lie in row `row` at the place (chunk ^ swizzle(row)).  Then
// neither the reads of one chunk from sixteen rows, nor the transposing reads of four rows, nor the stores of whole rows meet
// in a bank (a row is 32, 64 or 128 of the 64 banks long).  The counters put 41 % of the busy time of LDS down to conflicts all the same,
// of accesses that they do not name.
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
    uint32_t apart;         // |step| / 16, below 2^20 by the host's checks
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
        constexpr int APART = THREADS / PER;        // rows; their chunks have one place in all of them where it is a multiple of 16
        const int place = (c ^ swizzle<COLS>(i0)) << 3;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int i = i0 + u * APART;
            __bf16* to = img + i * COLS + (APART % 16 ? (c ^ swizzle<COLS>(i)) << 3 : place);
            if constexpr (BF16) {
                *reinterpret_cast<v4u*>(to) = x[u][0];
            } else {
                v8f f;
                v8bf s[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(x[u][e / 4][e % 4]);
                split_apart<false>(f, s);
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

template <int K>
struct Number {
    static constexpr int value = K;
};

// c[nb][a] + k[a] v[nb]: the same with the roles of rows and columns of c exchanged
template <int A, int NB, int TA, int TB>
__device__ __forceinline__ void update(const v8bf (&k)[A][TA], const v8bf (&v)[NB][TB], v4f (&c)[NB][A]) {
    constexpr int T = TA > TB ? TA : TB;
#pragma unroll
    for (int sum = T - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < TA; ++i)
            if (sum - i >= 0 && sum - i < TB)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int a = 0; a < A; ++a) c[nb][a] = mfma(k[a][i], v[nb][sum - i], c[nb][a]);
}

// kOut: outputs; kState: the state behind each piece of the parts but the last, from a zero state, into its place in w.parts;
// kMoment: outputs, and their derivative by log g summed against w.grad; kMomentState: kState, and the derivative of these
// states; kLast: the state behind the last part, where nobody wants outputs.
enum { kOut, kState, kMoment, kMomentState, kLast };
constexpr bool is_moment(int mode) { return mode == kMoment || mode == kMomentState; }
constexpr bool is_out(int mode) { return mode == kOut || mode == kMoment; }

template <int D, bool BF16, int MODE>
__global__ __launch_bounds__((ChunkCfg<D, BF16, is_moment(MODE)>::kThreads), (ChunkCfg<D, BF16, is_moment(MODE)>::waves(is_out(MODE)))) void
decay_chunk_kernel(Walks ws) {
    constexpr bool MOMENT = is_moment(MODE), OUT = is_out(MODE), STATES = MODE == kState || MODE == kMomentState;
    using F = ChunkCfg<D, BF16, MOMENT>;
    constexpr int C = F::C, W = F::W, NB = F::NB, THREADS = F::kThreads, NT = F::NT, TP = F::TP, LP = F::LP;
    constexpr int NW = THREADS / 64, NS = D / W, NJ = D / 32, NC = C / 16, NK = C / 32, ES = BF16 ? 2 : 4;
    constexpr int TM = MOMENT ? 3 : 1, MB = MOMENT ? NB : 1, MJ = MOMENT ? NJ : 1;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __bf16* const ki = reinterpret_cast<__bf16*>(lds);                  // [NT][C][D]
    __bf16* const vi = ki + F::kQ;                                      // [NT][C][W]
    __bf16* const qi = vi + F::kV;                                      // [NT][C][D]
    __bf16* const pi = qi + (OUT ? F::kQ : 0);                          // [TP][C][LP]: row t, column s
    __bf16* const mi = pi + TP * C * LP;                                // [3][C][LP] with MOMENT: the same, times t - s
    float* const pw = reinterpret_cast<float*>(pi + (OUT ? F::kP : 0)); // o_scale g^n, n = 0 .. C
    float* const pk = pw + C + 1 + C;                                   // kv_scale g^n, n = -C .. C, zero below 0
    float* const po = pk + C + 1 + 16;                                  // o_scale kv_scale g^n, n = -16 .. C, zero below 0

    // Slices and walks of one part, and heads that share K and V, run on one XCD (workgroups go to the eight in turn), where
    // they find each other's rows in its L2.
    const int turn = blockIdx.x >> 3, slice = turn % NS, k0 = turn / NS / ws.count;
    const Walk& w = ws.walk[turn / NS % ws.count];
    // the states in front of the last part are formed in shorter pieces, w.pieces of them to a part
    const int pieces = STATES ? w.pieces : 1, part_rows = STATES ? w.part_rows / w.pieces : w.part_rows;
    const int share = ws.walk[0].k.share, nparts = MODE == kLast ? 1 : STATES ? (w.nparts - 1) * pieces : w.nparts;
    const int64_t unit = (int64_t)(k0 / share * 8 + (blockIdx.x & 7)) * share + k0 % share;
    if (unit >= (int64_t)w.B * w.H * nparts) return;
    const int h = (int)(unit % w.H), b = (int)(unit / w.H / nparts);
    // in the order of the walk; the last part's state is nobody's start
    const int order = MODE == kLast ? w.nparts - 1 : (int)(unit / w.H % nparts), part = w.reverse ? w.nparts * pieces - 1 - order : order;

    const int tid = threadIdx.x, wave = tid >> 6;
    const int len = user_len(w.lengths, b, w.N);
    const int row0 = part * part_rows;
    const int rows = w.N - row0 < part_rows ? w.N - row0 : part_rows;   // below 0 for a piece past the end
    const int count = len - row0 < 0 ? 0 : (len - row0 < rows ? len - row0 : rows);
    const int pre = w.reverse ? 0 : 1;
    const float lg = w.log_decay[h];
    const int col0 = slice * W, mycol = col0 + wave * 16 * NB;          // the workgroup's columns of S, and the wave's

    for (int n = tid; n <= C; n += THREADS) {
        const float x = n ? expf(lg * (float)n) : 1.f;                  // log g may be -infinity
        pw[n] = w.o_scale * x;
        pk[n] = w.kv_scale * x;
        po[n] = w.o_scale * w.kv_scale * x;
        if (n) pk[-n] = 0.f;
        if (n && n <= 16) po[-n] = 0.f;
    }
    if constexpr (OUT) {
        // P above the diagonal, as far as the 32 rows of V that a product takes reach: zero, and never written again
        for (int n = tid; n < F::kP / LP * 2; n += THREADS) {
            const int t = n / 2 % C, k = n / 2 / C;
            if (!(t & 16)) *reinterpret_cast<v4u*>(pi + (k * C + t) * LP + (t & ~15) + 16 + 8 * (n & 1)) = v4u{0u, 0u, 0u, 0u};
        }
    }

    // S[j][nb][a]: rows 32 j + 8 g4 + 4 a + (0..3), column mycol + column(c16, nb) for lane 16 g4 + c16; T: its derivative.  With
    // two tiles their columns alternate in fours, so that a lane's entries of O^T are eight in a row.
    auto column = [](int c16, int nb) { return NB == 2 ? 8 * (c16 >> 2) + 4 * nb + (c16 & 3) : 16 * nb + c16; };
    v4f S[NJ][NB][2], T[MJ][MB][2];
    const size_t state_at = ((size_t)b * w.H + h) * D * D;
    const size_t part_at = (((size_t)b * w.H + h) * w.nparts * w.pieces + (STATES ? order : order * w.pieces)) * D * D;
    // f(the place of an entry in a state, the same in a transposed one, j, nb, a, i)
    auto entries = [&](auto f) __attribute__((always_inline)) {
        const int c16 = tid & 15, g4 = tid >> 4 & 3;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 32 * j + 8 * g4 + 4 * a + i, col = mycol + column(c16, nb);
                        f((uint32_t)(r * D + col), (uint32_t)(col * D + r), j, nb, a, i);
                    }
    };
    {
        // where there are parts all start from w.parts, the first too: state_out may be state_in
        const bool cut = w.nparts > 1;
        const float* start = STATES ? nullptr : cut ? w.parts + part_at : w.state_in ? w.state_in + state_at : nullptr;
        const bool turned = cut ? w.parts_turned : w.in_turned;
        entries([&](uint32_t at, uint32_t across, int j, int nb, int a, int i) {
            S[j][nb][a][i] = start ? start[turned ? across : at] : 0.f;
            if constexpr (MOMENT) T[j][nb][a][i] = cut && !STATES ? w.part_moments[part_at + at] : 0.f;
        });
    }

    const int64_t step = w.reverse ? -1 : 1;
    const int64_t first = w.reverse ? row0 + (int64_t)count - 1 : row0;
    const Rows<C> kr = Rows<C>::make(row_of(w.k, b, first, h), step * w.k.s.row);
    const Rows<C> vr = Rows<C>::make(row_of(w.v, b, first, h) + (size_t)col0 * ES, step * w.v.s.row);
    Rows<C> qr = kr, outr = kr, gradr = kr;
    if constexpr (OUT) {
        qr = Rows<C>::make(row_of(w.q, b, first, h), step * w.q.s.row);
        outr = Rows<C>::make(row_of(w.o, b, first, h), step * w.o.s.row);
    }
    if constexpr (MODE == kMoment) gradr = Rows<C>::make(row_of(w.grad, b, first, h), step * w.grad.s.row);
    Fetch<C, D, THREADS, BF16> fq, fk;
    Fetch<C, W, THREADS, BF16> fv;
    if (count) {
        fk.load(kr, 0, count);
        fv.load(vr, 0, count);
        if constexpr (OUT) fq.load(qr, 0, count);
    }

    // places in the images: chunk g4 of row c16; this lane's four elements of row 8 g4 + c16 / 4 for K^T (columns
    // 8 (c16 % 4) ..) and for V (this wave's columns, 8 (c16 % 4) .. or with one tile 4 (c16 % 4) ..)
    uint32_t row_at, kt_at, v_at;
    {
        const int c16 = tid & 15, g4 = tid >> 4 & 3, trow = 8 * g4 + (c16 >> 2);
        row_at = c16 * D + ((g4 ^ swizzle<D>(c16)) << 3);
        kt_at = trow * D + (((c16 & 3) ^ swizzle<D>(trow)) << 3);
        v_at = NB == 2 ? trow * W + (((4 * wave + (c16 & 3)) ^ swizzle<W>(trow)) << 3)
                       : trow * W + (((2 * wave + (c16 >> 1 & 1)) ^ swizzle<W>(trow)) << 3) + 4 * (c16 & 1);
    }
    // A chunk keeps (hi + lo) S: S is multiplied by a float, which also makes good what the ones before have rounded away (`owed`,
    // relative to S; one instruction an entry)
    struct Factor {
        float hi, lo;
    };
    auto uniform = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
    auto factor = [&](int n) {
        const Kept k = kept(lg, n);
        const float hi = k.near ? 1.f + k.by : k.by, y = hi - 1.f;
        return Factor{uniform(hi), uniform(k.near ? (1.f - (hi - y)) + (k.by - y) : 0.f)};
    };
    const Factor full = factor(C), last = factor(count % C);
    const float inverse = uniform(full.hi < 0.5f ? 0.f : 1.f / full.hi);
    float owed = 0.f;
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

        // V's rows 32 kk + 8 g4 + (0..7) of this wave's columns
        auto read_v = [&](int kk, v8bf (&v)[NB][NT]) __attribute__((always_inline)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int k = 0; k < NT; ++k) v[nb][k] = lds_turned<W>(vi + (k * C + 32 * kk) * W + 4 * nb, v_at);
        };
        v4f O[NB][NC], R[MB][MOMENT ? NC : 1];
        // O = Q S times g^(i+pre), R its derivative; the rows of Q are read a step ahead, or not (for fewer registers)
        auto from_state = [&](auto ahead) __attribute__((always_inline)) {
            constexpr int A = decltype(ahead)::value;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int t = 0; t < NC; ++t) {
                    O[nb][t] = v4f{0.f, 0.f, 0.f, 0.f};
                    if constexpr (MOMENT) R[nb][t] = v4f{0.f, 0.f, 0.f, 0.f};
                }
            v8bf q[1 + A][NC][NT];
            auto read_q = [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < NC; ++t)
#pragma unroll
                    for (int k = 0; k < NT; ++k) q[j & A][t][k] = lds8(qi + (k * C + 16 * t) * D + (row_at ^ (j << 5)));
            };
            if (A) read_q(0);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (!A) read_q(j);
                else if (j + 1 < NJ) read_q(j + 1);
                v8bf s[NB][TP];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    v8f x;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = S[j][nb][e / 4][e % 4];
                    split_apart<BF16>(x, s[nb]);
                }
                products(s, q[j & A], O);
                if constexpr (MOMENT) {
                    v8bf m[NB][3];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        v8f x;
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = T[j][nb][e / 4][e % 4];
                        split_apart<BF16>(x, m[nb]);
                    }
                    products(m, q[j & A], R);
                }
                // or the operands of all steps are read at once, and registers spilled
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int t = 0; t < NC; ++t) {
                const float x = pw[16 * t + c16 + pre];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (MOMENT) R[nb][t] = (R[nb][t] + (float)(16 * t + c16 + pre) * O[nb][t]) * x;
                    O[nb][t] *= x;
                }
            }
        };

        if constexpr (OUT) {
            // P^T, rows s, columns t, in tiles of 16: those up to the diagonal go round the waves, and every wave takes all of
            // its tiles at once (the last one twice where they do not come out even)
            constexpr int TILES = NC * (NC + 1) / 2, MINE = (TILES + NW - 1) / NW;
            int sb[MINE], tb[MINE];
            v4f p[MINE];
#pragma unroll
            for (int y = 0; y < MINE; ++y) {
                const int n = wave + y * NW < TILES ? wave + y * NW : TILES - 1;
                tb[y] = __builtin_amdgcn_readfirstlane(n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3);
                sb[y] = __builtin_amdgcn_readfirstlane(n) - tb[y] * (tb[y] + 1) / 2;
                p[y] = v4f{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
#pragma unroll
                for (int y = 0; y < MINE; ++y) {
                    v8bf a[1][NT], q[1][NT];
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        a[0][k] = lds8(ki + (k * C + 16 * sb[y]) * D + (row_at ^ (j << 5)));
                        q[0][k] = lds8(qi + (k * C + 16 * tb[y]) * D + (row_at ^ (j << 5)));
                    }
                    v4f c[1][1] = {{p[y]}};
                    products(a, q, c);
                    p[y] = c[0][0];
                }
                if (NT * MINE > 2 || (j & 1)) __builtin_amdgcn_sched_barrier(0);
            }
            // four entries of a column t, s = 4 g4 + (0..3), into images of K terms
            auto put = [&](v4f x, __bf16* to, auto terms) __attribute__((always_inline)) {
                constexpr int K = decltype(terms)::value;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const v4bf term = k ? __builtin_convertvector(x, v4bf) : first_term<BF16, 4>(x);
                    *reinterpret_cast<v4bf*>(to + k * C * LP) = term;
                    if (k + 1 < K)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = minus(x[i], v2bf{term[i & ~1], term[i | 1]}, i & 1);
                }
            };
            const int diagonal = c16 - 4 * g4;
#pragma unroll
            for (int y = 0; y < MINE; ++y) {
                const int to = (16 * tb[y] + c16) * LP + 16 * sb[y] + 4 * g4, ago = 16 * (tb[y] - sb[y]) + diagonal;
                v4f x = {po[ago], po[ago - 1], po[ago - 2], po[ago - 3]};
                asm volatile("" : "+v"(x));                 // or a branch goes round each of them
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = ago - i < 0 ? 0.f : p[y][i] * x[i];      // not 0 * p: rows after t may hold anything
                put(x, pi + to, Number<TP>());
                if constexpr (MOMENT) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] *= (float)(ago - i);
                    put(x, mi + to, Number<3>());
                }
            }
            from_state(Number<MOMENT ? 0 : 1>());
            __syncthreads();

            // tiles 2 t2 and 2 t2 + 1 of the columns of P's images, against 32 kk rows of V
            auto read_p = [&](const __bf16* img, int kk, int t2, auto& p) __attribute__((always_inline)) {
                constexpr int K = sizeof(p[0]) / sizeof(v8bf);
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int k = 0; k < K; ++k) p[y][k] = lds8(img + (k * C + 32 * t2 + 16 * y + c16) * LP + 32 * kk + 8 * g4);
            };
            auto add = [&](const auto& v, const auto& p, auto& to, int t2) __attribute__((always_inline)) {
                v4f o[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) o[nb][0] = to[nb][2 * t2], o[nb][1] = to[nb][2 * t2 + 1];
                products(v, p, o);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) to[nb][2 * t2] = o[nb][0], to[nb][2 * t2 + 1] = o[nb][1];
            };
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                v8bf v[NB][NT];
                read_v(kk, v);
#pragma unroll
                for (int t2 = kk; t2 < NK; ++t2) {
                    v8bf p[2][TP];
                    read_p(pi, kk, t2, p);
                    add(v, p, O, t2);
                    if constexpr (MOMENT) {
                        v8bf m[2][TM];
                        read_p(mi, kk, t2, m);
                        add(v, m, R, t2);
                    }
                }
                if (NT > 1 || MOMENT) __builtin_amdgcn_sched_barrier(0);
            }
            // A row of V that is not finite reaches the rows before it here, as 0 * V.  Then the products are taken again with
            // zeros for such values, and a column that has met one by row t is NaN from there on: the same products count them.
            // The last tile meets all rows of V.
            float probe = 0.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) probe = fmaf(O[nb][NC - 1][i], 0.f, probe);
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_expect(__any(probe != 0.f), 0)) {
                from_state(Number<0>());
#pragma unroll
                for (int t2 = 0; t2 < NK; ++t2) {
                    v4f met[NB][2];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) met[nb][0] = met[nb][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk <= t2; ++kk) {
                        v8bf v[NB][NT], bad[NB][1], p[2][TP], upto[2][1];
                        read_v(kk, v);
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                bool fine = true;
#pragma unroll
                                for (int k = 0; k < NT; ++k) {
                                    const bool f = finite32((float)v[nb][k][e]);
                                    fine = fine && f;
                                    if (!f) v[nb][k][e] = (__bf16)0.f;
                                }
                                bad[nb][0][e] = fine ? (__bf16)0.f : (__bf16)1.f;
                            }
                        read_p(pi, kk, t2, p);
                        add(v, p, O, t2);
                        if constexpr (MOMENT) {
                            v8bf m[2][TM];
                            read_p(mi, kk, t2, m);
                            add(v, m, R, t2);
                        }
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                upto[y][0][e] = 32 * kk + 8 * g4 + e <= 32 * t2 + 16 * y + c16 ? (__bf16)1.f : (__bf16)0.f;
                        products(bad, upto, met);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (met[nb][y][i] != 0.f) {
                                    O[nb][2 * t2 + y][i] = __builtin_nanf("");
                                    if constexpr (MOMENT) R[nb][2 * t2 + y][i] = __builtin_nanf("");
                                }
                }
            }
            float zc = 0.f;
            const char* const outp = outr.at(done);
            const char* const gradp = gradr.at(done);
#pragma unroll
            for (int t = 0; t < NC; ++t)
                if (16 * t + c16 < cnt) {
                    const bool o_float = !BF16 || w.o_float;
                    const int col = mycol + 4 * NB * g4;
                    char* const p = const_cast<char*>(outp) + (outr.off(16 * t + c16) + col * (o_float ? 4 : 2));
                    if (o_float) {
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) *reinterpret_cast<v4f*>(p + 16 * nb) = O[nb][t];
                    } else if constexpr (NB == 2) {
                        const v8f x = __builtin_shufflevector(O[0][t], O[NB - 1][t], 0, 1, 2, 3, 4, 5, 6, 7);
                        *reinterpret_cast<v8bf*>(p) = __builtin_convertvector(x, v8bf);
                    } else {
                        *reinterpret_cast<v4bf*>(p) = __builtin_convertvector(O[0][t], v4bf);
                    }
                    if constexpr (MODE == kMoment) {
                        static_assert(!MOMENT || NB == 1, "");
                        const char* q = gradp + (gradr.off(16 * t + c16) + col * ES);
                        v4f d;
                        if constexpr (BF16) {
                            const uint2 u = *reinterpret_cast<const uint2*>(q);
                            d = v4f{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
                        } else {
                            d = *reinterpret_cast<const v4f*>(q);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) zc = fmaf(R[0][t][e], d[e], zc);
                    }
                }
            if constexpr (MODE == kMoment) z += zc;
        }

        // the next rows are on their way while S is updated, where registers are free for them
        fk.load(kr, done + C, count);
        fv.load(vr, done + C, count);
        if constexpr (OUT) fq.load(qr, done + C, count);

        // S <- g^cnt S + K^T diag(g^(cnt-pre-j)) V, and T <- g^cnt (T + cnt S) + ... with the weights' derivative
        const Factor k = cnt == C ? full : last;
        const float fix = fmaf(owed, k.hi, k.lo), g = uniform(k.hi + fix);
        owed = uniform((fix - (g - k.hi)) * inverse);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (MOMENT) T[j][nb][a][i] = fmaf((float)cnt, S[j][nb][a][i], T[j][nb][a][i]) * g;
                        S[j][nb][a][i] *= g;
                    }
        if constexpr (MODE != kMoment) __builtin_amdgcn_sched_barrier(0);       // or registers are spilled
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            v8bf kt[2][2][NT];
            auto read_k = [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int k = 0; k < NT; ++k)
                        kt[j & 1][a][k] = lds_turned<D>(ki + (k * C + 32 * kk) * D + 4 * a, kt_at ^ (j << 5));
            };
            v8bf v[NB][3], m[MB][3], raw[NB][NT];
            read_v(kk, raw);
            read_k(0);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                v8f x = widen(raw[nb][NT - 1]);
#pragma unroll
                for (int k = NT - 2; k >= 0; --k) x += widen(raw[nb][k]);
                const int left = cnt - pre - (32 * kk + 8 * g4);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= pk[left - e];
                split<BF16>(x, v[nb]);
                if constexpr (MOMENT) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= (float)(left - e);
                    split<BF16>(x, m[nb]);
                }
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (j + 1 < NJ) read_k(j + 1);
                update(kt[j & 1], v, S[j]);
                if constexpr (MOMENT) update(kt[j & 1], m, T[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();        // everybody is done with the images
    }

    if constexpr (OUT) {
        // rows of this part that are not valid
        const int es = BF16 && !w.o_float ? 2 : 4, vecs = W * es / 16;
        for (int64_t i = tid; i < (int64_t)(rows - count) * vecs; i += THREADS) {
            char* p = row_of(w.o, b, row0 + count + i / vecs, h) + (size_t)col0 * es + i % vecs * 16;
            *reinterpret_cast<v4u*>(p) = v4u{0u, 0u, 0u, 0u};
        }
    }
    float* to = STATES ? w.parts + part_at : order == w.nparts - 1 && w.state_out ? w.state_out + state_at : nullptr;
    if (to) entries([&](uint32_t at, uint32_t, int j, int nb, int a, int i) { to[at] = S[j][nb][a][i]; });
    if constexpr (MODE == kMomentState)
        entries([&](uint32_t at, uint32_t, int j, int nb, int a, int i) {
            w.part_moments[part_at + at] = T[j][nb][a][i];
        });
    if constexpr (MODE == kMoment) {
        if (order == w.nparts - 1 && w.grad_state)
            entries([&](uint32_t at, uint32_t across, int j, int nb, int a, int i) {
                z += (double)w.grad_state[state_at + (w.in_turned ? across : at)] * T[j][nb][a][i];
            });
#pragma unroll
        for (int m = 32; m; m >>= 1) z += __shfl_xor(z, m);
        __syncthreads();        // the images are done with, and a part without rows has not come by a barrier
        double* const sum = reinterpret_cast<double*>(lds);
        if ((tid & 63) == 0) sum[wave] = z;
        __syncthreads();
        if (tid == 0) {
            for (int i = 1; i < NW; ++i) z += sum[i];
            w.moments[(((size_t)b * w.H + h) * w.nparts + part) * NS + slice] = z;
        }
    }
}

// parts[o] holds the state behind piece o of the walk from a zero state, for the pieces of all parts but the last; the first piece
// of every part, the last part's too, becomes the state that the part starts from.
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
    const int all = w.nparts * w.pieces, last = all - w.pieces, piece_rows = w.part_rows / w.pieces;
    float* p = w.parts + bh * all * DD + e;
    float* pm = MOMENT ? w.part_moments + bh * all * DD + e : nullptr;
    const Kept whole = kept(lg, piece_rows);
    for (int o = 0; o < last; ++o) {
        const int part = w.reverse ? all - 1 - o : o, row0 = part * piece_rows;
        const int rows = w.N - row0 < piece_rows ? w.N - row0 : piece_rows;
        const int count = len - row0 < 0 ? 0 : (len - row0 < rows ? len - row0 : rows);
        const Kept g = count == piece_rows ? whole : kept(lg, count);
        if constexpr (MOMENT) {
            const float add = pm[(size_t)o * DD], x = fmaf((float)count, s, t);
            if (o % w.pieces == 0) pm[(size_t)o * DD] = t;
            t = (count ? keep(x, g) : t) + add;
        }
        const float add = p[(size_t)o * DD];
        if (o % w.pieces == 0) p[(size_t)o * DD] = s;
        s = (count ? keep(s, g) : s) + add;
    }
    p[(size_t)last * DD] = s;
    if constexpr (MOMENT) pm[(size_t)last * DD] = t;
}

template <int D, bool BF16, int MODE>
hipError_t launch(const Walks& ws, int parts, hipStream_t stream) {
    using F = ChunkCfg<D, BF16, is_moment(MODE)>;
    auto kern = decay_chunk_kernel<D, BF16, MODE>;
    constexpr size_t bytes = F::lds_bytes(is_out(MODE));
    hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), bytes);
    if (e != hipSuccess) return e;
    const Walk& w = ws.walk[0];
    const int share = w.k.share;
    const int64_t groups = (int64_t)w.B * w.H * parts / share;
    const int64_t blocks = (groups + 7) / 8 * 8 * share * ws.count * (D / F::W);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(F::kThreads), bytes, stream, ws);
    return hipGetLastError();
}

template <int D, bool BF16>
hipError_t run(const Walks& ws, hipStream_t stream) {
    const Walk& w = ws.walk[0];
    hipError_t e;
    if (w.nparts > 1) {
        Walks one = ws;
        one.count = 1;
        e = w.moment ? launch<D, BF16, kMomentState>(one, (w.nparts - 1) * w.pieces, stream)
                     : launch<D, BF16, kState>(one, (w.nparts - 1) * w.pieces, stream);
        if (e != hipSuccess) return e;
        const dim3 grid((unsigned)((size_t)w.B * w.H * D * D / kJoinThreads));
        if (w.moment) hipLaunchKernelGGL(join_parts_kernel<true>, grid, dim3(kJoinThreads), 0, stream, w);
        else hipLaunchKernelGGL(join_parts_kernel<false>, grid, dim3(kJoinThreads), 0, stream, w);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!w.o.data) return launch<D, BF16, kLast>(ws, 1, stream);
    return w.moment ? launch<D, BF16, kMoment>(ws, w.nparts, stream) : launch<D, BF16, kOut>(ws, w.nparts, stream);
}

}  // namespace

hipError_t launch_decay_chunks(const Walks& ws, hipStream_t stream) {
    const Walk& w = ws.walk[0];
    switch (w.D) {
        case 64: return w.bf16 ? run<64, true>(ws, stream) : run<64, false>(ws, stream);
        case 128: return w.bf16 ? run<128, true>(ws, stream) : run<128, false>(ws, stream);
        case 256: return w.bf16 ? run<256, true>(ws, stream) : run<256, false>(ws, stream);
        default: return hipErrorInvalidValue;
    }
}

int moment_slices(int D) { return D == 256 ? 4 : 1; }

// Parts that a sequence is cut into.  Two workgroups of the kernel fit a compute unit, so 512 fill the GPU; every part but
// the last reads K and V once more, so there are no more than that takes, and none below 128 rows.  `walks` of them run in one
// launch.  The states in front of the last part are formed by one walk only; where its parts are few they are cut further, into
// up to four pieces of at least 256 rows (8 x 4096 rows of 16 heads at D = 128: 84 -> 42 us for 128 parts in four pieces).
DecayParts decay_parts(int B, int N, int H, int D, int walks) {
    const int64_t heads = (int64_t)B * H * (D == 256 ? 2 : 1), have = heads * walks;
    int64_t n = (512 + have - 1) / have;
    const int64_t most = N / 128;
    if (n > most) n = most;
    if (n < 2) return {1, (N + 63) / 64 * 64, 1};
    const int64_t rows = (N + n - 1) / n;
    int64_t pieces = 512 / (heads * (n - 1));
    if (pieces > 4) pieces = 4;
    if (pieces > rows / 256) pieces = rows / 256;
    if (pieces < 1) pieces = 1;
    const int64_t unit = 64 * pieces;
    const int part_rows = (int)((rows + unit - 1) / unit * unit);
    return {ceil_div(N, part_rows), part_rows, (int)pieces};
}

}  // namespace solar
