// C ABI of the sequence operators (rotary positions, linear attention with a decay, layer norm): argument validation on
// the host and launches on the caller's stream.  See include/solar.h.
#include "../../include/solar.h"

#include <cmath>
#include <limits.h>

#include <algorithm>
#include <utility>

#include "sequence.h"

namespace {

using namespace solar;

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// Most workgroups of 256 threads in a launch (the runtime counts threads in 32 bits).
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 1;

// A tensor of heads [B,N,heads,D] from its pointer and strides in elements (null: contiguous).  `written`: no two elements
// may share an address.
bool take(const void* p, const solar_strides* s, int B, int N, int heads, int D, size_t es, int share, bool written,
          Heads* out) {
    if (!p || misaligned(p, 16)) return false;
    int64_t st[3] = {(int64_t)N * heads * D, (int64_t)heads * D, D};
    if (s) { st[0] = s->batch; st[1] = s->row; st[2] = s->head; }
    const int64_t size[3] = {B, N, heads}, step = (int64_t)(16 / es);
    for (int i = 0; i < 3; ++i) {
        if (size[i] == 1) { st[i] = 0; continue; }       // never stepped along
        if (st[i] < 0 || st[i] % step || st[i] > ((int64_t)1 << 48)) return false;
    }
    if (written) {
        int order[3] = {0, 1, 2};
        std::sort(order, order + 3, [&](int a, int b) { return st[a] < st[b]; });
        int64_t extent = D;
        for (int i : order) {
            if (size[i] == 1) continue;
            if (st[i] < extent) return false;
            extent = st[i] * (size[i] - 1) + extent;
        }
    }
    out->data = const_cast<char*>(static_cast<const char*>(p));
    out->s = {st[0] * (int64_t)es, st[1] * (int64_t)es, st[2] * (int64_t)es};
    out->share = share;
    return true;
}

bool known(solar_dtype t) { return t == SOLAR_F32 || t == SOLAR_BF16; }

// The kernels of the decayed attention step through up to 64 rows with 32-bit offsets.
bool rows_near(const Heads& t) { return t.s.row < (1 << 24); }

solar_status check_decay(int B, int N, int H, int Hkv, int D, float scale, solar_dtype t) {
    if (B <= 0 || N <= 0 || H <= 0 || Hkv <= 0 || D <= 0 || !known(t) || H % Hkv || !std::isfinite(scale))
        return SOLAR_ERR_INVALID_ARG;
    if (D != 64 && D != 128 && D != 256) return SOLAR_ERR_UNSUPPORTED;
    if (N > 1 << 30) return SOLAR_ERR_UNSUPPORTED;
    // Workgroups of the row form go by users, heads and slices of 32 columns.  Those of the chunked form go by users and shared heads,
    // rounded up to a multiple of eight, times the heads that share one: B = 1 with one K head makes eight times H, at slices of at least
    // twice the columns and up to 512 threads: less than 2^32 threads too, the most that a launch takes.  Parts are only cut where
    // there are less than 512; the gradients' two walks run at once, but with shared heads H D <= 2^22.
    if ((int64_t)B * H * (D / 32) > kMaxBlocks / 4) return SOLAR_ERR_UNSUPPORTED;
    return SOLAR_OK;
}

struct DecayCarve {
    DecayParts cut;
    float *parts, *part_moments;    // [B,H,parts * pieces,D,D], none for one part
    float *dk, *dv;                 // [B,N,H,D] of every head, where heads share K and V
    double* moments;                // [B,H,parts,slices]
    size_t total;
};

DecayCarve carve_decay(void* ws, int B, int N, int H, int Hkv, int D, bool backward) {
    DecayCarve c = {};
    char* at = static_cast<char*>(ws);
    auto part = [&](size_t floats) {
        float* p = reinterpret_cast<float*>(at);
        at += align256(sizeof(float) * floats);
        return p;
    };
    if (!backward && N <= kDecayRows) return c;
    c.cut = decay_parts(B, N, H, D, backward ? 2 : 1);
    const size_t states = c.cut.parts > 1 ? (size_t)B * H * c.cut.parts * c.cut.pieces * D * D : 0;
    c.parts = part(states);
    if (backward) {
        const size_t shared = H != Hkv ? (size_t)B * N * H * D : 0;
        c.part_moments = part(states);
        c.dk = part(shared);
        c.dv = part(shared);
        c.moments = reinterpret_cast<double*>(part((size_t)2 * B * H * c.cut.parts * moment_slices(D)));
    }
    c.total = (size_t)(at - static_cast<char*>(ws));
    return c;
}

}  // namespace

extern "C" {

solar_status solar_rotary_frequencies(int rot, double base, solar_rotary_scaling scaling, double factor,
                                      int original_length, double turns_low, double turns_high, double* freq) {
    if (!freq || rot < 2 || rot % 2 || !(base > 0.) || !std::isfinite(base)) return SOLAR_ERR_INVALID_ARG;
    if (scaling < SOLAR_ROTARY_UNSCALED || scaling > SOLAR_ROTARY_BY_PARTS) return SOLAR_ERR_INVALID_ARG;
    if (scaling != SOLAR_ROTARY_UNSCALED && (!(factor > 0.) || !std::isfinite(factor))) return SOLAR_ERR_INVALID_ARG;
    if (scaling == SOLAR_ROTARY_BASE) {
        if (rot < 4) return SOLAR_ERR_INVALID_ARG;       // one frequency, of 1: no base to scale
        base *= std::pow(factor, (double)rot / (rot - 2));
    }
    if (scaling == SOLAR_ROTARY_BY_PARTS &&
        (original_length < 1 || !(turns_high > turns_low) || !std::isfinite(turns_low) || !std::isfinite(turns_high)))
        return SOLAR_ERR_INVALID_ARG;
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2. * i / rot);
        if (scaling == SOLAR_ROTARY_LINEAR) f /= factor;
        if (scaling == SOLAR_ROTARY_BY_PARTS) {
            const double turns = original_length * f * 0.15915494309189533577;
            double keep = (turns - turns_low) / (turns_high - turns_low);
            keep = keep < 0. ? 0. : keep > 1. ? 1. : keep;
            f *= keep + (1. - keep) / factor;
        }
        freq[i] = f;
    }
    return SOLAR_OK;
}

solar_status solar_rotary(const void* Q, const void* K, const int32_t* lengths, const int32_t* positions,
                          const double* freq, int B, int N, int H, int Hkv, int D, int rot, solar_rotary_layout layout,
                          int inverse, float amplitude, solar_dtype t, const solar_strides* strides, void* Qout,
                          void* Kout, void* stream) {
    if (!freq || misaligned(freq, 8) || B <= 0 || N <= 0 || H <= 0 || D <= 0 || rot < 2 || rot % 2 || rot > D || !known(t) ||
        !std::isfinite(amplitude))
        return SOLAR_ERR_INVALID_ARG;
    if (layout != SOLAR_ROTARY_HALF && layout != SOLAR_ROTARY_INTERLEAVED) return SOLAR_ERR_INVALID_ARG;
    if (!K != !Kout || (K && Hkv <= 0)) return SOLAR_ERR_INVALID_ARG;
    if (D % 8 || D > 512) return SOLAR_ERR_UNSUPPORTED;
    const size_t es = t == SOLAR_BF16 ? 2 : 4;
    Rotary r = {};
    if (!take(Q, strides, B, N, H, D, es, 1, false, &r.in[0]) ||
        !take(Qout, strides ? strides + 2 : nullptr, B, N, H, D, es, 1, true, &r.out[0]))
        return SOLAR_ERR_INVALID_ARG;
    r.in[1] = r.in[0];
    r.out[1] = r.out[0];
    if (K && (!take(K, strides ? strides + 1 : nullptr, B, N, Hkv, D, es, 1, false, &r.in[1]) ||
              !take(Kout, strides ? strides + 3 : nullptr, B, N, Hkv, D, es, 1, true, &r.out[1])))
        return SOLAR_ERR_INVALID_ARG;
    // in place only with the same places, and not one over the other
    for (int i = 0; i < (K ? 2 : 1); ++i)
        if (r.in[i].data == r.out[i].data && (r.in[i].s.batch != r.out[i].s.batch || r.in[i].s.row != r.out[i].s.row ||
                                              r.in[i].s.head != r.out[i].s.head))
            return SOLAR_ERR_INVALID_ARG;
    if (K && (Qout == K || Kout == Q || Qout == Kout)) return SOLAR_ERR_INVALID_ARG;
    if ((int64_t)B * N > kMaxBlocks * kRotaryRows || (int64_t)H + (K ? Hkv : 0) > 65536) return SOLAR_ERR_UNSUPPORTED;
    r.heads[0] = H;
    r.heads[1] = K ? Hkv : 0;
    r.lengths = lengths;
    r.positions = positions;
    r.freq = freq;
    r.B = B; r.N = N; r.D = D; r.rot = rot;
    r.interleaved = layout == SOLAR_ROTARY_INTERLEAVED;
    r.inverse = inverse != 0;
    r.bf16 = t == SOLAR_BF16;
    r.amplitude = amplitude;
    return launch_rotary(r, (hipStream_t)stream) == hipSuccess ? SOLAR_OK : SOLAR_ERR_HIP;
}

size_t solar_decay_workspace_bytes(int B, int N, int H, int Hkv, int D, solar_dtype t, int backward) {
    if (check_decay(B, N, H, Hkv, D, 1.f, t) != SOLAR_OK) return 0;
    return carve_decay(nullptr, B, N, H, Hkv, D, backward != 0).total;
}

solar_status solar_decay_attention(const void* Q, const void* K, const void* V, const float* log_decay,
                                   const int32_t* lengths, const float* state_in, int B, int N, int H, int Hkv, int D,
                                   float scale, solar_dtype t, const solar_strides* strides, void* O, float* state_out,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    const solar_status v = check_decay(B, N, H, Hkv, D, scale, t);
    if (v != SOLAR_OK) return v;
    if (!log_decay || !K || !V || (!O && !state_out) || (O && !Q)) return SOLAR_ERR_INVALID_ARG;
    if (misaligned(state_in, 16) || misaligned(state_out, 16)) return SOLAR_ERR_INVALID_ARG;
    if (O && (O == Q || O == K || O == V)) return SOLAR_ERR_INVALID_ARG;     // other workgroups still read what O's rows replace
    const size_t es = t == SOLAR_BF16 ? 2 : 4;
    const int share = H / Hkv;
    Walk w = {};
    if (!take(K, strides ? strides + 1 : nullptr, B, N, Hkv, D, es, share, false, &w.k) ||
        !take(V, strides ? strides + 2 : nullptr, B, N, Hkv, D, es, share, false, &w.v))
        return SOLAR_ERR_INVALID_ARG;
    if (O) {
        if (!take(Q, strides, B, N, H, D, es, 1, false, &w.q) ||
            !take(O, strides ? strides + 3 : nullptr, B, N, H, D, es, 1, true, &w.o))
            return SOLAR_ERR_INVALID_ARG;
    } else {
        w.q = w.k;
    }
    if (!rows_near(w.k) || !rows_near(w.v) || !rows_near(w.q) || !rows_near(w.o)) return SOLAR_ERR_UNSUPPORTED;
    const DecayCarve c = carve_decay(workspace, B, N, H, Hkv, D, false);
    if (c.total && (!workspace || workspace_bytes < c.total || misaligned(workspace, 256))) return SOLAR_ERR_WORKSPACE;
    w.lengths = lengths;
    w.log_decay = log_decay;
    w.state_in = state_in;
    w.state_out = state_out;
    w.B = B; w.N = N; w.H = H; w.D = D;
    w.o_scale = scale;
    w.kv_scale = 1.f;
    w.bf16 = t == SOLAR_BF16;
    w.nparts = c.cut.parts;
    w.part_rows = c.cut.rows;
    w.pieces = c.cut.pieces;
    w.parts = c.parts;
    const hipError_t e = N <= kDecayRows ? launch_decay_rows(w, (hipStream_t)stream)
                                         : launch_decay_chunks({{w}, 1}, (hipStream_t)stream);
    return e == hipSuccess ? SOLAR_OK : SOLAR_ERR_HIP;
}

solar_status solar_decay_attention_backward(const void* Q, const void* K, const void* V, const void* dO,
                                            const float* log_decay, const int32_t* lengths, const float* state_in,
                                            const float* dstate_out, int B, int N, int H, int Hkv, int D, float scale,
                                            solar_dtype t, const solar_strides* strides, void* dQ, void* dK, void* dV,
                                            float* dstate_in, float* dlog_decay, void* workspace,
                                            size_t workspace_bytes, void* stream) {
    const solar_status v = check_decay(B, N, H, Hkv, D, scale, t);
    if (v != SOLAR_OK) return v;
    if (!log_decay) return SOLAR_ERR_INVALID_ARG;
    if (misaligned(state_in, 16) || misaligned(dstate_out, 16) || misaligned(dstate_in, 16)) return SOLAR_ERR_INVALID_ARG;
    for (const void* out : {dQ, dK, dV})
        for (const void* in : {Q, K, V, dO})
            if (out == in) return SOLAR_ERR_INVALID_ARG;
    if (dQ == dK || dQ == dV || dK == dV || (dstate_in && (dstate_in == dstate_out || dstate_in == state_in)))
        return SOLAR_ERR_INVALID_ARG;
    const size_t es = t == SOLAR_BF16 ? 2 : 4;
    const int share = H / Hkv;
    auto at = [&](int i) { return strides ? strides + i : nullptr; };
    Heads q, k, vv, g, dq, dk, dv;
    if (!take(Q, at(0), B, N, H, D, es, 1, false, &q) || !take(K, at(1), B, N, Hkv, D, es, share, false, &k) ||
        !take(V, at(2), B, N, Hkv, D, es, share, false, &vv) || !take(dO, at(3), B, N, H, D, es, 1, false, &g) ||
        !take(dQ, at(4), B, N, H, D, es, 1, true, &dq) || !take(dK, at(5), B, N, Hkv, D, es, 1, true, &dk) ||
        !take(dV, at(6), B, N, Hkv, D, es, 1, true, &dv))
        return SOLAR_ERR_INVALID_ARG;
    for (const Heads& x : {q, k, vv, g, dq, dk, dv})
        if (!rows_near(x)) return SOLAR_ERR_UNSUPPORTED;
    // rows of the float work arrays, and a thread for every four columns of their sums
    if (share > 1 && ((int64_t)H * D > 1 << 22 || (int64_t)B * N * Hkv * (D / 4) > kMaxBlocks * 256)) return SOLAR_ERR_UNSUPPORTED;
    const DecayCarve c = carve_decay(workspace, B, N, H, Hkv, D, true);
    if (c.total && (!workspace || workspace_bytes < c.total || misaligned(workspace, 256))) return SOLAR_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    Walk w = {};
    w.lengths = lengths;
    w.log_decay = log_decay;
    w.B = B; w.N = N; w.H = H; w.D = D;
    w.bf16 = t == SOLAR_BF16;
    w.nparts = c.cut.parts;
    w.part_rows = c.cut.rows;
    w.pieces = c.cut.pieces;
    w.parts = c.parts;
    w.part_moments = c.part_moments;
    // dq_t = scale S_t do_t: the same walk with do for q, v for k and k for v, its state transposed
    Walk a = w;
    a.q = g; a.k = vv; a.v = k; a.o = dq;
    a.state_in = state_in;
    a.in_turned = true;
    a.o_scale = scale;
    a.kv_scale = 1.f;
    if (dlog_decay) {
        // sum_t <do_t, d o_t / d log g>: o_t = scale S_t^T q_t, so the same walk gives it as <q_t, d dq_t / d log g>
        a.moment = true;
        a.grad = q;
        a.grad_state = dstate_out;
        a.moments = c.moments;
    }
    hipError_t e = launch_decay_chunks({{a}, 1}, st);
    if (e != hipSuccess) return SOLAR_ERR_HIP;
    if (dlog_decay) {
        e = launch_moment_sum(c.moments, B, H, c.cut.parts * moment_slices(D), dlog_decay, st);
        if (e != hipSuccess) return SOLAR_ERR_HIP;
    }
    // dv_t = G_t^T k_t, dk_t = G_t v_t with G_t = scale q_t do_t^T + g G_{t+1}: walks from the last row on, with one state
    Walk d = w;
    d.reverse = true;
    d.o_scale = 1.f;
    d.kv_scale = scale;
    d.state_in = dstate_out;
    d.o_float = share > 1;
    Heads part;
    if (share > 1 && !take(c.dv, nullptr, B, N, H, D, sizeof(float), 1, true, &part)) return SOLAR_ERR_WORKSPACE;
    d.q = k; d.k = q; d.v = g; d.o = share > 1 ? part : dv;
    d.state_out = dstate_in;
    Walk f = d;
    if (share > 1) part.data = reinterpret_cast<char*>(c.dk);
    f.q = vv; f.k = g; f.v = q; f.o = share > 1 ? part : dk;
    f.in_turned = f.parts_turned = true;
    f.state_out = nullptr;
    e = launch_decay_chunks({{d, f}, 2}, st);
    if (e != hipSuccess) return SOLAR_ERR_HIP;
    if (share > 1) {
        e = launch_share_sum(c.dk, B, N, H, Hkv, D, dk, w.bf16, st);
        if (e != hipSuccess) return SOLAR_ERR_HIP;
        e = launch_share_sum(c.dv, B, N, H, Hkv, D, dv, w.bf16, st);
        if (e != hipSuccess) return SOLAR_ERR_HIP;
    }
    return SOLAR_OK;
}

static solar_status check_norm(int rows, int groups, int d) {
    if (rows <= 0 || groups <= 0 || d <= 0) return SOLAR_ERR_INVALID_ARG;
    if (d > kNormMaxD || groups > 1 << 20 || (int64_t)groups * d > (1 << 26) || (int64_t)rows * groups > INT_MAX) return SOLAR_ERR_UNSUPPORTED;
    return SOLAR_OK;
}

solar_status solar_layer_norm(const void* In, const float* weight, const float* bias, int rows, int groups, int d,
                              float eps, solar_dtype t_in, solar_dtype t_out, void* Out, float* mean, float* rstd,
                              void* stream) {
    const solar_status v = check_norm(rows, groups, d);
    if (v != SOLAR_OK) return v;
    if (!In || !Out || misaligned(In, 16) || misaligned(Out, 16) || !known(t_in) || !known(t_out) || !(eps >= 0.f) ||
        !std::isfinite(eps))
        return SOLAR_ERR_INVALID_ARG;
    if (Out == In && t_in != t_out) return SOLAR_ERR_INVALID_ARG;
    return launch_layer_norm(In, weight, bias, rows, groups, d, eps, t_in == SOLAR_BF16, t_out == SOLAR_BF16, Out, mean,
                             rstd, (hipStream_t)stream) == hipSuccess ? SOLAR_OK : SOLAR_ERR_HIP;
}

size_t solar_layer_norm_workspace_bytes(int rows, int groups, int d) {
    if (check_norm(rows, groups, d) != SOLAR_OK) return 0;
    return align256(sizeof(float) * norm_partial_floats(rows, groups, d));
}

solar_status solar_layer_norm_backward(const void* In, const float* weight, const float* mean, const float* rstd,
                                       const void* dOut, int rows, int groups, int d, solar_dtype t_in,
                                       solar_dtype t_out, void* dIn, float* dweight, float* dbias, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    const solar_status v = check_norm(rows, groups, d);
    if (v != SOLAR_OK) return v;
    if (!In || !mean || !rstd || !dOut || !dIn || misaligned(In, 16) || misaligned(dOut, 16) || misaligned(dIn, 16) ||
        !known(t_in) || !known(t_out))
        return SOLAR_ERR_INVALID_ARG;
    if (dIn == dOut && t_in != t_out) return SOLAR_ERR_INVALID_ARG;
    if (dweight || dbias) {
        const size_t need = solar_layer_norm_workspace_bytes(rows, groups, d);
        if (!workspace || workspace_bytes < need || misaligned(workspace, 256)) return SOLAR_ERR_WORKSPACE;
    }
    return launch_layer_norm_backward(In, weight, mean, rstd, dOut, rows, groups, d, t_in == SOLAR_BF16,
                                      t_out == SOLAR_BF16, dIn, dweight, dbias, static_cast<float*>(workspace),
                                      (hipStream_t)stream) == hipSuccess ? SOLAR_OK : SOLAR_ERR_HIP;
}

}  // extern "C"
