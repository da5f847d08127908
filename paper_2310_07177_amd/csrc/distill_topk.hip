// distill_topk.hip -- distillation loss and gradient of a student's rows against
// the record of their teacher's rows (gfx950).
//
// Method: with the record's tokens as k buckets and every other token in one
// more, teacher and student are distributions over k + 1 buckets:
//   p = softmax(top_1 / tau, .., top_k / tau, rest)   (no rest: p of the last
//                                                       bucket is 0)
//   q = (q_1, .., q_k, Q),  q_j = softmax(s / tau)_j,  Q the others' sum
// and D is the divergence between them.  A student logit s_j enters through its
// bucket b(j) alone, so with w_b = dD/dq_b the chain rule through the softmax is
//   dD/ds_j = q_j f_b(j) / tau,   f_b = w_b - sum_b' q_b' w_b'
//   FKL  f_b = 1 - p_b / q_b
//   RKL  f_b = log(q_b / p_b) - D
//   JSD  f_b = (1 - beta) (log(q_b / m_b) - KL(q || m)),  m = beta p + (1 - beta) q
// The row is read once: the gradient of every token outside the record is its
// exponential times one number.
//
// The others' mass Q is summed over the tokens outside the record (one bit per
// token in LDS says which are in it) rather than taken as 1 minus the others, with a
// shift of its own, so log Q is exact to fp32 rounding however small Q is.
#include "osd.h"
#include "osd_device.hpp"
#include "osd_internal.hpp"
#include "distill_common.hpp"
#include "stream_device.hpp"
#include "topk_device.hpp"

namespace osd {
namespace {

struct DistillTopkArgs {
    const int32_t* ids;
    const char* top;
    const float* rest;
    int64_t teacher_rows;  // record rows between sequences
    int k;
    const char* student;
    int64_t student_stride;  // bytes between sequences
    int N, K, V;             // N = B * K rows
    const uint8_t* mask;
    int kind;
    double beta;
    double c2;       // log2(e) / tau
    double inv_tau;
    float* row_loss;
    char* grad;
    LossTail tail;
};

// One row's buckets, by wave 0: slot i = j * 64 + lane in turn, the others last
// (in every lane).  In: the record's student logits s_x and teacher logits s_t,
// the row's largest logit, the others' largest and their mass relative to it
// (0: none), the teacher's rest in log2 units (-inf: none).  Out: each token's
// gradient in s_g, 2^-z f for the others' (z the student's log2 normaliser
// relative to the row's largest logit, f their factor over tau) and D in nats.
struct RowTerms {
    double others;
    double D;
};
__device__ __forceinline__ RowTerms row_terms(const DistillTopkArgs& a, const float* s_x, const float* s_t, float* s_g,
                                     float top, float all, double sum, double rest, bool bad) {
    const int lane = threadIdx.x & (kWave - 1), k = a.k;
    const double none = -__builtin_huge_val();
    const double first = double(s_t[0]);
    const auto xs = [&](int i) __attribute__((always_inline)) { return i < k ? (double(s_x[i]) - double(top)) * a.c2 : none; };
    const auto ts = [&](int i) __attribute__((always_inline)) { return i < k ? (double(s_t[i]) - first) * a.c2 : none; };
    double sx = 0.0, st = 0.0;
#pragma unroll 1
    for (int i = lane; i < k; i += kWave) {
        sx += exp2_f64(xs(i));
        st += exp2_f64(ts(i));
    }
    const double xo = sum > 0.0 ? (double(all) - double(top)) * a.c2 + log2_f64(sum) : none;
    sx = wave_sum(sx) + exp2_f64(xo);
    st = wave_sum(st) + exp2_f64(rest);
    bad = bad || !(sx > 0.0) || !(st > 0.0);
    const double zx = log2_f64(bad ? 1.0 : sx), zt = log2_f64(bad ? 1.0 : st);
    const double wp = a.beta, wq = 1.0 - a.beta;
    const double xz = xo - zx, tz = rest - zt;  // log2 Q, log2 P
    // A bucket's terms of D (JSD: of KL(p || m) and KL(q || m)) and its log ratio,
    // in log2 units.
    struct Term {
        double d0, d1, l;
    };
    const auto term = [&](double lp, double lq) __attribute__((always_inline)) {
        const double p = exp2_f64(lp), q = exp2_f64(lq);
        if (a.kind == OSD_FKL) return Term{p > 0.0 ? p * (lp - lq) : 0.0, 0.0, 0.0};
        if (a.kind == OSD_RKL) return Term{q > 0.0 ? q * (lq - lp) : 0.0, 0.0, lq - lp};
        // m = p when beta = 1, q when beta = 0.
        const double m = wp * p + wq * q;
        const double lm = wp == 0.0 ? lq : (wq == 0.0 ? lp : (m > 0.0 ? log2_f64(m) : none));
        return Term{wp > 0.0 && p > 0.0 ? p * (lp - lm) : 0.0, wq > 0.0 && q > 0.0 ? q * (lq - lm) : 0.0, lq - lm};
    };
    double d0 = 0.0, d1 = 0.0;
#pragma unroll 1
    for (int i = lane; i < k; i += kWave) {
        const Term t = term(ts(i) - zt, xs(i) - zx);
        d0 += t.d0;
        d1 += t.d1;
    }
    const Term o = term(tz, xz);
    d0 = wave_sum(d0) + o.d0;
    d1 = wave_sum(d1) + o.d1;
    // The factor f of a bucket's tokens over tau.
    const auto factor = [&](double l) __attribute__((always_inline)) {
        return (a.kind == OSD_RKL ? l - d0 : wq * (l - d1)) * (kLn2 * a.inv_tau);
    };
    const double nan = __builtin_nan("");
#pragma unroll 1
    for (int i = lane; i < k; i += kWave) {
        const double lp = ts(i) - zt, lq = xs(i) - zx, p = exp2_f64(lp), q = exp2_f64(lq);
        double g;
        if (a.kind == OSD_FKL)
            g = (q - p) * a.inv_tau;
        else
            g = q > 0.0 && (a.kind == OSD_RKL || wq > 0.0) ? q * factor(term(lp, lq).l) : 0.0;
        s_g[i] = float(bad ? nan : g);
    }
    const double Q = exp2_f64(xz);
    double f = 0.0;
    if (Q > 0.0) {
        if (a.kind == OSD_FKL)
            f = (1.0 - exp2_f64(tz) / Q) * a.inv_tau;
        else if (a.kind == OSD_RKL || wq > 0.0)
            f = factor(o.l);
    }
    const double D = a.kind == OSD_JSD ? (wp > 0.0 ? wp * d0 : 0.0) + (wq > 0.0 ? wq * d1 : 0.0) : d0;
    return RowTerms{bad ? nan : f * exp2_f64(-zx), bad ? nan : D * kLn2};
}

// The chunk with the elements of bit mask f replaced by -inf.
template <typename Fmt>
__device__ inline chunk_t drop_elements(const chunk_t& c, uint32_t f) {
    uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (Fmt::kPerChunk == 8) {
            if ((f >> (2 * i)) & 1u) w[i] = (w[i] & 0xFFFF0000u) | 0xFF80u;
            if ((f >> (2 * i + 1)) & 1u) w[i] = (w[i] & 0xFFFFu) | 0xFF800000u;
        } else {
            if ((f >> i) & 1u) w[i] = 0xFF800000u;
        }
    }
    return chunk_t{w[0], w[1], w[2], w[3]};
}

// A workgroup of NR row waves, which hold the row, and one record wave, which
// holds no part of it: it reads the record, flags its tokens and takes the
// bucket terms, so their fp64 arithmetic shares no registers with the row
// (in one of the row waves it spilled up to a hundred of them) and the record of
// the next row is read while this row's gradient is written.
template <typename Fmt, int NR, int CPT, int MINR>
__global__ __launch_bounds__((NR + 1) * kWave, 4) void distill_topk_kernel(DistillTopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk, W = NR * kWave, kSlots = OSD_MAX_TOPK / kWave;
    __shared__ uint32_t s_flag[(W * CPT + 3) / 4];  // a byte per chunk, a bit per element
    __shared__ float s_x[OSD_MAX_TOPK], s_t[OSD_MAX_TOPK], s_g[OSD_MAX_TOPK];
    __shared__ double s_s[NR], s_part;
    __shared__ float s_m[NR], s_top, s_others;
    __shared__ LossTail s_tail;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int k = a.k;
    const HeldRow<Fmt, W, CPT, MINR> held(a.V);
    const int64_t row_bytes = int64_t(a.V) * Fmt::kBytes;
    for (int i = tid; i < (W * CPT + 3) / 4; i += W + kWave) s_flag[i] = 0u;
    if (tid == 0) {
        s_tail.row_ws = a.tail.row_ws;
        s_tail.done = a.tail.done;
        s_tail.loss_out = a.tail.loss_out;
        s_tail.mask = a.tail.mask;
        s_tail.nrows = a.tail.nrows;
        s_tail.G = a.tail.G;
        s_part = 0.0;
    }
    __syncthreads();
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        char* grow = a.grad ? a.grad + n * row_bytes : nullptr;
        if (a.mask && a.mask[n] == 0) {
            if (grow) zero_row<W + kWave>(make_rsrc(grow, uint32_t(row_bytes)), uint32_t(row_bytes), opaque_tid());
            if (tid == 0 && a.row_loss) a.row_loss[n] = 0.0f;
            continue;
        }
        const int64_t b = n / a.K, i = n - b * a.K;
        const char* row = a.student + b * a.student_stride + i * row_bytes;
        if (wid == NR) {
            const int64_t rec = b * a.teacher_rows + i;
            int id[kSlots];
            float x[kSlots], t[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const int slot = j * kWave + lane;
                id[j] = slot < k ? a.ids[rec * k + slot] : -1;
                t[j] = slot < k ? Fmt::load_one(a.top + rec * k * Fmt::kBytes, slot) : kNegInf;
            }
            const float rest = a.rest ? a.rest[rec] : kNegInf;
            bool bad = !(rest < -kNegInf);
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                if (id[j] < -1 || id[j] >= a.V) {
                    bad = true;
                    id[j] = -1;
                }
                x[j] = id[j] >= 0 ? Fmt::load_one(row, id[j]) : kNegInf;
                if (id[j] < 0) t[j] = kNegInf;
            }
            // Flags: the word and bit of a token's element; set twice, the record
            // holds it twice.
            const auto word = [&](int token) __attribute__((always_inline)) { return token / EPC >> 2; };
            const auto bit = [&](int token) __attribute__((always_inline)) {
                const int ch = token / EPC, e = token - ch * EPC + (ch >= held.cut.nfull ? held.cut.dup : 0);
                return 1u << ((ch & 3) * 8 + e);
            };
            float xm = kNegInf;
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const int slot = j * kWave + lane;
                if (slot < k) {
                    s_x[slot] = x[j];
                    s_t[slot] = t[j];
                }
                if (id[j] >= 0) {
                    const uint32_t f = bit(id[j]);
                    bad = bad || (atomicOr(&s_flag[word(id[j])], f) & f) != 0;
                    bad = bad || !(x[j] < -kNegInf) || !(t[j] < -kNegInf);
                }
                xm = fmaxf(xm, x[j]);
            }
            bad = bad || (lane == 0 && t[0] == kNegInf);
            __syncthreads();  // 1: the flags are set
            __syncthreads();  // 2: the row waves' sums are there
            const float m = lane < NR ? s_m[lane] : kNegInf;
            const float all = wave_max(m), top = fmaxf(all, wave_max(xm));
            const double sum = wave_sum(lane < NR ? s_s[lane] * exp2_f64((double(m) - double(all)) * a.c2) : 0.0);
            // (A NaN or +inf outside the record makes the sum NaN.)
            bad = __ballot(bad) != 0 || !is_finite(top) || sum != sum;
            const RowTerms r = row_terms(a, s_x, s_t, s_g, top, all, sum, double(rest) * 1.4426950408889634074, bad);
            if (lane == 0) {
                s_top = top;
                s_others = float(r.others);
                s_part += r.D;
                if (a.row_loss) a.row_loss[n] = float(r.D);
            }
            __syncthreads();  // 3: the row's factors are there
#pragma unroll
            for (int j = 0; j < kSlots; ++j)
                if (id[j] >= 0) atomicAnd(&s_flag[word(id[j])], ~bit(id[j]));
            if (!grow) continue;
            __syncthreads();  // 4: the others' gradient is written
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                if (id[j] < 0) continue;
                const float g = s_g[j * kWave + lane];
                if constexpr (EPC == 8)
                    reinterpret_cast<uint16_t*>(grow)[id[j]] = uint16_t(pack_bf16x2(g, 0.0f));
                else
                    reinterpret_cast<float*>(grow)[id[j]] = g;
            }
            continue;
        }
        const float c2 = float(a.c2);
        chunk_t c[CPT];
        int t = opaque_tid();
        held.load(c, row, a.V, t);
        __syncthreads();  // 1
        t = opaque_tid();
        held.pad(c, t);
        // The others: their largest logit, and their mass relative to the thread's
        // own largest.
        float m = kNegInf;
        held.each([&](int r) __attribute__((always_inline)) {
            const int ch = r * W + t;
            const uint32_t f = (s_flag[ch >> 2] >> ((ch & 3) * 8)) & 0xFFu;
            if (f) c[r] = drop_elements<Fmt>(c[r], f);
            m = fmaxf(m, chunk_max<Fmt>(c[r]));
        });
        const float ref = m > kNegInf ? m : 0.0f;
        double S = 0.0;
        held.each([&](int r) __attribute__((always_inline)) {
            asm volatile("" : "+v"(c[r]));
            float e8[EPC];
#pragma unroll
            for (int e = 0; e < EPC; ++e) e8[e] = exp2_fast((Fmt::get(c[r], e) - ref) * c2);
#pragma unroll
            for (int w = 1; w < EPC; w <<= 1)
#pragma unroll
                for (int e = 0; e < EPC; e += 2 * w) e8[e] = e8[e] + e8[e + w];
            S += double(e8[0]);
        });
        const float mw = wave_max(m);
        S = wave_sum(S * exp2_f64((double(m) - double(mw)) * a.c2));
        if (lane == 0) {
            s_m[wid] = mw;
            s_s[wid] = S;
        }
        __syncthreads();  // 2
        __syncthreads();  // 3
        if (!grow) continue;
        const float at = s_top, scale = s_others;
        const rsrc_t rs = make_rsrc(grow, uint32_t(row_bytes));
        t = opaque_tid();
        held.each([&](int r) __attribute__((always_inline)) {
            asm volatile("" : "+v"(c[r]));
            float g[EPC];
#pragma unroll
            for (int e = 0; e < EPC; ++e) g[e] = exp2_fast((Fmt::get(c[r], e) - at) * c2) * scale;
            held.store(rs, r, pack_grad<Fmt>(g), t);
        });
        // The record's tokens are written over the zeros left in their places.
        wait_memory();
        __syncthreads();  // 4
    }
    __syncthreads();
    finish_loss<W + kWave>(s_tail, &s_part);
}

template <typename Fmt, int NR, int CPT, int MINR>
hipError_t launch_tile(const DistillTopkLaunch& L, DistillTopkArgs a) {
    constexpr int W = (NR + 1) * kWave;
    int g = L.cus * (2048 / W);
    if (g > kMaxDistillTopkGroups) g = kMaxDistillTopkGroups;
    if (g > a.N) g = a.N;
    a.tail.G = g;
    return launch_kernel(&distill_topk_kernel<Fmt, NR, CPT, MINR>, dim3(g), dim3(W), 0, L.stream, a);
}

template <typename Fmt>
hipError_t launch_fmt(const DistillTopkLaunch& L, const DistillTopkArgs& a) {
    const int waves = ((L.V + Fmt::kPerChunk - 1) / Fmt::kPerChunk + kWave - 1) / kWave;  // of one chunk a lane
    if (waves <= 3 * 2) return launch_tile<Fmt, 3, 2, 1>(L, a);
    if (waves <= 3 * 6) return launch_tile<Fmt, 3, 6, 3>(L, a);
    if (waves <= 7 * 5) return launch_tile<Fmt, 7, 5, 3>(L, a);
    if (waves <= 7 * 10) return launch_tile<Fmt, 7, 10, 6>(L, a);
    if (waves <= 15 * 9) return launch_tile<Fmt, 15, 9, 5>(L, a);
    if (waves <= 15 * 18) return launch_tile<Fmt, 15, 18, 10>(L, a);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_distill_topk(const DistillTopkLaunch& L) {
    DistillTopkArgs a{};
    const int es = L.dtype == 1 ? 2 : 4;
    a.ids = L.ids;
    a.top = static_cast<const char*>(L.top);
    a.rest = L.rest;
    a.teacher_rows = L.teacher_rows;
    a.k = L.k;
    a.student = static_cast<const char*>(L.student);
    a.student_stride = L.student_stride * es;
    a.N = L.B * L.K;
    a.K = L.K;
    a.V = L.V;
    a.mask = L.mask;
    a.kind = L.kind;
    a.beta = double(L.beta);
    a.c2 = scaled_log2e(L.tau);
    a.inv_tau = 1.0 / double(L.tau);
    a.row_loss = L.row_loss_out;
    a.grad = static_cast<char*>(L.grad_out);
    a.tail = LossTail{L.partials, L.done_counter, L.loss_out, L.mask, a.N, 0};
    return L.dtype == 1 ? launch_fmt<BF16>(L, a) : launch_fmt<F32>(L, a);
}

}  // namespace osd
