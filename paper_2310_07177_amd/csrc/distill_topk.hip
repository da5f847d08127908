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
// In bulk, with two workgroups a CU whose loads and stores take turns, 16384 rows of
// 32000 bf16 logits, 6 in 10 of them masked, take 316 us, 4.6 TB/s.  Of 512 rows of 32128,
// all resident at once, nothing overlaps: 23.5 us are 3 to start, 5 to load, 4 to sum,
// 2 for the terms, 2 to store and the rest for the stores to leave the caches.
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
    // Split rows.
    int segments;  // workgroups a row
    DistillTopkPart* parts;
    float* split_x;
};

// One row's buckets: by one wave: a slot a lane in turn, the others last
// (in every lane).  In: the record's student logits s_x and teacher logits s_t,
// the row's largest logit, the others' largest and their mass relative to it
// (0: none), the teacher's rest in log2 units (-inf: none).  Out: each token's
// gradient in s_g, the gradient at the others' largest logit (the others' go by it
// and their exponentials relative to it: relative to the row's largest these may
// all vanish in 32 bits while the factor P / Q overflows) and D in nats.
struct RowTerms {
    double others;
    double D;
};
__device__ __forceinline__ RowTerms row_terms(const DistillTopkArgs& a, const float* s_x, const float* s_t, double* s_p,
                                              double* s_q, float* s_g, float top, float all, double sum, double rest,
                                              bool bad) {
    const int lane = opaque_tid() & (kWave - 1), k = a.k;
    const double none = -__builtin_huge_val();
    const double first = double(s_t[0]);
    const auto xs = [&](int i) __attribute__((always_inline)) { return i < k ? (double(s_x[i]) - double(top)) * a.c2 : none; };
    const auto ts = [&](int i) __attribute__((always_inline)) { return i < k ? (double(s_t[i]) - first) * a.c2 : none; };
    double sx = 0.0, st = 0.0;
#pragma unroll 1
    for (int i = lane; i < k; i += kWave) {
        const double q = exp2_f64(xs(i)), p = exp2_f64(ts(i));
        s_q[i] = q;
        s_p[i] = p;
        sx += q;
        st += p;
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
    const auto term = [&](double p, double lp, double q, double lq) __attribute__((always_inline)) {
        if (a.kind == OSD_FKL) return Term{p > 0.0 ? p * (lp - lq) : 0.0, 0.0, 0.0};
        if (a.kind == OSD_RKL) return Term{q > 0.0 ? q * (lq - lp) : 0.0, 0.0, lq - lp};
        // m = p when beta = 1, q when beta = 0.
        const double m = wp * p + wq * q;
        const double lm = wp == 0.0 ? lq : (wq == 0.0 ? lp : (m > 0.0 ? log2_f64(m) : none));
        return Term{wp > 0.0 && p > 0.0 ? p * (lp - lm) : 0.0, wq > 0.0 && q > 0.0 ? q * (lq - lm) : 0.0, lq - lm};
    };
    double d0 = 0.0, d1 = 0.0;
    const double ix = 1.0 / (bad ? 1.0 : sx), it = 1.0 / (bad ? 1.0 : st);
#pragma unroll 1
    for (int i = lane; i < k; i += kWave) {
        const double p = s_p[i] * it, q = s_q[i] * ix;
        const Term t = term(p, ts(i) - zt, q, xs(i) - zx);
        s_p[i] = a.kind == OSD_FKL ? p : t.l;
        s_q[i] = q;
        d0 += t.d0;
        d1 += t.d1;
    }
    const double P = exp2_f64(tz), Q = exp2_f64(xz);
    const Term o = term(P, tz, Q, xz);
    d0 = wave_sum(d0) + o.d0;
    d1 = wave_sum(d1) + o.d1;
    // The factor f of a bucket's tokens over tau.
    const auto factor = [&](double l) __attribute__((always_inline)) {
        return (a.kind == OSD_RKL ? l - d0 : wq * (l - d1)) * (kLn2 * a.inv_tau);
    };
    const double nan = __builtin_nan("");
#pragma unroll 1
    for (int i = lane; i < k; i += kWave) {
        const double q = s_q[i], l = s_p[i];
        double g;
        if (a.kind == OSD_FKL)
            g = (q - l) * a.inv_tau;
        else
            g = q > 0.0 && (a.kind == OSD_RKL || wq > 0.0) ? q * factor(l) : 0.0;
        s_g[i] = float(bad ? nan : g);
    }
    double g = 0.0;
    const double most = exp2_f64((double(all) - double(top)) * a.c2 - zx);  // q of the others' largest
    // (FKL: q_j - P q_j / Q, of which the second part stays where q_j and Q vanish.)
    if (a.kind == OSD_FKL)
        g = sum > 0.0 ? (most - P / sum) * a.inv_tau : 0.0;
    else if (Q > 0.0 && (a.kind == OSD_RKL || wq > 0.0))
        g = most * factor(o.l);
    const double D = a.kind == OSD_JSD ? (wp > 0.0 ? wp * d0 : 0.0) + (wq > 0.0 ? wq * d1 : 0.0) : d0;
    return RowTerms{bad ? nan : g, bad ? nan : D * kLn2};
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
    __shared__ double s_p[OSD_MAX_TOPK], s_q[OSD_MAX_TOPK], s_s[NR], s_part;
    __shared__ float s_m[NR], s_at, s_others;
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
            bool bad = false;
            // Flags: the word and bit of a token's element; set twice, the record
            // holds it twice.  (The row waves wait for nothing else of the record.)
            const auto word = [&](int token) __attribute__((always_inline)) { return token / EPC >> 2; };
            const auto bit = [&](int token) __attribute__((always_inline)) {
                const int ch = token / EPC, e = token - ch * EPC + (ch >= held.cut.nfull ? held.cut.dup : 0);
                return 1u << ((ch & 3) * 8 + e);
            };
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                if (id[j] < -1 || id[j] >= a.V) {
                    bad = true;
                    id[j] = -1;
                }
                if (id[j] >= 0) {
                    const uint32_t f = bit(id[j]);
                    bad = bad || (atomicOr(&s_flag[word(id[j])], f) & f) != 0;
                }
            }
            __syncthreads();  // 1: the flags are set
            bad = bad || !(rest < -kNegInf);
#pragma unroll
            for (int j = 0; j < kSlots; ++j) x[j] = id[j] >= 0 ? Fmt::load_one(row, id[j]) : kNegInf;
            float xm = kNegInf;
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const int slot = j * kWave + lane;
                if (id[j] < 0) t[j] = kNegInf;
                if (slot < k) {
                    s_x[slot] = x[j];
                    s_t[slot] = t[j];
                }
                if (id[j] >= 0) bad = bad || !(x[j] < -kNegInf) || !(t[j] < -kNegInf);
                xm = fmaxf(xm, x[j]);
            }
            bad = bad || (lane == 0 && t[0] == kNegInf);
            __syncthreads();  // 2: the row waves' sums are there
            const float m = lane < NR ? s_m[lane] : kNegInf;
            const float all = wave_max(m), top = fmaxf(all, wave_max(xm));
            const double sum = wave_sum(lane < NR ? s_s[lane] * exp2_f64((double(m) - double(all)) * a.c2) : 0.0);
            // (A NaN or +inf outside the record makes the sum NaN.)
            bad = __ballot(bad) != 0 || !is_finite(top) || sum != sum;
            const RowTerms r = row_terms(a, s_x, s_t, s_p, s_q, s_g, top, all, sum, double(rest) * 1.4426950408889634074, bad);
            if (lane == 0) {
                s_at = all > kNegInf ? all : 0.0f;
                s_others = float(r.others);
                s_part += r.D;
                if (a.row_loss) a.row_loss[n] = float(r.D);
            }
            __syncthreads();  // 3: the row's factors are there
#pragma unroll
            for (int j = 0; j < kSlots; ++j)
                if (id[j] >= 0) atomicAnd(&s_flag[word(id[j])], ~bit(id[j]));
            wave_lds_order();  // (before the next row's are set)
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
        const float at = s_at, scale = s_others;
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

// Few rows are split over workgroups, in two launches: each workgroup of the first
// takes the others' mass in its segment and the logits of the record's tokens there,
// each of the second the row's bucket terms and the gradient of its segment, read
// again.  (Every workgroup of a row takes the terms for itself.  Taken by the last
// workgroup of the first launch to arrive they waited for three more trips to memory:
// 4 rows of 128256 bf16 logits, k = 256, 14.8 us against 11.6.)  A row of 256 KB in one
// CU is bound by its instructions, 28 us.
constexpr int kPartWaves = 4;

template <typename Fmt, int CPT>
__global__ __launch_bounds__(kPartWaves* kWave, 4) void distill_topk_part_kernel(DistillTopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk, NW = kPartWaves, W = NW * kWave;
    static_assert(W >= OSD_MAX_TOPK, "a slot a thread");
    __shared__ uint32_t s_flag[W * CPT / 4];  // a byte per chunk, a bit per element
    __shared__ double s_s[NW];
    __shared__ float s_m[NW];
    __shared__ int s_twice;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int n = blockIdx.x / a.segments, p = blockIdx.x - n * a.segments;
    if (a.mask && a.mask[n] == 0) return;
    const int b = n / a.K, i = n - b * a.K;
    const char* row = a.student + b * a.student_stride + int64_t(i) * a.V * Fmt::kBytes;
    const int64_t rec = b * a.teacher_rows + i;
    const int start = p * CPT * W;
    const HeldSegment<Fmt, W, CPT> held(a.V, start);
    chunk_t c[CPT];
    const int id = tid < a.k ? a.ids[rec * a.k + tid] : -1;
    held.template load<0>(c, row, a.V, tid);
    for (int w = tid; w < CPT * W / 4; w += W) s_flag[w] = 0u;
    if (tid == 0) s_twice = 0;
    __syncthreads();
    // The record's tokens in the segment: their flags (set twice, the record holds
    // one twice) and logits.
    if (id >= 0 && id < a.V) {
        const int whole = id / EPC, ch = whole - start;
        if (ch >= 0 && ch < CPT * W) {
            const uint32_t f = 1u << ((ch & 3) * 8 + id - whole * EPC + (whole >= held.cut.nfull ? held.cut.dup : 0));
            if (atomicOr(&s_flag[ch >> 2], f) & f) s_twice = 1;
            a.split_x[int64_t(n) * OSD_MAX_TOPK + tid] = Fmt::load_one(row, id);
        }
    }
    __syncthreads();
    held.pad(c, tid);
    float m = kNegInf;
#pragma unroll
    for (int r = 0; r < CPT; ++r) {
        const int ch = r * W + tid;
        const uint32_t f = (s_flag[ch >> 2] >> ((ch & 3) * 8)) & 0xFFu;
        if (f) c[r] = drop_elements<Fmt>(c[r], f);
        m = fmaxf(m, chunk_max<Fmt>(c[r]));
    }
    m = wave_max(m);
    const float ref = m > kNegInf ? m : 0.0f, c2 = float(a.c2);
    double S = 0.0;
#pragma unroll
    for (int r = 0; r < CPT; ++r) {
        asm volatile("" : "+v"(c[r]));  // unpacked anew, not held from the first sweep
        float e8[EPC];
#pragma unroll
        for (int e = 0; e < EPC; ++e) e8[e] = exp2_fast((Fmt::get(c[r], e) - ref) * c2);
#pragma unroll
        for (int w = 1; w < EPC; w <<= 1)
#pragma unroll
            for (int e = 0; e < EPC; e += 2 * w) e8[e] = e8[e] + e8[e + w];
        S += double(e8[0]);
        __builtin_amdgcn_sched_barrier(0);
    }
    S = wave_sum(S);
    if (lane == 0) {
        s_m[wid] = m;
        s_s[wid] = S;
    }
    __syncthreads();
    if (wid != 0) return;
    m = lane < NW ? s_m[lane] : kNegInf;
    const float all = wave_max(m);
    S = wave_sum(lane < NW ? s_s[lane] * exp2_f64((double(m) - double(all)) * a.c2) : 0.0);
    if (lane == 0) a.parts[int64_t(n) * a.segments + p] = DistillTopkPart{s_twice ? __builtin_nan("") : S, all};
}

// (GRAD: a.segments workgroups a row; without, one.)
template <typename Fmt, int CPT, bool GRAD>
__global__ __launch_bounds__(kPartWaves* kWave, 4) void distill_topk_finish_kernel(DistillTopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk, NW = kPartWaves, W = NW * kWave;
    __shared__ float s_x[OSD_MAX_TOPK], s_t[OSD_MAX_TOPK], s_g[OSD_MAX_TOPK];
    __shared__ double s_p[OSD_MAX_TOPK], s_q[OSD_MAX_TOPK], s_part;
    __shared__ float s_xm[NW], s_others;
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int k = a.k, n = GRAD ? blockIdx.x / a.segments : blockIdx.x, p = GRAD ? blockIdx.x - n * a.segments : 0;
    const int64_t row_bytes = int64_t(a.V) * Fmt::kBytes;
    const int start = p * CPT * W;
    const HeldSegment<Fmt, W, CPT> held(a.V, start);
    char* grow = a.grad + n * row_bytes;
    const rsrc_t rs = make_rsrc(grow, uint32_t(row_bytes));
    if (a.mask && a.mask[n] == 0) {
        if constexpr (GRAD)
            for (int r = 0; r < CPT; ++r) held.store(rs, r, chunk_t{0u, 0u, 0u, 0u}, tid);
        if (p) return;
        if (tid == 0) {
            if (a.row_loss) a.row_loss[n] = 0.0f;
            s_part = 0.0;
        }
        finish_loss<W>(a.tail, &s_part, n);
        return;
    }
    const int b = n / a.K, i = n - b * a.K;
    const int64_t rec = b * a.teacher_rows + i;
    chunk_t c[CPT];
    if constexpr (GRAD) held.template load<kStreamAux>(c, a.student + b * a.student_stride + i * row_bytes, a.V, tid);
    int id = tid < k ? a.ids[rec * k + tid] : -1;
    float t = tid < k ? Fmt::load_one(a.top + rec * k * Fmt::kBytes, tid) : kNegInf;
    float x = tid < k ? a.split_x[int64_t(n) * OSD_MAX_TOPK + tid] : kNegInf;
    const float rest = a.rest ? a.rest[rec] : kNegInf;
    if (tid == 0) s_bad = 0;
    // The segments' masses, joined by each wave for itself.
    float all = kNegInf;
    double sum = 0.0;
    {
        const DistillTopkPart* parts = a.parts + int64_t(n) * a.segments;
        float m = kNegInf;
        double s = 0.0;
#pragma unroll 1
        for (int j = lane; j < a.segments; j += kWave) {
            const DistillTopkPart part = parts[j];
            const float mx = fmaxf(m, part.top);
            s = mx > kNegInf ? s * exp2_f64((double(m) - double(mx)) * a.c2) +
                                   part.sum * exp2_f64((double(part.top) - double(mx)) * a.c2)
                             : s + part.sum;  // (0, or NaN)
            m = mx;
        }
        all = wave_max(m);
        sum = wave_sum(all > kNegInf ? s * exp2_f64((double(m) - double(all)) * a.c2) : s);
    }
    bool bad = id < -1 || id >= a.V;
    if (bad) id = -1;
    if (id < 0) x = t = kNegInf;
    if (tid < k) {
        s_x[tid] = x;
        s_t[tid] = t;
    }
    bad = bad || !(rest < -kNegInf) || (tid == 0 && t == kNegInf) ||
          (id >= 0 && (!(x < -kNegInf) || !(t < -kNegInf)));
    const float xm = wave_max(x == x ? x : kNegInf);
    if (lane == 0) s_xm[wid] = xm;
    __syncthreads();
    if (__ballot(bad) && lane == 0) s_bad = 1;
    __syncthreads();
    float top = all;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_xm[w]);
    // (A NaN or +inf outside the record makes the sum NaN.)
    bad = s_bad || !is_finite(top) || sum != sum;
    if (wid == 0) {
        const RowTerms r = row_terms(a, s_x, s_t, s_p, s_q, s_g, top, all, sum,
                                     double(rest) * 1.4426950408889634074, bad);
        if (lane == 0) {
            s_others = float(r.others);
            s_part = r.D;
        }
    }
    __syncthreads();
    if constexpr (GRAD) {
        const float at = all > kNegInf ? all : 0.0f, scale = s_others, c2 = float(a.c2);
#pragma unroll
        for (int r = 0; r < CPT; ++r) {
            float v[EPC];
#pragma unroll
            for (int e = 0; e < EPC; ++e) v[e] = exp2_fast((Fmt::get(c[r], e) - at) * c2) * scale;
            held.store(rs, r, pack_grad<Fmt>(v), tid);
            __builtin_amdgcn_sched_barrier(0);
        }
        // The record's tokens are written over what stands in their places.
        wait_memory();
        __syncthreads();
        const int ch = id / EPC - start;
        if (id >= 0 && ch >= 0 && ch < CPT * W) {
            if constexpr (EPC == 8)
                reinterpret_cast<uint16_t*>(grow)[id] = uint16_t(pack_bf16x2(s_g[tid], 0.0f));
            else
                reinterpret_cast<float*>(grow)[id] = s_g[tid];
        }
    }
    if (p) return;
    if (tid == 0 && a.row_loss) a.row_loss[n] = float(s_part);
    finish_loss<W>(a.tail, &s_part, n);
}

template <typename Fmt, int CPT>
hipError_t launch_segments(const DistillTopkLaunch& L, DistillTopkArgs a, int chunks) {
    constexpr int W = kPartWaves * kWave;
    a.segments = (chunks + CPT * W - 1) / (CPT * W);
    const int64_t groups = int64_t(a.N) * a.segments;
    if (groups > kDistillTopkParts + int64_t(a.N) * kDistillTopkLongest) return hipErrorInvalidValue;
    a.tail.G = a.N;
    const dim3 all(static_cast<uint32_t>(groups)), each(static_cast<uint32_t>(a.N));
    const LaunchesTogether together;  // the second reads parts and split_x
    const hipError_t st = launch_kernel(&distill_topk_part_kernel<Fmt, CPT>, all, dim3(W), 0, L.stream, a);
    if (st != hipSuccess) return st;
    return a.grad ? launch_kernel(&distill_topk_finish_kernel<Fmt, CPT, true>, all, dim3(W), 0, L.stream, a)
                  : launch_kernel(&distill_topk_finish_kernel<Fmt, 1, false>, each, dim3(W), 0, L.stream, a);
}

// Segments as short as leave about kDistillTopkParts workgroups (four a CU).
template <typename Fmt>
hipError_t launch_split(const DistillTopkLaunch& L, const DistillTopkArgs& a, int chunks) {
    const int64_t most = int64_t(kDistillTopkParts) * kPartWaves * kWave, all = int64_t(a.N) * chunks;
    if (all <= most) return launch_segments<Fmt, 1>(L, a, chunks);
    if (all <= 2 * most) return launch_segments<Fmt, 2>(L, a, chunks);
    if (all <= 4 * most) return launch_segments<Fmt, 4>(L, a, chunks);
    return launch_segments<Fmt, 8>(L, a, chunks);
}

template <typename Fmt, int NR, int CPT, int MINR>
hipError_t launch_tile(const DistillTopkLaunch& L, DistillTopkArgs a) {
    constexpr int W = (NR + 1) * kWave;
    // Twice as many workgroups as are resident at once (1024 threads a CU: the record wave's
    // fp64 terms take 108 to 128 registers, whatever the row waves hold) take the rows in
    // turn.  Where a mask leaves some of them more to do than others, eight times as many
    // even that out for long rows.  16384 bf16 rows (of 64000: 8192) with 1, 4, 8 in 10
    // unmasked and all, us, without that and with it:
    //   1000   54  78 108 101   122 124 130 127
    //   4000   63 107 148 138   122 131 151 149
    //   8000   95 139 191 186   127 139 189 191
    //   16000 155 231 323 335   143 231 326 358
    //   18500 203 244 359 369   177 244 353 401
    //   24000 217 282 390 409   201 266 384 446
    //   32000 280 355 472 492   266 317 445 513
    //   64000 265 412 555 544   233 375 538 568
    // Of 2048 rows it is the same.  (The tile changes at 17920.)
    const int each = a.mask && NR * CPT >= 70 ? 8 : 1;
    int g = L.cus * (2048 / W) * each;
    if (g > kMaxDistillTopkGroups) g = kMaxDistillTopkGroups;
    if (g > a.N) g = a.N;
    a.tail.G = g;
    return launch_kernel(&distill_topk_kernel<Fmt, NR, CPT, MINR>, dim3(g), dim3(W), 0, L.stream, a);
}

template <typename Fmt>
hipError_t launch_fmt(const DistillTopkLaunch& L, const DistillTopkArgs& a) {
    const int chunks = (L.V + Fmt::kPerChunk - 1) / Fmt::kPerChunk;
    // One workgroup a row or several (us, with and without a gradient): a row of 16000
    // bf16 logits 11.2 and 9.6 against 10.0 and 8.6, of 128256 28.0 and 21.2 against
    // 10.1 and 9.4, but of 4000 9.0 and 8.4 against 9.7 and 8.5; 128 rows of 32128
    // 15.9 and 13.2 against 14.6 and 12.1, 256 of them 18.3 and 15.4 against 19.3 and 17.3;
    // 512 of 128256, where a CU holds one row, 75.5 and 54.5 against 78.4 and 42.1.
    if (chunks > 1024 && a.N <= kDistillTopkSplitRows &&
        (2 * a.N <= L.cus || (!a.grad && chunks > 7 * 10 * kWave)))
        return launch_split<Fmt>(L, a, chunks);
    const int waves = (chunks + kWave - 1) / kWave;  // of one chunk a lane
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
    a.parts = L.parts;
    a.split_x = L.split_x;
    return L.dtype == 1 ? launch_fmt<BF16>(L, a) : launch_fmt<F32>(L, a);
}

}  // namespace osd
