// topk_device.hpp -- building blocks of the operators on the record of a row's
// top logits (gfx950, wave64).
//
// A record of a row of V logits holds k slots in descending order of logit
// (ascending token id among equal ones): token id and logit, id -1 and logit
// -inf in slots past the row's finite logits; and, where it was asked for, the
// logarithm of the mass of every other token.
#pragma once

#include "osd_device.hpp"
#include "stream_device.hpp"

namespace osd {

// 2^x in fp64 for x <= 0 (x below -1100 gives 0): x = n + r with |r| <= 1/2
// through the whole number that adding 1.5 * 2^52 leaves in the low mantissa
// bits, 2^r by a polynomial of degree 8 (Remez on the relative error: 8e-13),
// 2^n by ldexp.  fp64 vector instructions run at the rate of unpacked fp32 ones
// on this part, so this costs about twice what v_exp_f32 with its fp64 sum does,
// and a draw decided on such masses agrees with exact arithmetic to about 1e-12 of
// the row's mass: fp32 exponentials leave up to 1e-7, which over a flat row of 32000
// tokens moves one draw in a hundred.
__device__ inline double exp2_f64(double x) {
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52
    x = __builtin_fmax(x, -1100.0);
    const double z = x + kMagic;
    const int n = int(uint32_t(__builtin_bit_cast(uint64_t, z)));
    const double r = x - (z - kMagic);
    double p = 1.3175858099999285e-06;
    p = __builtin_fma(p, r, 1.5309737421788504e-05);
    p = __builtin_fma(p, r, 0.00015403851748798368);
    p = __builtin_fma(p, r, 0.0013333452062249912);
    p = __builtin_fma(p, r, 0.009618128542862288);
    p = __builtin_fma(p, r, 0.05550410939341708);
    p = __builtin_fma(p, r, 0.2402265069888037);
    p = __builtin_fma(p, r, 0.6931471805465141);
    p = __builtin_fma(p, r, 0.9999999999997623);
    return __builtin_ldexp(p, n);
}

// log2 of a positive finite double to about 1e-12: the exponent, v_log_f32 of
// the mantissa (6e-8) and one Newton step on 2^y = m.
__device__ inline double log2_f64(double x) {
    const double m = __builtin_amdgcn_frexp_mant(x);  // [1/2, 1)
    const double y = double(__builtin_amdgcn_logf(float(m)));
    return double(__builtin_amdgcn_frexp_exp(x)) + y + (m * exp2_f64(-1.0 - y) * 2.0 - 1.0) * 1.4426950408889634074;
}

// Between LDS accesses of one lane and those of other lanes of its wave to the same
// words: the compiler keeps their order (the wave's own LDS accesses run in order; no
// instruction).
__device__ inline void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The larger of two floats, NaN if either is one.
__device__ inline float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Wave maximum that keeps a NaN; every lane gets it.
__device__ inline float wave_max_nan(float v) {
    const bool any = __ballot(v != v) != 0;
    const float m = wave_max(v == v ? v : kNegInf);
    return any ? __builtin_nanf("") : m;
}

// A logit that can carry mass (neither NaN nor an infinity).
__device__ inline bool is_finite(float x) { return x > kNegInf && x < -kNegInf; }

// One order for the logits of both formats: float_key with the zeros equal.
// A NaN takes the largest key.
__device__ inline uint32_t order_key(float x) { return x == x ? float_key(x + 0.0f) : 0xFFFFFFFFu; }
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;
constexpr uint32_t kKeyPosInf = 0xFF800000u;

// Stores chunk ch of the row at the descriptor's base (whole: it is known to have no
// padding).
template <typename Fmt>
__device__ __forceinline__ void store_chunk(const RowCut<Fmt>& cut, rsrc_t rs, int ch, bool whole, const chunk_t& c) {
    if (whole || ch < cut.nfull) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(__attribute__((ext_vector_type(4))) int, c), rs,
                                               ch * 16, 0, kStreamAux);
        return;
    }
    if (ch >= cut.nchunks) return;
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    int lead = cut.dup;
    asm volatile("" : "+v"(lead));  // compared here, not hoisted (see pad_lead)
#pragma unroll
    for (int e = 0; e < Fmt::kPerChunk; ++e) {
        if (e < lead) continue;
        const int off = cut.last_off + e * Fmt::kBytes;
        if constexpr (Fmt::kPerChunk == 8)
            __builtin_amdgcn_raw_buffer_store_b16(static_cast<unsigned short>(w[e >> 1] >> (16 * (e & 1))), rs, off, 0,
                                                  0);
        else
            __builtin_amdgcn_raw_buffer_store_b32(w[e], rs, off, 0, 0);
    }
}

// A row of any length and alignment held in registers: chunk r * W + tid in
// round r of its `rounds` rounds (at most CPT).  Every round is a basic block of
// its own (a scalar branch: rounds past the row cost nothing), which also keeps the
// scheduler from holding the unpacked values of several rounds at once.  Only
// the last round holds padding.  Loads and stores go through a buffer
// descriptor: one offset register serves all rounds.  (tid: opaque_tid() in a loop
// over rows, or the offsets of every round are hoisted out of it and spilled.)
template <typename Fmt, int W, int CPT, int MINR = 1>
struct HeldRow {
    RowCut<Fmt> cut;
    int rounds;
    __device__ explicit HeldRow(int V) : cut(V), rounds((cut.nchunks + W - 1) / W) {}

    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int r = 0; r < CPT; ++r)
            if (r < MINR || r < rounds) {
                f(r);
                __builtin_amdgcn_sched_barrier(0);
            }
    }
    __device__ __forceinline__ void load(chunk_t (&c)[CPT], const void* row, int V, int tid) const {
        if (MINR == 1 && V < Fmt::kPerChunk) {
#pragma unroll
            for (int r = 0; r < CPT; ++r) c[r] = load_short<Fmt>(row, V);
            return;
        }
        const rsrc_t rs = make_rsrc(row, uint32_t(V) * Fmt::kBytes);
#pragma unroll
        for (int r = 0; r < CPT; ++r) {
            c[r] = chunk_t{0u, 0u, 0u, 0u};  // (or an earlier row's chunks stay live)
            if (r < MINR || r < rounds) {
                int off = (r * W + tid) * 16;
                if (r >= MINR - 1) off = min(off, cut.last_off);
                c[r] = __builtin_bit_cast(chunk_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, kStreamAux));
            }
        }
    }
    // Padding in place of what the last round holds past the row (and before
    // the last chunk's own elements).
    __device__ __forceinline__ void pad(chunk_t (&c)[CPT], int tid) const {
#pragma unroll
        for (int r = 0; r < CPT; ++r)
            if (r >= MINR - 1 && r == rounds - 1) c[r] = pad_lead<Fmt>(c[r], cut.lead(r * W + tid));
    }
    __device__ __forceinline__ void store(rsrc_t rs, int r, const chunk_t& c, int tid) const {
        store_chunk(cut, rs, r * W + tid, r < rounds - 1, c);
    }
};

// W * CPT chunks of a row from chunk `start` on, in a workgroup of W threads' registers: every
// round is loaded, past the row's end its last chunk, padded.
template <typename Fmt, int W, int CPT>
struct HeldSegment {
    RowCut<Fmt> cut;
    int start;
    bool whole;  // no padding in it
    __device__ HeldSegment(int V, int start) : cut(V), start(start), whole(start + CPT * W <= cut.nfull) {}
    template <int AUX>
    __device__ __forceinline__ void load(chunk_t (&c)[CPT], const void* row, int V, int tid) const {
        const rsrc_t rs = make_rsrc(row, uint32_t(V) * Fmt::kBytes);
#pragma unroll
        for (int r = 0; r < CPT; ++r)
            c[r] = __builtin_bit_cast(chunk_t, __builtin_amdgcn_raw_buffer_load_b128(
                                                   rs, min((start + r * W + tid) * 16, cut.last_off), 0, AUX));
    }
    __device__ __forceinline__ void pad(chunk_t (&c)[CPT], int tid) const {
        if (whole) return;
#pragma unroll
        for (int r = 0; r < CPT; ++r) c[r] = pad_lead<Fmt>(c[r], cut.lead(start + r * W + tid));
    }
    __device__ __forceinline__ void store(rsrc_t rs, int r, const chunk_t& c, int tid) const {
        store_chunk(cut, rs, start + r * W + tid, whole, c);
    }
};

// log2(e) / T, finite as a float however small T is; 0 at T == 0.
inline double scaled_log2e(float T) {
    if (T == 0.0f) return 0.0;
    const double c = 1.4426950408889634074 / double(T);
    return c < 3.0e38 ? c : 3.0e38;
}

}  // namespace osd
