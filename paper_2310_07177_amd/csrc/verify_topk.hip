// verify_topk.hip -- verification of proposals drawn from the draft's record
// (gfx950).
//
// Method: with q the softmax over the record's slots (0 elsewhere) and p the
// target's softmax over the whole row, proposal y_i is accepted when
// u q(y_i) < p(y_i), and the first rejection at row a draws from max(0, p - q)
// (Appendix A.1, Eq. 5).  p and max(0, p - q) differ at the record's tokens only,
// so the masses of a row's cells (256 chunks, 2048 bf16 or
// 1024 fp32 logits; in rows of more than 32 of these twice as many), known
// from the sums that normalise p, need no more than the record's corrections to
// place the draw in a cell, and one cell of row a is read again.
//
// One launch.  Workgroups of four waves: a wave takes one cell of a row 0 .. k_b
// (its largest logit and the sum of exponentials relative to it), or the record
// of one position (its normaliser, the proposal's q, the target's logits at its
// tokens).  They post what they found in the workspace, and the last of a sequence
// to arrive decides and draws.
//
// Precision: a cell's sum takes v_exp_f32 and is summed in fp64 from pairs up.
// A term is then off by at most kTerm = 1.8e-7 of itself: 8.5e-8 by the instruction (the
// most over every argument from -126 to 127), 6e-8 by the sum of a pair, 3.4e-8 by its
// argument.  (The rounding of (x - m) c2 alone would be 2 n ln 2 2^-24 of a term 2^-n,
// the same in equal terms: 1e-6 at n = 12.  bf16 logits have exact products with 16
// bits of c2, see cell_sum; the others take reduced arguments, see Near.)  With errors
// d_j of the terms the normaliser is off by D = sum p_j d_j, and the mass R_t up to a token
// that is left of p, less the point u R, by
//   E = (1 - u) sum_{j <= t} p_j e_j - u sum_{j > t} p_j e_j,
// e_j = d_j - D where the token keeps mass and d_j where the record takes all of it (its
// exact exponential is subtracted).  With A the mass of p up to the token, collecting d_j,
//   |E| <= kTerm (A (1 - u) + (1 - A) u + A (1 - A) + 2 c),
// where c is the mass of the cell that holds the token: its tokens are summed anew, with
// errors of their own (1.2e-7, and 6e-8 by rounding what the record leaves).
// A draw whose point lies within that of an edge of its token's interval is decided again
// on fp64 exponentials of the whole row (1e-12), and so is a test where u q / p and 1
// differ by less than kNearRatio (the normaliser is off by kTerm).  That holds up its
// sequence by 25 + 6 us at V = 128256, one draw in seventy (B = 256, K = 8, bf16: 120 us a
// call, 97 if none were), and by 7 + 4 us at V = 32128, one in two hundred (B = 64: 19.3 us a
// call, some 28 with one).  fp64 exponentials throughout took three times as long for the
// cells (20.6 us of the latter for them alone), reduced arguments in all cells 142 us; the
// record's tokens taken away by the sums' own exponentials, and a bound that gains by
// it, left four in five of these draws and cost 0.5 us of the 19.3.
#include "osd.h"
#include "osd_device.hpp"
#include "osd_internal.hpp"
#include "stream_device.hpp"
#include "topk_device.hpp"

namespace osd {
namespace {

constexpr int kW = 256, kNW = kW / kWave;
constexpr int kSlots = OSD_MAX_TOPK / kWave;
constexpr int kSlotPad = 8;       // (the row's last chunk reads up to 7 elements before its own)
constexpr int kTable = 1024;      // places for the ids of a record (at most 256)
constexpr double kTerm = 1.8e-7;
constexpr double kNearRatio = 2.0e-7;  // (kTerm and the roundings of fp64 ones)
// Workgroups per launch (a grid stays below 2^32 work-items).
constexpr int64_t kMaxGrid = int64_t(1) << 22;

struct VerifyTopkArgs {
    const char* target;
    const int32_t* ids;
    const char* top;
    int k;
    int K, V, cells;
    int groups;      // workgroups for the cells of one row
    int records;     // workgroups for the records of one sequence
    const int32_t* tokens;
    const int32_t* draft_len;
    const float* u_accept;
    const float* u_resample;
    double c2;
    float hi, lo, inv;   // c2 = hi + lo, 1 / c2; hi NaN where Near does not serve
    float hi16, lo16;    // c2 = hi16 + lo16, hi16 of 16 significant bits
    VerifyTopkRow* rows;
    int32_t* accepted_len;
    int32_t* out_tokens;
    uint8_t* reject_mask;
    int64_t first;   // first sequence of this launch
};

// What the workgroups of a sequence post, at the device-wide coherence point.
__device__ inline void post(double* p, double v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void post(float* p, float v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ inline T posted(const T* p) {
    return __hip_atomic_load(const_cast<T*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename Fmt>
__device__ inline chunk_t row_chunk(const char* row, int ch, const RowCut<Fmt>& cut, int V) {
    if (V < Fmt::kPerChunk) return ch == 0 ? load_short<Fmt>(row, V) : pad_chunk<Fmt>();
    return load_off(row, cut.off(ch));
}

// A cell is kPer chunks a lane of one wave.
template <typename Fmt, int kPer>
__device__ inline void load_cell(chunk_t (&c)[kPer], const char* row, int cell, const RowCut<Fmt>& cut, int V) {
    const int lane = threadIdx.x & (kWave - 1), ch0 = cell * kPer * kWave + lane;
#pragma unroll
    for (int r = 0; r < kPer; ++r) c[r] = row_chunk<Fmt>(row, ch0 + r * kWave, cut, V);
}

// 2^(x c2 - k) for logits x whose scaled value is at most k + 1, from 2^-120 on (what
// is smaller counts as that, and -inf too).  n = rint(x c2) and the rest
// r = x c2 - n come from x by multiply-adds, not from a rounded difference: with
// |k| < 2^20, r is off by 2^-25 + 2^-26 + 2^-28 at most (its roundings; c2 as a sum of two
// floats).  n - k lands in the low bits of `z` and is added to the exponent of 2^r.
constexpr float kLargestShift = 0x1p20f;
struct Near {
    float hi, lo, z, least, most;  // z: 1.5 * 2^23 - k
    __device__ Near(const VerifyTopkArgs& a, float k, float largest)
        : hi(a.hi), lo(a.lo), z(12582912.0f - k), least((k - 120.0f) * a.inv), most(largest) {}
    __device__ __forceinline__ float pow2(float x) const {
        x = __builtin_amdgcn_fmed3f(x, least, most);
        const float t = __builtin_fmaf(x, hi, z), n = t - z;
        const float r = __builtin_fmaf(x, lo, __builtin_fmaf(x, hi, -n));
        return __uint_as_float(__float_as_uint(exp2_fast(r)) + (__float_as_uint(t) << 23));
    }
};

// Wave total of floats, in every lane.
template <int CTRL, int ROWS>
__device__ inline float dpp_add_f32(float v) {
    return v + __uint_as_float(dpp_sum_src<CTRL, ROWS>(__float_as_uint(v)));
}
__device__ inline float wave_sum_f32(float v) {
    v = dpp_add_f32<kDppRowShr1, 0xF>(v);
    v = dpp_add_f32<kDppRowShr2, 0xF>(v);
    v = dpp_add_f32<kDppRowShr4, 0xF>(v);
    v = dpp_add_f32<kDppRowShr8, 0xF>(v);
    v = dpp_add_f32<kDppRowBcast15, 0xA>(v);
    v = dpp_add_f32<kDppRowBcast31, 0xC>(v);
    return readlane_f32(v, kWave - 1);
}

// The chunk with -inf replaced by the lowest finite bf16 value.
__device__ inline chunk_t finite_pairs(const chunk_t& c) {
    const auto f = [](uint32_t w) {
        w -= (w & 0xFFFF0000u) == 0xFF800000u ? 0x10000u : 0u;
        return w - ((w & 0xFFFFu) == 0xFF80u ? 1u : 0u);
    };
    return chunk_t{f(c.x), f(c.y), f(c.z), f(c.w)};
}

// The sum of a chunk's exponentials, in fp64 from pairs up.
template <int EPC>
__device__ __forceinline__ double pair_sum(const float (&e)[EPC]) {
    double s = double(e[0] + e[1]);
#pragma unroll
    for (int i = 2; i < EPC; i += 2) s += double(e[i] + e[i + 1]);
    return s;
}

// The chunk with its first `lead` elements replaced by the lowest finite bf16 value.
__device__ inline chunk_t lowest_lead(const chunk_t& c, int lead) {
    const auto w = [lead](uint32_t x, int e) {
        return lead > e + 1 ? 0xFF7FFF7Fu : (lead > e ? (x & 0xFFFF0000u) | 0xFF7Fu : x);
    };
    return chunk_t{w(c.x, 0), w(c.y, 2), w(c.z, 4), w(c.w, 6)};
}

// One cell by one wave: its largest logit m, and the sum S of exponentials (0 where
// there is no finite one), relative to m or, with the mean of the logits over their mass
// given (not NaN), as sum 2^(x hi16): 2^(mean lo16) S is then that of 2^(x c2).
template <typename Fmt, int kPer>
__device__ inline void cell_sum(const VerifyTopkArgs& a, chunk_t (&c)[kPer], int cell, const RowCut<Fmt>& cut, float& m,
                                double& S, float& mean) {
    constexpr int EPC = Fmt::kPerChunk;
    const int lane = threadIdx.x & (kWave - 1), ch0 = cell * kPer * kWave + lane;
    const bool end = (cell + 1) * kPer * kWave > cut.nfull;  // the row's end
    // (bf16: padding of the lowest finite value serves the path that is taken most.)
    if (end) {
#pragma unroll
        for (int r = 0; r < kPer; ++r) {
            const int lead = cut.lead(ch0 + r * kWave);
            if constexpr (EPC == 8)
                c[r] = lowest_lead(c[r], lead);
            else
                c[r] = pad_lead<Fmt>(c[r], lead);
        }
    }
    const auto largest = [&] {
        float x = kNegInf;
        if constexpr (EPC == 8) {
            // Pairs of bf16 patterns as f16 numbers, see chunks_max (which drops a NaN).
            typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
            h2_t h = __builtin_bit_cast(h2_t, c[0].x);
#pragma unroll
            for (int i = 1; i < 4 * kPer; ++i)
                h = __builtin_elementwise_maximum(h, __builtin_bit_cast(h2_t, uint32_t(c[i / 4][i % 4])));
            const uint32_t b = __builtin_bit_cast(uint32_t, h);
            x = max_nan(__uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u));
            if (__ballot(!(__builtin_fabsf(x) < 0x1p121f)) == 0) return wave_max_nan(x);
            x = kNegInf;
        }
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int e = 0; e < EPC; ++e) x = max_nan(x, Fmt::get(c[r], e));
        opaque<kPer>(c);
        return wave_max_nan(x);
    };
    m = largest();
    S = 0.0;
    mean = __builtin_nanf("");
    if constexpr (EPC == 8) {
        // x hi16 is exact (8 bits times 16), so v_exp_f32 takes it as it is.  What lo16 adds,
        // a factor 2^(x lo16), is taken for the cell at the mean of x over its mass: off by
        // half the variance of x lo16 ln 2 there, 2e-9 for halves 24 octaves apart.
        // (Largest logits of 2^-60 to 2^100 leave the others their range.)
        const float h = m * a.hi16;
        if (h >= -60.0f && h <= 100.0f) {
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {
                float X = 0.0f;
                S = 0.0;
#pragma unroll
                for (int r = 0; r < kPer; ++r) {
                    float e8[EPC];
#pragma unroll
                    for (int e = 0; e < EPC; ++e) {
                        const float x = Fmt::get(c[r], e);
                        e8[e] = exp2_fast(x * a.hi16);
                        X = __builtin_fmaf(e8[e], x, X);
                    }
                    S += pair_sum<EPC>(e8);
                    __builtin_amdgcn_sched_barrier(0);
                }
                S = wave_sum(S);
                mean = wave_sum_f32(X) * __builtin_amdgcn_rcpf(float(S));
                if (is_finite(mean)) return;
                // A -inf (times 0): again with the lowest finite value in its place.  (Or X
                // overflows, with logits of 1e10 at such temperatures: the other ways.)
#pragma unroll
                for (int r = 0; r < kPer; ++r) c[r] = finite_pairs(c[r]);
            }
            S = 0.0;
            mean = __builtin_nanf("");
        }
        if (end) {
#pragma unroll
            for (int r = 0; r < kPer; ++r) c[r] = pad_lead<Fmt>(c[r], cut.lead(ch0 + r * kWave));
            m = largest();
        }
    }
    if (!is_finite(m)) return;
    const float k = __builtin_rintf(m * a.hi);
    if (!(__builtin_fabsf(k) < kLargestShift)) {
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                S += exp2_f64((double(Fmt::get(c[r], e)) - double(m)) * a.c2);
                if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // few registers
            }
        S = wave_sum(S);
        return;
    }
    const Near near(a, k, m);
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        float e8[EPC];
#pragma unroll
        for (int e = 0; e < EPC; ++e) e8[e] = near.pow2(Fmt::get(c[r], e));
        S += pair_sum<EPC>(e8);
        __builtin_amdgcn_sched_barrier(0);
    }
    S = wave_sum(S) * exp2_f64(double(k) - double(m) * a.c2);
}

struct VerifyTopkLds {
    union {
        int32_t table[kNW][kTable];            // ids seen, by wave
        uint16_t slot[kSlotPad + 512 * 8 + 8];  // 1 + the slot of each token of one cell, or 0
    };
    double row_sum[OSD_MAX_K + 1];             // target rows: normaliser
    float row_top[OSD_MAX_K + 1];              //              largest logit, NaN or -inf if unusable
    int verdict[OSD_MAX_K + 1];                // 0 accepted, 1 stop here, 2 invalid, 3 too near to tell
    double row_t[OSD_MAX_K + 1];               // for the last: the target's exponential times q_sum,
    double row_uq[OSD_MAX_K + 1];              //               u times the draft's
    int id[OSD_MAX_TOPK];                      // the record at the first rejection: token (-1: none),
    double q[OSD_MAX_TOPK];                    // q, and
    double e[OSD_MAX_TOPK];                    // the target's exponential
    uint64_t fixed[kMaxCells];                 // corrections by cell, 2^-62
    double sum[kMaxCells];                     // the drawn row's cells
    double wave[kNW], low, high;
    int hit[kNW], last, token;
    int stop, invalid, is_last;
};

// Totals over each half of the wave, in all its lanes.
__device__ inline double half_sum(double v) {
    v = dpp_add_step<kDppRowShr1, 0xF>(v);
    v = dpp_add_step<kDppRowShr2, 0xF>(v);
    v = dpp_add_step<kDppRowShr4, 0xF>(v);
    v = dpp_add_step<kDppRowShr8, 0xF>(v);
    v = dpp_add_step<kDppRowBcast15, 0xA>(v);
    const double lo = readlane_f64(v, 31), hi = readlane_f64(v, 63);
    return (threadIdx.x & 32) ? hi : lo;
}
__device__ inline float half_max_nan(float x) {
    uint32_t k = order_key(x);
    k = dpp_umax_step<kDppRowShr1, 0xF>(k);
    k = dpp_umax_step<kDppRowShr2, 0xF>(k);
    k = dpp_umax_step<kDppRowShr4, 0xF>(k);
    k = dpp_umax_step<kDppRowShr8, 0xF>(k);
    k = dpp_umax_step<kDppRowBcast15, 0xA>(k);
    const uint32_t lo = readlane_u32(k, 31), hi = readlane_u32(k, 63);
    return key_float((threadIdx.x & 32) ? hi : lo);  // (the largest key is a NaN's pattern too)
}

// The record of one position by one wave, posted: the softmax's reference and
// normaliser (0: no record), the proposal's q, the target's logits at the
// record's tokens and at the proposal.
template <typename Fmt>
__device__ inline void post_record(const VerifyTopkArgs& a, int64_t b, int i, int32_t* table, VerifyTopkRow& out) {
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t pos = b * a.K + i;
    const char* row = a.target + (b * (a.K + 1) + i) * a.V * Fmt::kBytes;
    const int y = a.tokens[pos];
    int id[kSlots];
    float x[kSlots], m = kNegInf;
    bool ok = true;
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
        const int s = j * kWave + lane;
        id[j] = s < a.k ? a.ids[pos * a.k + s] : -1;
        x[j] = s < a.k ? Fmt::load_one(a.top + pos * a.k * Fmt::kBytes, s) : kNegInf;
    }
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
        const int s = j * kWave + lane;
        if (id[j] < -1 || id[j] >= a.V) {
            ok = false;
            id[j] = -1;
        }
        if (id[j] >= 0) {
            ok = ok && x[j] < -kNegInf;
            post(&out.slot[s], Fmt::load_one(row, id[j]));
        } else {
            x[j] = kNegInf;
        }
        m = fmaxf(m, x[j]);
    }
    m = wave_max(m);
    ok = ok && m > kNegInf;
    double q[kSlots], s = 0.0, mine = 0.0;
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
        q[j] = x[j] > kNegInf ? exp2_f64((double(x[j]) - double(m)) * a.c2) : 0.0;
        s += q[j];
        if (id[j] == y) mine += q[j];
    }
    s = wave_sum(s);
    mine = wave_sum(mine);
    // An id twice: its place in the table is taken by an equal one.
#pragma unroll
    for (int t = 0; t < kTable / kWave; ++t) table[t * kWave + lane] = -1;
    wave_lds_order();
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
        if (id[j] < 0) continue;
        int h = int((uint32_t(id[j]) * 2654435761u) >> 22);
        for (int t = 0; t < kTable; ++t) {
            const int old = atomicCAS(&table[h], -1, id[j]);
            if (old == -1) break;
            if (old == id[j]) {
                ok = false;
                break;
            }
            h = (h + 1) & (kTable - 1);
        }
    }
    ok = __ballot(!ok) == 0;
    if (lane == 0) {
        const float t = y >= 0 && y < a.V ? Fmt::load_one(row, y) : __builtin_nanf("");
        post(&out.q_top, m);
        post(&out.q_sum, ok ? s : 0.0);
        post(&out.q_token, mine);
        post(&out.t_token, t);
    }
}

// The drawn row, in every thread.
struct Draw {
    const char* row;
    double top, sum, inv;  // largest logit, normaliser and its reciprocal
    float k;          // Near's shift
    double unit;      // and the probability mass of one of its units
    double point;     // in probability mass
    double u;
    double cum;       // lane c: mass up to and with cell c
    double before;    // the same of p alone
    uint64_t lives;   // cells with mass
    bool with_q;      // the residual, or p alone
};

// The smallest token whose running mass exceeds the point; the last one with mass
// if rounding put the point past it (-1: none has).  sure: the point is further from both
// edges of the token's interval than these may be off.
template <typename Fmt, int kPer, bool EXACT>
__device__ __forceinline__ int find_token(const VerifyTopkArgs& a, const Draw& d, VerifyTopkLds& s, bool& sure) {
    constexpr int EPC = Fmt::kPerChunk, kCell = kPer * kWave, kEach = kCell / kW, kTokens = kCell * EPC;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    const RowCut<Fmt> cut(a.V);
    const Near near(a, d.k, float(d.top));
    const double per = 1.0 / d.unit;
    // The first cell that may hold the point (the sums of the cells and of their
    // elements differ by rounding), then upwards; down from there only if rounding
    // put the point past the last token.
    sure = false;
    if (d.lives == 0) return -1;  // (no cell to read)
    const uint64_t from = __ballot((d.lives >> lane & 1) && d.cum > d.point - 1e-14);
    int cell = from ? __builtin_ctzll(from) : 63 - __builtin_clzll(d.lives);
    const int start = cell;
    bool up = true;
    while (true) {
        const int ch0 = cell * kCell + tid * kEach;
        chunk_t c[kEach];
#pragma unroll
        for (int n = 0; n < kEach; ++n) c[n] = row_chunk<Fmt>(d.row, ch0 + n, cut, a.V);
        double base = cell > 0 ? readlane_f64(d.cum, cell - 1) : 0.0;
        const bool mine = d.with_q && tid < a.k && s.id[tid] / kTokens == cell && s.id[tid] >= 0;
        const int at = mine ? s.id[tid] - cell * kTokens : 0;
        if (mine) s.slot[kSlotPad + at] = uint16_t(tid + 1);
        if (tid == 0) s.last = -1;
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kEach; ++n) c[n] = pad_lead<Fmt>(c[n], cut.lead(ch0 + n));
        // The masses of the thread's tokens in d.unit: of p, then without the record's part
        // (few threads hold any of it).  In fp64 they are taken again when needed.
        float w[EXACT ? 1 : kEach * EPC];
        if constexpr (!EXACT) {
#pragma unroll
            for (int n = 0; n < kEach; ++n) {
                const int first = cut.token((ch0 + n) * EPC);
                const uint16_t* slots = s.slot + (first - cell * kTokens + kSlotPad);
                int slot[EPC], any = 0;
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    slot[e] = slots[e];
                    any |= slot[e];
                    w[n * EPC + e] = near.pow2(Fmt::get(c[n], e));
                }
                if (any) {
#pragma unroll
                    for (int e = 0; e < EPC; ++e)
                        if (slot[e]) w[n * EPC + e] = float(fmax(double(w[n * EPC + e]) - s.q[slot[e] - 1] * per, 0.0));
                }
            }
        }
        // f(token, mass) for the thread's tokens in order.
        const auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < kEach; ++n) {
                const int first = cut.token((ch0 + n) * EPC);
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    if constexpr (EXACT) {
                        const float t = Fmt::get(c[n], e);
                        if (t > kNegInf) {
                            double p = exp2_f64((double(t) - d.top) * a.c2) * d.inv;
                            const int slot = s.slot[first + e - cell * kTokens + kSlotPad];
                            if (slot) p = fmax(p - s.q[slot - 1], 0.0);
                            f(first + e, p);
                        }
                        __builtin_amdgcn_sched_barrier(0);  // few registers
                    } else {
                        f(first + e, double(w[n * EPC + e]) * d.unit);
                    }
                }
            }
        };
        double run = 0.0;
        int lastpos = -1;
        each([&](int token, double p) __attribute__((always_inline)) {
            run += p;
            if (p > 0.0) lastpos = token;
        });
        const double upto = wave_scan_add(run);
        if (lane == kWave - 1) s.wave[wid] = upto;
        if (lastpos >= 0 && __ballot(lastpos >= 0) >> lane == 1) atomicMax(&s.last, lastpos);
        __syncthreads();
        for (int i = 0; i < wid; ++i) base += s.wave[i];
        base += upto - run;
        const uint64_t past = __ballot(run > 0.0 && base + run > d.point);
        if (lane == 0) s.hit[wid] = past ? wid * kWave + __builtin_ctzll(past) : 0x7FFFFFFF;
        __syncthreads();
        int hit = s.hit[0];
        for (int i = 1; i < kNW; ++i) hit = min(hit, s.hit[i]);
        if (tid == hit) {  // the first thread whose tokens reach past the point
            int token = -1;
            double low = 0.0, high = 0.0;
            each([&](int t, double p) __attribute__((always_inline)) {
                if (token < 0 && p > 0.0) {
                    low = base;
                    high = base + p;
                    if (high > d.point) token = t;
                }
                base += p;
            });
            s.token = token >= 0 ? token : lastpos;
            s.low = low;
            s.high = high;
        }
        __syncthreads();
        if (mine) s.slot[kSlotPad + at] = 0;
        if (up && hit != 0x7FFFFFFF) {
            // (The edges lie in this cell: the largest bound over A there.)
            const double from = cell > 0 ? readlane_f64(d.before, cell - 1) : 0.0, to = readlane_f64(d.before, cell);
            const double A = fmin(fmax(1.0 - d.u, from), to);
            const double unsure =
                kTerm * (A * (1.0 - d.u) + (1.0 - A) * d.u + A * (1.0 - A) + 2.0 * (to - from)) + 1e-11;
            sure = s.high - d.point > unsure && d.point - s.low > unsure;
            return s.token;
        }
        const int last = s.last;
        const uint64_t more = d.lives & ~((2ull << cell) - 1);
        if (up && more) {
            cell = __builtin_ctzll(more);
        } else {
            if (last >= 0) return last;
            if (up) cell = start;
            up = false;
            const uint64_t fewer = d.lives & ((1ull << cell) - 1);
            if (!fewer) return -1;
            cell = 63 - __builtin_clzll(fewer);
        }
        __syncthreads();
    }
}

// log2 of what a posted sum of a cell counts relative to a row's largest logit.
template <int EPC>
__device__ inline double cell_scale(const VerifyTopkArgs& a, float m, float mean, float top) {
    if (EPC == 8 && mean == mean) return double(mean) * double(a.lo16) - double(top) * a.c2;
    return (double(m) - double(top)) * a.c2;
}

// The sums of a row's cells from fp64 exponentials relative to the row's largest logit,
// by the whole workgroup (0 past the last cell; barriers inside and at the end).  Small
// code, and the next chunks on their way: a row of 128256 bf16 logits takes 25 us, and 40 with
// one chunk on its way.
template <typename Fmt, int kPer>
__device__ __forceinline__ void exact_cells(const VerifyTopkArgs& a, const char* row, double top, VerifyTopkLds& s) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    const RowCut<Fmt> cut(a.V);
    if (tid < kMaxCells) s.sum[tid] = 0.0;
    __syncthreads();
    const auto chunk = [&](int i) { return ((i / kPer * kNW + wid) * kPer + i % kPer) * kWave + lane; };
    const int n = a.cells > wid ? ((a.cells - 1 - wid) / kNW + 1) * kPer : 0;
    // (A row shorter than one chunk: nothing is read, and all but chunk 0 is padding.)
    const bool tiny = a.V < Fmt::kPerChunk;
    const rsrc_t rs = make_rsrc(row, tiny ? 0u : uint32_t(a.V) * Fmt::kBytes);
    const auto load = [&](int i) {
        return __builtin_bit_cast(chunk_t, __builtin_amdgcn_raw_buffer_load_b128(rs, cut.off(chunk(i)), 0, 0));
    };
    constexpr int kRing = 4;
    static_assert(kPer % kRing == 0, "");
    chunk_t ahead[kRing];
#pragma unroll
    for (int j = 0; j < kRing; ++j) ahead[j] = load(j);
    if (tiny) ahead[0] = load_short<Fmt>(row, a.V);
    double S = 0.0;
#pragma unroll 1
    for (int i = 0; i < n; i += kRing) {
#pragma unroll
        for (int j = 0; j < kRing; ++j) {
            const chunk_t x = pad_lead<Fmt>(ahead[j], cut.lead(chunk(i + j)));
            ahead[j] = load(i + j + kRing);
#pragma unroll
            for (int e = 0; e < Fmt::kPerChunk; ++e) S += exp2_f64((double(Fmt::get(x, e)) - top) * a.c2);
        }
        if ((i + kRing) % kPer == 0) {
            S = wave_sum(S);
            if (lane == 0) s.sum[i / kPer * kNW + wid] = S;
            S = 0.0;
        }
    }
    __syncthreads();
}

// The last workgroup of a sequence: the tests, the first rejection, the draw.
template <typename Fmt, int kPer>
__device__ __forceinline__ void decide(const VerifyTopkArgs& a, int64_t b, int kb, VerifyTopkLds& s) {
    constexpr int EPC = Fmt::kPerChunk, kTokens = kPer * kWave * EPC;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    const int K = a.K;
    VerifyTopkRow* rows = a.rows + b * (K + 1);
    const int32_t* y = a.tokens + b * K;
    const int token = lane < kb ? y[lane] : 0;  // position lane's proposal
    // Half a wave per row, two rows after another; all that was posted of them is
    // requested at once.
    constexpr int kBatch = 2, kRows = 2 * kNW;
    const int cell = lane & 31;
#pragma unroll 1
    for (int i0 = 2 * wid + (lane >> 5); i0 - (lane >> 5) <= kb; i0 += kBatch * kRows) {
        float m[kBatch], t[kBatch], u[kBatch], mean[kBatch];
        double v[kBatch], qs[kBatch], qt[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = min(i0 + j * kRows, kb);
            const VerifyTopkRow& r = rows[i];
            const bool rec = i < kb;
            m[j] = cell < a.cells ? posted(&r.top[cell]) : kNegInf;
            v[j] = cell < a.cells ? posted(&r.sum[cell]) : 0.0;
            mean[j] = EPC == 8 && cell < a.cells ? posted(&r.mean[cell]) : __builtin_nanf("");
            qs[j] = rec ? posted(&r.q_sum) : 1.0;
            qt[j] = rec ? posted(&r.q_token) : 0.0;
            t[j] = rec ? posted(&r.t_token) : 0.0f;
            u[j] = rec ? a.u_accept[b * K + i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = i0 + j * kRows;
            const float top = half_max_nan(m[j]);
            const double sum = half_sum(v[j] * exp2_f64(cell_scale<EPC>(a, m[j], mean[j], top)));
            int verdict = 1;
            if (!is_finite(top) || t[j] != t[j] || !(qs[j] > 0.0))
                verdict = 2;
            else if (i < kb) {  // u q / q_sum < p / sum
                const double p = t[j] > kNegInf ? exp2_f64((double(t[j]) - double(top)) * a.c2) : 0.0;
                const double uq = double(u[j]) * qt[j], pq = p * qs[j];
                verdict = __builtin_fabs(uq * sum - pq) < kNearRatio * pq ? 3 : uq * sum < pq ? 0 : 1;
                if (verdict == 3 && cell == 0) {
                    s.row_t[i] = pq;
                    s.row_uq[i] = uq;
                }
            }
            // (A proposal outside the vocabulary, wherever it is, is caught below.)
            if (cell == 0 && i <= kb) {
                s.row_top[i] = top;
                s.row_sum[i] = sum;
                s.verdict[i] = verdict;
            }
        }
    }
    if (tid < kMaxCells) s.fixed[tid] = 0;
    static_assert((kSlotPad + kTokens + 8) * sizeof(s.slot[0]) <= sizeof(s.slot), "a cell's tokens and the padding");
    for (int i = tid; i < (kSlotPad + kTokens + 8) / 2; i += kW) reinterpret_cast<uint32_t*>(s.slot)[i] = 0u;
    __syncthreads();
    // The first position that is not accepted.  Where the sums of v_exp_f32 do not tell,
    // on fp64 exponentials of its row.
    int v, acc;
#pragma unroll 1
    while (true) {
        v = lane <= kb ? s.verdict[lane] : 1;
        acc = __builtin_ctzll(__ballot(v != 0));
        if (__builtin_amdgcn_readlane(v, acc) != 3) break;
        exact_cells<Fmt, kPer>(a, a.target + (b * (K + 1) + acc) * a.V * Fmt::kBytes, double(s.row_top[acc]), s);
        const double sum = half_sum(s.sum[cell]);
        __syncthreads();
        if (tid == 0) s.verdict[acc] = s.row_uq[acc] * sum < s.row_t[acc] ? 0 : 1;
        __syncthreads();
    }
    bool invalid = __ballot(token < 0 || token >= a.V) != 0 || __builtin_amdgcn_readlane(v, acc) == 2;
    int extra = -1;
    if (!invalid) {
        const bool rejected = acc < kb;
        const VerifyTopkRow& r = rows[acc];
        Draw d;
        d.row = a.target + (b * (K + 1) + acc) * a.V * Fmt::kBytes;
        d.top = double(s.row_top[acc]);
        d.sum = s.row_sum[acc];
        d.inv = 1.0 / d.sum;
        // Slot s by thread s: q, and what of p it takes away from its cell.
        const auto correct = [&] {
            if (s.id[tid] >= 0)
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.fixed[s.id[tid] / kTokens]),
                          (unsigned long long)(fmin(s.e[tid] * d.inv, s.q[tid]) * 0x1p62));
        };
        const float m = cell < a.cells ? posted(&r.top[cell]) : kNegInf;
        const float mean = EPC == 8 && cell < a.cells ? posted(&r.mean[cell]) : __builtin_nanf("");
        double S = cell < a.cells ? posted(&r.sum[cell]) : 0.0;
        if (rejected && tid < a.k) {
            const int64_t pos = b * K + acc;
            const int id = a.ids[pos * a.k + tid];
            const float x = Fmt::load_one(a.top + pos * a.k * Fmt::kBytes, tid), t = posted(&r.slot[tid]);
            const double ref = double(posted(&r.q_top)), qs = posted(&r.q_sum);
            s.id[tid] = id;
            s.q[tid] = x > kNegInf ? exp2_f64((double(x) - ref) * a.c2) / qs : 0.0;
            s.e[tid] = id >= 0 && t > kNegInf ? exp2_f64((double(t) - d.top) * a.c2) : 0.0;
            correct();
        }
        d.u = double(a.u_resample[b]);
        __syncthreads();
        double weight = exp2_f64(cell_scale<EPC>(a, m, mean, float(d.top)));
        const auto masses = [&] {  // lane c < 32 of every wave: cell c
            const double mass = lane < kMaxCells ? S * weight * d.inv : 0.0;
            d.lives = __ballot(mass > 0.0);
            d.with_q = rejected;
            d.before = wave_scan_add(mass);
            d.cum = wave_scan_add(fmax(mass - double(s.fixed[cell]) * 0x1p-62, 0.0));
            if (readlane_f64(d.cum, kWave - 1) <= 0.0) {  // rounding left nothing: from p
                d.cum = d.before;
                d.with_q = false;
            }
            d.point = d.u * readlane_f64(d.cum, kWave - 1);
        };
        masses();
        bool sure = false;
        d.k = __builtin_rintf(s.row_top[acc] * a.hi);
        // (Nothing left of p by these sums: fp64 ones have to say so before p is drawn from.)
        if (d.with_q == rejected && __builtin_fabsf(d.k) < kLargestShift) {
            d.unit = exp2_f64(double(d.k) - d.top * a.c2) * d.inv;
            extra = find_token<Fmt, kPer, false>(a, d, s, sure);
        }
        if (!sure) {  // again with fp64 exponentials
            __syncthreads();
            if (tid < kMaxCells) s.fixed[tid] = 0;
            exact_cells<Fmt, kPer>(a, d.row, d.top, s);
            S = s.sum[cell];
            weight = 1.0;
            d.sum = half_sum(S);
            d.inv = 1.0 / d.sum;
            if (rejected && tid < a.k) correct();
            __syncthreads();
            masses();
            extra = find_token<Fmt, kPer, true>(a, d, s, sure);
        }
        invalid = extra < 0;
    }
    if (tid <= K) {
        const int64_t o = b * (K + 1) + tid;
        a.out_tokens[o] = invalid || tid > acc ? -1 : (tid == acc ? extra : token);
        if (tid == 0) a.accepted_len[b] = invalid ? -1 : acc;
        if (a.reject_mask && tid < K) a.reject_mask[b * K + tid] = !invalid && tid == acc && acc < kb ? 1 : 0;
    }
}

template <typename Fmt, int kPer>
__global__ __launch_bounds__(kW, kPer == 4 ? 5 : 4) void verify_topk_kernel(VerifyTopkArgs a) {
    __shared__ VerifyTopkLds s;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int K = a.K;
    const uint32_t per = uint32_t(a.records + (K + 1) * a.groups);
    const uint32_t seq = blockIdx.x / per, unit = blockIdx.x - seq * per;
    const int64_t b = a.first + seq;
    const int kb = a.draft_len ? a.draft_len[b] : K;
    if (kb < 1 || kb > K) {
        if (unit == 0 && tid <= K) {
            a.out_tokens[b * (K + 1) + tid] = -1;
            if (tid == 0) a.accepted_len[b] = -1;
            if (a.reject_mask && tid < K) a.reject_mask[b * K + tid] = 0;
        }
        return;
    }
    VerifyTopkRow* rows = a.rows + b * (K + 1);
    if (unit < uint32_t(a.records)) {
        const int i = int(unit) * kNW + wid;
        if (i < kb) post_record<Fmt>(a, b, i, s.table[wid], rows[i]);
    } else {
        const uint32_t u = unit - uint32_t(a.records);
        const int i = int(u / uint32_t(a.groups)), g = int(u - uint32_t(i) * uint32_t(a.groups));
        if (i > kb) return;
        const RowCut<Fmt> cut(a.V);
        const char* x = a.target + (b * (K + 1) + i) * a.V * Fmt::kBytes;
        const int cell = g * kNW + wid;
        if (cell < a.cells) {
            chunk_t c[kPer];
            float m, mean;
            double S;
            load_cell<Fmt, kPer>(c, x, cell, cut, a.V);
            cell_sum<Fmt, kPer>(a, c, cell, cut, m, S, mean);
            if (lane == 0) {
                post(&rows[i].sum[cell], S);
                if constexpr (Fmt::kPerChunk == 8) post(&rows[i].mean[cell], mean);
                post(&rows[i].top[cell], m);
            }
        }
    }
    // A wave's posts are in place before the workgroup's arrival is issued.
    wait_memory();
    __syncthreads();
    if (tid == 0) s.is_last = arrive(&rows[0].arrivals) == uint32_t(a.records + (kb + 1) * a.groups) - 1;
    __syncthreads();
    if (!s.is_last) return;
    if (tid == 0) __hip_atomic_store(&rows[0].arrivals, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    decide<Fmt, kPer>(a, b, kb, s);
}

template <typename Fmt, int kPer>
hipError_t launch_cells(const VerifyTopkLaunch& L, VerifyTopkArgs a, int chunks) {
    a.cells = (chunks + kPer * kWave - 1) / (kPer * kWave);
    if (a.cells > kMaxCells) return hipErrorInvalidValue;
    a.records = (a.K + kNW - 1) / kNW;
    a.groups = (a.cells + kNW - 1) / kNW;
    const int64_t per = a.records + int64_t(a.K + 1) * a.groups, most = kMaxGrid / per;
    for (int64_t f = 0; f < L.B; f += most) {
        a.first = f;
        const unsigned g = unsigned((L.B - f < most ? L.B - f : most) * per);
        const hipError_t e = launch_kernel(&verify_topk_kernel<Fmt, kPer>, dim3(g), dim3(kW), 0, L.stream, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename Fmt>
hipError_t launch_fmt(const VerifyTopkLaunch& L, const VerifyTopkArgs& a) {
    const int chunks = (L.V + Fmt::kPerChunk - 1) / Fmt::kPerChunk;
    return chunks <= kMaxCells * 4 * kWave ? launch_cells<Fmt, 4>(L, a, chunks) : launch_cells<Fmt, 8>(L, a, chunks);
}

}  // namespace

hipError_t launch_verify_topk(const VerifyTopkLaunch& L) {
    VerifyTopkArgs a{};
    a.target = static_cast<const char*>(L.target);
    a.ids = L.ids;
    a.top = static_cast<const char*>(L.top);
    a.k = L.k;
    a.K = L.K;
    a.V = L.V;
    a.tokens = L.tokens;
    a.draft_len = L.draft_len;
    a.u_accept = L.u_accept;
    a.u_resample = L.u_resample;
    a.c2 = scaled_log2e(L.temperature);
    // (Where T or 1 / T is beyond 1e30 fp64 serves alone.)
    a.hi = a.c2 > 1e-30 && a.c2 < 1e30 ? float(a.c2) : __builtin_nanf("");
    a.lo = float(a.c2 - double(a.hi));
    a.inv = float(1.0 / a.c2);
    const uint32_t bits = __builtin_bit_cast(uint32_t, float(a.c2));
    a.hi16 = a.hi == a.hi ? __builtin_bit_cast(float, (bits + 0x80u) & 0xFFFFFF00u) : a.hi;
    a.lo16 = float(a.c2 - double(a.hi16));
    a.rows = L.rows;
    a.accepted_len = L.accepted_len;
    a.out_tokens = L.out_tokens;
    a.reject_mask = L.reject_mask;
    return L.dtype == 1 ? launch_fmt<BF16>(L, a) : launch_fmt<F32>(L, a);
}

}  // namespace osd
