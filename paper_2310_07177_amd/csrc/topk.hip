// topk.hip -- the record of a row's top logits, and a token drawn from it
// (gfx950).
//
// Method: one workgroup streams a row once.  Each thread keeps, for each of up to
// sixteen groups of its chunks, the largest logit and the sum of exponentials.  The
// k-th largest of the threads' maxima (to 16 bits of the ordered key, by a
// histogram of one wave) is at most the k-th largest logit, since k threads met an
// element that large; so the elements at or above it, the candidates, are all the
// record can hold, and there are few more than k of them.  Each wave looks through the
// groups of its threads that reach the threshold once more, an element a lane, and
// picks the candidates; these are grouped by key and ranked within their group by
// counting, so the record does not depend on the order of their arrival.  A row with
// more candidates than LDS holds (many equal logits, as a finite value in masked places
// where fewer than k are left; the largest ones side by side; k near the 256 threads of
// a short row) gets the exact k-th (logit, id) by bisection over the row first, some 55
// times over it: 576 rows of 8000 bf16 logits 10 us at k = 64, 22 at 240, 194 at 256; 64
// rows of 128256, ten of them not the type's lowest, 949 us, and 15 of ordinary ones.
//
// The mass of the tokens outside the record is the sum over the groups below the
// threshold, what the others hold besides candidates, and the candidates that were
// not taken: nothing is subtracted, so it keeps its relative accuracy down to 2^-60 of the
// largest logit's; below that it is summed over the row once more, relative to the
// largest logit outside.  The draw sums fp64 exponentials of the record's logits.
//
// What bounds it in bulk is instruction issue: a row of 64 KB arrives at a CU in 2.7
// us, in which its four SIMDs issue some 6500 vector instructions, and the sweep
// over 32128 logits takes 2700 (unpacking, one multiply-add, exponential and add an
// element, maxima two elements an instruction).  So everything else is kept to few
// waves and few instructions: rows held in registers (two sweeps, half the waves
// a CU) with the candidates collected from them and ranked by comparing all pairs
// took twice as many instructions, and 2048 rows of 128256 bf16 logits 232 us.
#include <utility>

#include "osd.h"
#include "osd_device.hpp"
#include "osd_internal.hpp"
#include "stream_device.hpp"
#include "topk_device.hpp"

namespace osd {
namespace {

constexpr int kCap = 1024;   // candidates that LDS holds
constexpr int kQueue = 128;  // groups of one wave's queue
constexpr int kBins = 256;   // 16-bit keys of one histogram
constexpr int kAhead = 8;    // chunks a thread requests ahead
// Workgroups per launch (a grid stays below 2^32 work-items).
constexpr int64_t kMaxGrid = int64_t(1) << 21;

struct TopkArgs {
    const char* x;
    int64_t stride;  // bytes between rows
    int V, k;
    double c2;       // log2(e) / T, 0 at T == 0
    const float* u;
    int32_t* ids;
    void* top;
    float* rest;
    int32_t* tokens;
    int64_t first;  // first row of this launch
};

template <int W>
struct TopkLds {
    union {
        int queue[W / kWave][kQueue];  // groups to look through, by wave
        uint64_t sorted[kCap];         // the candidates in order
    };
    uint64_t cand[kCap];
    uint32_t key[W];             // the threads' maxima
    uint32_t bin[kBins];         // counts, then where each bin's candidates begin
    uint32_t fill[kBins];
    double sum[W / kWave];
    uint32_t maxkey, tkey, ncand, count, far;
};

// Candidates come first: larger logit, then lower id.
__device__ inline uint64_t composite(uint32_t key, int token) { return (uint64_t(key) << 32) | uint32_t(~token); }

// Inclusive scan of 32-bit counts over the wave.
template <int CTRL, int ROWS>
__device__ inline uint32_t dpp_count_step(uint32_t v) {
    return v + dpp_sum_src<CTRL, ROWS>(v);
}
__device__ inline uint32_t wave_scan_count(uint32_t v) {
    v = dpp_count_step<kDppRowShr1, 0xF>(v);
    v = dpp_count_step<kDppRowShr2, 0xF>(v);
    v = dpp_count_step<kDppRowShr4, 0xF>(v);
    v = dpp_count_step<kDppRowShr8, 0xF>(v);
    v = dpp_count_step<kDppRowBcast15, 0xA>(v);
    v = dpp_count_step<kDppRowBcast31, 0xC>(v);
    return v;
}
__device__ inline uint32_t wave_max_key(uint32_t k) {
    k = dpp_umax_step<kDppRowShr1, 0xF>(k);
    k = dpp_umax_step<kDppRowShr2, 0xF>(k);
    k = dpp_umax_step<kDppRowShr4, 0xF>(k);
    k = dpp_umax_step<kDppRowShr8, 0xF>(k);
    k = dpp_umax_step<kDppRowBcast15, 0xA>(k);
    k = dpp_umax_step<kDppRowBcast31, 0xC>(k);
    return readlane_u32(k, kWave - 1);
}
// A value that every lane holds.
__device__ inline uint32_t uniform(uint32_t v) { return uint32_t(__builtin_amdgcn_readfirstlane(int(v))); }
// The lane's place among those of a ballot.
__device__ inline uint32_t lanes_below(uint64_t ballot) {
    return __builtin_amdgcn_mbcnt_hi(uint32_t(ballot >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(ballot), 0u));
}

// The candidates in order, by the whole workgroup: grouped by the 256 16-bit
// keys from the largest down (the last group holds all below), and each
// ranked within its group by counting.  (cand is complete; barriers inside and
// at the end.)
template <int kW>
__device__ __forceinline__ void sort_candidates(TopkLds<kW>& s, int nc, uint32_t maxkey) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const auto group = [&](uint64_t v) { return min((maxkey >> 16) - uint32_t(v >> 48), uint32_t(kBins - 1)); };
    if (tid < kBins) s.bin[tid] = s.fill[tid] = 0u;
    __syncthreads();
    for (int i = tid; i < nc; i += kW) atomicAdd(&s.bin[group(s.cand[i])], 1u);
    __syncthreads();
    if (tid < kWave) {
        uint32_t* bins = &s.bin[lane * 4];
        const uint32_t b0 = bins[0], b1 = bins[1], b2 = bins[2], b3 = bins[3];
        const uint32_t before = wave_scan_count(b0 + b1 + b2 + b3) - (b0 + b1 + b2 + b3);
        bins[0] = before;
        bins[1] = before + b0;
        bins[2] = before + b0 + b1;
        bins[3] = before + b0 + b1 + b2;
    }
    __syncthreads();
    // (In `sorted` for now in any order within a group.)
    for (int i = tid; i < nc; i += kW) {
        const uint64_t v = s.cand[i];
        const uint32_t g = group(v);
        s.sorted[s.bin[g] + atomicAdd(&s.fill[g], 1u)] = v;
    }
    __syncthreads();
    constexpr int kMost = kCap / kW;
    uint64_t v[kMost];
    int rank[kMost];
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        const int i = tid + j * kW;
        rank[j] = -1;
        if (i >= nc) continue;
        v[j] = s.sorted[i];
        const uint32_t g = group(v[j]);
        const int first = int(s.bin[g]), last = first + int(s.fill[g]);
        rank[j] = first;
        for (int o = first; o < last; ++o) rank[j] += s.sorted[o] > v[j] ? 1 : 0;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMost; ++j)
        if (rank[j] >= 0) s.sorted[rank[j]] = v[j];
    __syncthreads();
}

// The largest element of a chunk, NaN if one is.  For bf16 the 16-bit patterns
// are first compared as f16 numbers, two per packed instruction (see chunks_max):
// both are sign-magnitude with the exponent above the mantissa; a pattern that is an f16
// infinity or NaN (a bf16 magnitude of 2^121 or more) leaves an unusable
// result, and the chunk is decided element by element.
template <typename Fmt>
__device__ __forceinline__ float chunk_top(const chunk_t& c) {
    if constexpr (Fmt::kPerChunk == 8) {
        typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
        const auto H = [](uint32_t w) { return __builtin_bit_cast(h2_t, w); };
        const h2_t h = __builtin_elementwise_maximum(
            __builtin_elementwise_maximum(__builtin_elementwise_maximum(H(c.x), H(c.y)), H(c.z)), H(c.w));
        const uint32_t b = __builtin_bit_cast(uint32_t, h);
        const float lo = __uint_as_float(b << 16), hi = __uint_as_float(b & 0xFFFF0000u);
        if (__builtin_fabsf(lo) < 0x1p121f && __builtin_fabsf(hi) < 0x1p121f) return fmaxf(lo, hi);
    }
    float x = Fmt::get(c, 0);
#pragma unroll
    for (int e = 1; e < Fmt::kPerChunk; ++e) x = max_nan(x, Fmt::get(c, e));
    return x;
}

// f(r) for r = 0 .. N-1 as constants (more steps than the compiler unrolls).
template <typename F, int... R>
__device__ __forceinline__ void unrolled(std::integer_sequence<int, R...>, F f) {
    (f(std::integral_constant<int, R>{}), ...);
}

// Calls f(logit, token) for the elements of the row (-inf: padding too), every chunk of it by
// the whole workgroup (rare: small code before speed; two or four chunks of a thread
// requested at a time were no faster).
template <typename Fmt, int W, typename F>
__device__ __forceinline__ void over_row(const char* row, const RowCut<Fmt>& cut, int V, F f) {
#pragma unroll 1
    for (int ch = threadIdx.x; ch < cut.nchunks; ch += W) {
        chunk_t c = V < Fmt::kPerChunk ? load_short<Fmt>(row, V) : load_off(row, cut.off(ch));
        c = pad_lead<Fmt>(c, cut.lead(ch));
#pragma unroll
        for (int e = 0; e < Fmt::kPerChunk; ++e) f(Fmt::get(c, e), cut.token(ch * Fmt::kPerChunk + e));
    }
}

// A tile holds rows of MINR to GROUPS * G rounds: only rounds from MINR on ask whether
// the row has them or ends in them (asked in every round, 2048 rows of 128256 bf16 logits
// took 141 us instead of 126, 4.2 TB/s).  Of 512 threads three workgroups share a CU
// with 80 registers a lane (and 8 to 16 bytes of scratch a lane in the tiles of sixteen
// groups), two with 96: these 2048 rows took 133 us and 152.
template <typename Fmt, int W, int GROUPS, int G, int MINR>
__global__ __launch_bounds__(W, W == 1024 ? 4 : W == 512 ? 6 : 5) void topk_row_kernel(TopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk, NW = W / kWave, kRounds = GROUPS * G, kKeys = W / kWave;
    static_assert(W >= kBins && W >= OSD_MAX_TOPK && NW <= 16 && GROUPS <= 16, "");
    __shared__ TopkLds<W> s;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int64_t n = a.first + blockIdx.x;
    const int k = a.k;
    const char* row = a.x + n * a.stride;
    const RowCut<Fmt> cut(a.V);
    const int rounds = (cut.nchunks + W - 1) / W;
    const float c2 = float(a.c2);
    if (tid == 0) s.ncand = 0u;

    // One sweep: round r is chunk r * W + tid, in group r / G.
    float gmax[GROUPS], gsum[GROUPS];
    float ref = kNegInf, shift = 0.0f;  // the sums are relative to 2^shift, shift = ref c2
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        gmax[g] = kNegInf;
        gsum[g] = 0.0f;
    }
    {
        const rsrc_t rs = make_rsrc(row, uint32_t(a.V) * Fmt::kBytes);
        constexpr int kRing = kRounds < kAhead ? kRounds : kAhead;
        chunk_t c[kRing];
        // (Kept in the caches, where the candidates' groups are read from again: 64
        // rows of 32003 fp32 logits take 8.6 us, and 9.8 us streamed past them.)
        const auto load = [&](int r) __attribute__((always_inline)) {
            if (r >= MINR && r >= rounds) return;
            int off = (r * W + tid) * 16;
            if (r >= MINR - 1) off = min(off, cut.last_off);
            if constexpr (kRounds == 1) {
                if (a.V < EPC) {
                    c[0] = load_short<Fmt>(row, a.V);
                    return;
                }
            }
            c[r % kRing] = __builtin_bit_cast(chunk_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
        };
#pragma unroll
        for (int r = 0; r < kRing; ++r) load(r);
        unrolled(std::make_integer_sequence<int, kRounds>{}, [&](auto step) __attribute__((always_inline)) {
            constexpr int r = decltype(step)::value;
            if (r < MINR || r < rounds) {
                chunk_t x = c[r % kRing];
                if (r >= MINR - 1 && r == rounds - 1) x = pad_lead<Fmt>(x, cut.lead(r * W + tid));
                const float top = chunk_top<Fmt>(x);
                gmax[r / G] = r % G ? max_nan(gmax[r / G], top) : top;
                if (a.rest) {
                    if (!(ref > kNegInf)) {  // the first chunk with a finite logit
                        ref = top;
                        shift = top > kNegInf ? fmaxf(top * c2, -1.0e30f) : 0.0f;  // (so low: no mass)
                    }
                    float e8[EPC];
#pragma unroll
                    for (int e = 0; e < EPC; ++e) e8[e] = exp2_fast(__builtin_fmaf(Fmt::get(x, e), c2, -shift));
#pragma unroll
                    for (int w = 1; w < EPC; w <<= 1)
#pragma unroll
                        for (int e = 0; e < EPC; e += 2 * w) e8[e] = e8[e] + e8[e + w];
                    gsum[r / G] = r % G ? gsum[r / G] + e8[0] : e8[0];
                }
                __builtin_amdgcn_sched_barrier(0);
                if (r + kRing < kRounds) load(r + kRing);
            }
        });
    }
    float m = gmax[0];
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) m = max_nan(m, gmax[g]);
    s.key[tid] = order_key(m);
    __syncthreads();
    if (wid == 0) {
        // The k-th largest of the threads' maxima, to the upper 16 bits of its
        // key: a histogram of the 256 such keys from the largest down (two octaves),
        // and of the next 256 from the largest below these while they hold fewer
        // than k.
        const auto most_below = [&](uint32_t end16) {
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < kKeys; ++j) {
                const uint32_t key = s.key[j * kWave + lane];
                v = max(v, (key >> 16) < end16 ? key : 0u);
            }
            return wave_max_key(v);
        };
        uint32_t most = most_below(0x10000u);
        if (lane == 0) s.maxkey = most;
        uint32_t tkey = kKeyNegInf + 1, before = 0;
#pragma unroll 1
        while (most > kKeyNegInf) {  // (else fewer than k threads met a finite logit)
            const uint32_t base = most >> 16;
            uint32_t* bins = &s.bin[lane * 4];
            bins[0] = bins[1] = bins[2] = bins[3] = 0u;
            wave_lds_order();
#pragma unroll
            for (int j = 0; j < kKeys; ++j) {
                const uint32_t at = base - (s.key[j * kWave + lane] >> 16);
                if (at < uint32_t(kBins)) atomicAdd(&s.bin[at], 1u);
            }
            wave_lds_order();
            const uint32_t b0 = bins[0], b1 = bins[1], b2 = bins[2], b3 = bins[3];
            wave_lds_order();
            const uint32_t upto = wave_scan_count(b0 + b1 + b2 + b3) + before;
            const uint64_t full = __ballot(upto >= uint32_t(k));
            if (full) {
                const uint32_t left = upto - b0 - b1 - b2 - b3;
                const uint32_t j = (left + b0 < uint32_t(k)) + (left + b0 + b1 < uint32_t(k)) +
                                   (left + b0 + b1 + b2 < uint32_t(k));
                const int l = __builtin_ctzll(full);
                tkey = max(tkey, (base - uint32_t(l) * 4 - readlane_u32(j, l)) << 16);
                break;
            }
            before = readlane_u32(upto, kWave - 1);
            most = most_below(base < uint32_t(kBins) ? 0u : base - uint32_t(kBins) + 1);
        }
        if (lane == 0) s.tkey = tkey;
    }
    __syncthreads();
    const uint32_t maxkey = uniform(s.maxkey);
    if (maxkey >= kKeyPosInf || maxkey <= kKeyNegInf) {  // an infinity, a NaN, no finite logit
        for (int r = tid; r < k; r += W) {
            a.ids[n * k + r] = -1;
            if constexpr (EPC == 8)
                static_cast<uint16_t*>(a.top)[n * k + r] = 0xFF80u;
            else
                static_cast<float*>(a.top)[n * k + r] = kNegInf;
        }
        if (tid == 0 && a.rest) a.rest[n] = kNegInf;
        if (tid == 0 && a.tokens) a.tokens[n] = -1;
        return;
    }
    const float top = key_float(maxkey);
    const auto weight = [&](float x) __attribute__((always_inline)) { return exp2_fast((x - top) * c2); };
    // Candidates: logits above tx, and those equal to it up to token ttok.
    float tx = key_float(uniform(s.tkey));
    int ttok = 0x7FFFFFFF;
    // The thread's groups to look through: those that reach the threshold, and all
    // of them where the sums may have left fp32's range (a later chunk more than
    // 2^100 above the first) or the shift its precision.
    uint32_t flags = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) flags |= uint32_t(gmax[g] >= tx) << g;
    const uint32_t every = (1u << ((rounds + G - 1) / G)) - 1u;
    if (a.rest && ((m - ref) * c2 > 100.0f || __builtin_fabsf(top) * c2 > 65536.0f)) flags = every;
    int nc = 0;
    double S = 0.0;
#pragma unroll 1
    for (int pass = 0;; ++pass) {
        S = 0.0;
        int* queue = s.queue[wid];
        const uint32_t mine = uint32_t(__popc(flags)), upto = wave_scan_count(mine);
        const int total = int(readlane_u32(upto, kWave - 1));
#pragma unroll 1
        for (int first = 0; first < total; first += kQueue) {
            int at = int(upto - mine) - first;
            for (uint32_t f = flags; f; f &= f - 1, ++at)
                if (uint32_t(at) < uint32_t(kQueue)) queue[at] = (__builtin_ctz(f) * G) * W + tid;  // its first chunk
            wave_lds_order();
            const int elements = min(total - first, kQueue) * G * EPC;
            constexpr int kStep = 4;  // elements a lane requests at once
#pragma unroll 1
            for (int i0 = lane; i0 - lane < elements; i0 += kStep * kWave) {
                float x[kStep];
                int token[kStep];
#pragma unroll
                for (int j = 0; j < kStep; ++j) {
                    const int i = i0 + j * kWave;
                    x[j] = kNegInf;
                    if (i < elements) {
                        token[j] = (queue[i / (G * EPC)] + (i / EPC) % G * W) * EPC + i % EPC;
                        if (token[j] < a.V) x[j] = Fmt::load_one(row, token[j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < kStep; ++j) {
                    const bool in = x[j] > tx || (x[j] == tx && token[j] <= ttok);
                    const uint64_t ins = __ballot(in);
                    if (ins) {
                        uint32_t p = 0;
                        if (lane == 0) p = atomicAdd(&s.ncand, uint32_t(__popcll(ins)));
                        p = readlane_u32(p, 0) + lanes_below(ins);
                        if (in && p < uint32_t(kCap)) s.cand[p] = composite(order_key(x[j]), token[j]);
                    }
                    if (a.rest && !in) S += double(weight(x[j]));
                }
            }
            wave_lds_order();
        }
        __syncthreads();
        nc = int(uniform(s.ncand));
        if (nc <= kCap || pass) break;
        // Bisection for the largest key that k logits reach, then for the id up
        // to which its equals fill the record: `lo` always has k, `hi` has not.
        uint64_t lo = composite(order_key(tx), 0x7FFFFFFF), hi = composite(maxkey, 0) + 1;
#pragma unroll 1
        while (hi - lo > 1) {
            const uint64_t mid = lo + (hi - lo) / 2;
            const float mx = key_float(uint32_t(mid >> 32));
            const uint32_t mtok = ~uint32_t(mid);
            if (tid == 0) s.count = 0u;
            __syncthreads();
            uint32_t v = 0;
            over_row<Fmt, W>(row, cut, a.V, [&](float x, int token) __attribute__((always_inline)) {
                v += uint32_t(int(x > mx) | (int(x == mx) & int(uint32_t(token) <= mtok)));
            });
            v = readlane_u32(wave_scan_count(v), kWave - 1);
            if (lane == 0) atomicAdd(&s.count, v);
            __syncthreads();
            if (uniform(s.count) >= uint32_t(k))
                lo = mid;
            else
                hi = mid;
            __syncthreads();
        }
        tx = key_float(uint32_t(lo >> 32));
        ttok = int(~uint32_t(lo));
        if (tid == 0) s.ncand = 0u;
        __syncthreads();
        // (Groups below the new threshold keep their sums.)
        if (flags != every || !a.rest) {
            flags = 0;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) flags |= uint32_t(gmax[g] >= tx) << g;
        }
    }
    // The mass outside, relative to the row's largest logit.
    if (a.rest) {
        float t = 0.0f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) t += (flags >> g) & 1u ? 0.0f : gsum[g];
        if (t > 0.0f) S += double(t) * exp2_f64(double(shift) - double(top) * double(c2));
        S = wave_sum(S);
        if (lane == 0) s.sum[wid] = S;
    }
    sort_candidates<W>(s, nc, maxkey);
    for (int r = tid; r < k; r += W) {
        const uint64_t v = s.sorted[r];
        const bool in = r < nc;
        const float x = in ? key_float(uint32_t(v >> 32)) : kNegInf;
        a.ids[n * k + r] = in ? int(~uint32_t(v)) : -1;
        if constexpr (EPC == 8)
            static_cast<uint16_t*>(a.top)[n * k + r] = uint16_t(__float_as_uint(x) >> 16);
        else
            static_cast<float*>(a.top)[n * k + r] = x;
    }
    if (wid == 0 && a.rest) {
        double t = lane < NW ? s.sum[lane] : 0.0;
        for (int r = k + lane; r < nc; r += kWave) t += double(weight(key_float(uint32_t(s.sorted[r] >> 32))));
        t = wave_sum(t);
        if (lane == 0) {
            // (Fewer candidates than slots: they are the row's finite logits.)
            s.far = t < 0x1p-60 && nc >= k && k < a.V;
            if (!s.far) a.rest[n] = t > 0.0 ? float(log2_f64(t) * kLn2) : kNegInf;
        }
    }
    if (a.rest) {
        __syncthreads();
        // Far below the largest logit fp32 exponentials relative to it, or to a thread's
        // first chunk, leave their range one after another (2^-126): the others' largest
        // logit, then their mass relative to that, over the row once more each (576 rows of
        // 32128 bf16 logits ~ N(0, 9), k = 64: 17 us at T = 1, 38 at T = 0.1, where most
        // rows come here).
        if (uniform(s.far)) {
            const uint64_t last = s.sorted[k - 1];
            const float xk = key_float(uint32_t(last >> 32));
            const int tk = int(~uint32_t(last));
            const auto outside = [&](float x, int token) __attribute__((always_inline)) {
                return int(x < xk) | (int(x == xk) & int(token > tk)) ? x : kNegInf;
            };
            float most = kNegInf;
            over_row<Fmt, W>(row, cut, a.V, [&](float x, int token) __attribute__((always_inline)) {
                most = fmaxf(most, outside(x, token));
            });
            most = wave_max(most);
            if (lane == 0) s.key[wid] = float_key(most);
            __syncthreads();
            most = wave_max(lane < NW ? key_float(s.key[lane]) : kNegInf);
            double mass = 0.0;
            if (most > kNegInf)
                over_row<Fmt, W>(row, cut, a.V, [&](float x, int token) __attribute__((always_inline)) {
                    mass += double(exp2_fast((outside(x, token) - most) * c2));
                });
            mass = wave_sum(mass);
            if (lane == 0) s.sum[wid] = mass;
            __syncthreads();
            if (wid == 0) {
                mass = wave_sum(lane < NW ? s.sum[lane] : 0.0);
                if (lane == 0)
                    a.rest[n] = most > kNegInf
                                    ? float(((double(most) - double(top)) * a.c2 + log2_f64(mass)) * kLn2)
                                    : kNegInf;
            }
        }
    }
    if (wid == NW - 1 && a.tokens) {
        const int held = min(nc, k);
        if (a.c2 == 0.0) {
            if (lane == 0) a.tokens[n] = int(~uint32_t(s.sorted[0]));
            return;
        }
        // Lane l holds ranks 4 l .. 4 l + 3.
        const double top0 = double(key_float(uint32_t(s.sorted[0] >> 32)));
        double e[4], run = 0.0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = lane * 4 + j;
            e[j] = r < held ? exp2_f64((double(key_float(uint32_t(s.sorted[r] >> 32))) - top0) * a.c2) : 0.0;
            run += e[j];
        }
        const double upto = wave_scan_add(run);
        const double point = double(a.u[n]) * readlane_f64(upto, kWave - 1);
        double p = upto - run;
        int hit = 0x7FFFFFFF, lastpos = -1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p += e[j];
            if (e[j] > 0.0) lastpos = lane * 4 + j;
            if (e[j] > 0.0 && p > point && hit == 0x7FFFFFFF) hit = lane * 4 + j;
        }
        const uint64_t any = __ballot(hit != 0x7FFFFFFF);
        const uint64_t pos = __ballot(lastpos >= 0);
        int rank = any ? __shfl(hit, __builtin_ctzll(any), kWave) : __shfl(lastpos, 63 - __builtin_clzll(pos), kWave);
        if (lane == 0) a.tokens[n] = int(~uint32_t(s.sorted[rank]));
    }
}

template <typename Fmt, int W, int GROUPS, int G, int MINR>
hipError_t launch_tile(const TopkLaunch& L, TopkArgs a) {
    for (int64_t f = 0; f < L.N; f += kMaxGrid) {
        a.first = f;
        const unsigned g = unsigned(L.N - f < kMaxGrid ? L.N - f : kMaxGrid);
        const hipError_t e = launch_kernel(&topk_row_kernel<Fmt, W, GROUPS, G, MINR>, dim3(g), dim3(W), 0, L.stream, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename Fmt>
hipError_t launch_fmt(const TopkLaunch& L, const TopkArgs& a) {
    const int chunks = (L.V + Fmt::kPerChunk - 1) / Fmt::kPerChunk;
    if (chunks <= 256) return launch_tile<Fmt, 256, 1, 1, 1>(L, a);
    if (chunks <= 1024) return launch_tile<Fmt, 256, 4, 1, 2>(L, a);
    if (chunks > 16384) return hipErrorInvalidValue;
    // Threads a row (us, measured together, at 64, 256, 576 and 2048 rows).  32128 bf16 logits: 256 threads 12.0,
    // 14.4, 18.3 and 40.8, 512 9.5, 11.3, 17.6 and 39.8, 1024 9.5, 10.8, 25.0 and 40.9;
    // 64000: 256 20.6, 23.4, 29.0 and 75.5, 512 13.5, 16.3, 26.0 and 71.1, 1024 12.3, 15.2, 35.2
    // and 75.7.
    if (chunks <= 4096) return launch_tile<Fmt, 512, 8, 1, 3>(L, a);
    if (L.N <= L.cus) return launch_tile<Fmt, 1024, 16, 1, 5>(L, a);
    if (chunks <= 8192) return launch_tile<Fmt, 512, 16, 1, 9>(L, a);
    return launch_tile<Fmt, 512, 16, 2, 17>(L, a);
}

}  // namespace

hipError_t launch_topk(const TopkLaunch& L) {
    TopkArgs a{};
    a.x = static_cast<const char*>(L.x);
    a.stride = L.stride * (L.dtype == 1 ? 2 : 4);
    a.V = L.V;
    a.k = L.k;
    a.c2 = scaled_log2e(L.temperature);
    a.u = L.u;
    a.ids = L.ids;
    a.top = L.top;
    a.rest = L.rest;
    a.tokens = L.tokens;
    return L.dtype == 1 ? launch_fmt<BF16>(L, a) : launch_fmt<F32>(L, a);
}

}  // namespace osd
