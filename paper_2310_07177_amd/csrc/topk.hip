// topk.hip -- the record of a row's top logits, and a token drawn from it
// (gfx950).
//
// Method: a workgroup holds a row in registers.  Each thread takes the maximum
// of its elements; the k-th largest of the threads' maxima (to 16 bits of the
// ordered key) is at most the k-th largest logit, since k threads hold an element
// that large, so the elements at or above it, the candidates, are all the record
// can hold.  There are few more than k of them (a thread rarely holds two): they
// are collected in LDS and ranked by counting, for each, the candidates before
// it, so the record does not depend on the order of their arrival.  A row with
// more candidates than LDS holds (many equal logits, or the largest ones side by
// side) gets the exact k-th (logit, id) by bisection first.
//
// The mass of the tokens outside the record is summed over the elements below
// the threshold, then the candidates that were not taken: nothing is subtracted,
// so it keeps its relative accuracy however small it is.  The draw sums fp64
// exponentials of the record's logits.
#include "osd.h"
#include "osd_device.hpp"
#include "osd_internal.hpp"
#include "stream_device.hpp"
#include "topk_device.hpp"

namespace osd {
namespace {

constexpr int kCap = 1024;  // candidates that LDS holds
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
    uint64_t cand[kCap];
    uint64_t sorted[kCap];
    uint32_t digit[4][16];
    uint32_t count[2];
    double sum[W / kWave];
    uint32_t ncand;
    uint32_t maxkey;
};

// Candidates come first: larger logit, then lower id.
__device__ inline uint64_t composite(uint32_t key, int token) { return (uint64_t(key) << 32) | uint32_t(~token); }

template <typename Fmt, int W, int CPT>
__global__ __launch_bounds__(W, 4) void topk_row_kernel(TopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk, NW = W / kWave;
    __shared__ TopkLds<W> s;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    const int64_t n = a.first + blockIdx.x;
    const int k = a.k;
    const HeldRow<Fmt, W, CPT> held(a.V);
    chunk_t c[CPT];
    held.load(c, a.x + n * a.stride, a.V, tid);
    if (tid < 64) s.digit[tid / 16][tid % 16] = 0u;
    if (tid == 0) {
        s.ncand = 0u;
        s.maxkey = 0u;
    }
    __syncthreads();
    held.pad(c, tid);

    float m = kNegInf;
    held.each([&](int r) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < EPC; ++e) m = max_nan(m, Fmt::get(c[r], e));
    });
    const uint32_t mk = order_key(m);
    {
        const float wm = wave_max_nan(m);
        if (lane == 0) atomicMax(&s.maxkey, order_key(wm));
    }
    // The k-th largest maximum, four bits at a time.
    uint32_t prefix = 0;
#pragma unroll
    for (int step = 0; step < 4; ++step) {
        const int sh = 12 - 4 * step;
        uint32_t mine = 0;
#pragma unroll
        for (int d = 1; d < 16; ++d) {
            const uint32_t cnt = uint32_t(__popcll(__ballot((mk >> 16) >= (prefix | (uint32_t(d) << sh)))));
            if (lane == d) mine = cnt;
        }
        if (lane < 16) atomicAdd(&s.digit[step][lane], mine);
        __syncthreads();
        const uint32_t total = s.digit[step][lane & 15];
        const int d = __popcll(__ballot(lane >= 1 && lane < 16 && total >= uint32_t(k)));
        prefix |= uint32_t(d) << sh;
    }
    const uint32_t maxkey = s.maxkey;
    const bool empty = maxkey >= kKeyPosInf || maxkey <= kKeyNegInf;  // an infinity, a NaN, no finite logit
    if (empty) {
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
    // Candidates: logits above tx, and those equal to it up to token ttok.
    float tx = key_float(max(prefix << 16, kKeyNegInf + 1));
    int ttok = 0x7FFFFFFF;
    double S = 0.0;
    const float c2 = float(a.c2), top = key_float(maxkey);
    const auto weight = [&](float x) __attribute__((always_inline)) { return exp2_fast((x - top) * c2); };
    // Collects the candidates; the others among the logits equal to tx are
    // added to S.
    const auto collect = [&]() __attribute__((always_inline)) {
        if (!(m >= tx)) return;
        held.each([&](int r) __attribute__((always_inline)) {
            asm volatile("" : "+v"(c[r]));
            if (!(chunk_max<Fmt>(c[r]) >= tx)) return;
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                const float x = Fmt::get(c[r], e);
                if (!(x >= tx)) continue;
                const int tok = held.token(r, e, opaque_tid());
                if (x > tx || tok <= ttok) {
                    const uint32_t p = atomicAdd(&s.ncand, 1u);
                    if (p < uint32_t(kCap)) s.cand[p] = composite(order_key(x), tok);
                } else if (a.rest) {
                    S += double(weight(x));
                }
            }
        });
    };
    collect();
    __syncthreads();
    if (s.ncand > uint32_t(kCap)) {
        // Bisection for the largest key that k logits reach, then for the id up
        // to which its equals fill the record: `lo` always has k, `hi` has not.
        uint64_t lo = composite(order_key(tx), 0x7FFFFFFF), hi = composite(maxkey, 0) + 1;
        int flip = 0;
#pragma unroll 1
        while (hi - lo > 1) {
            const uint64_t mid = lo + (hi - lo) / 2;
            const uint32_t mkey = uint32_t(mid >> 32), mtok = ~uint32_t(mid);
            uint32_t v = 0;
            held.each([&](int r) __attribute__((always_inline)) {
                asm volatile("" : "+v"(c[r]));
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    const uint32_t key = order_key(Fmt::get(c[r], e));
                    v += key > mkey || (key == mkey && uint32_t(held.token(r, e, opaque_tid())) <= mtok) ? 1u : 0u;
                }
            });
            __syncthreads();
            if (tid == 0) s.count[flip] = 0u;
            __syncthreads();
            atomicAdd(&s.count[flip], v);
            __syncthreads();
            if (s.count[flip] >= uint32_t(k))
                lo = mid;
            else
                hi = mid;
            flip ^= 1;
        }
        tx = key_float(uint32_t(lo >> 32));
        ttok = int(~uint32_t(lo));
        __syncthreads();
        if (tid == 0) s.ncand = 0u;
        S = 0.0;
        __syncthreads();
        collect();
        __syncthreads();
    }
    const int nc = int(s.ncand);
    for (int i = tid; i < nc; i += W) {
        const uint64_t me = s.cand[i];
        int rank = 0;
        for (int j = 0; j < nc; ++j) rank += s.cand[j] > me ? 1 : 0;
        s.sorted[rank] = me;
    }
    // The mass outside: logits below the threshold, relative to the row's
    // largest.
    if (a.rest) {
        held.each([&](int r) __attribute__((always_inline)) {
            asm volatile("" : "+v"(c[r]));
            float e8[EPC];
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                const float x = Fmt::get(c[r], e);
                e8[e] = x < tx ? weight(x) : 0.0f;
            }
#pragma unroll
            for (int w = 1; w < EPC; w <<= 1)
#pragma unroll
                for (int e = 0; e < EPC; e += 2 * w) e8[e] = e8[e] + e8[e + w];
            S += double(e8[0]);
        });
        S = wave_sum(S);
        if (lane == 0) s.sum[wid] = S;
    }
    __syncthreads();
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
        for (int r = k + lane; r < nc; r += kWave)
            t += double(weight(key_float(uint32_t(s.sorted[r] >> 32))));
        t = wave_sum(t);
        if (lane == 0) a.rest[n] = t > 0.0 ? float(log2_pos(t) * kLn2) : kNegInf;
    }
    if (wid == NW - 1 && a.tokens) {
        const int held = nc < k ? nc : k;
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

template <typename Fmt, int W, int CPT>
hipError_t launch_tile(const TopkLaunch& L, TopkArgs a) {
    for (int64_t f = 0; f < L.N; f += kMaxGrid) {
        a.first = f;
        const unsigned g = unsigned(L.N - f < kMaxGrid ? L.N - f : kMaxGrid);
        const hipError_t e = launch_kernel(&topk_row_kernel<Fmt, W, CPT>, dim3(g), dim3(W), 0, L.stream, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename Fmt>
hipError_t launch_fmt(const TopkLaunch& L, TopkArgs a) {
    const int chunks = (L.V + Fmt::kPerChunk - 1) / Fmt::kPerChunk;
    if (chunks <= 256) return launch_tile<Fmt, 256, 1>(L, a);
    if (chunks <= 1024) return launch_tile<Fmt, 256, 4>(L, a);
    if (chunks <= 2048) return launch_tile<Fmt, 512, 4>(L, a);
    if (chunks <= 4096) return launch_tile<Fmt, 512, 8>(L, a);
    if (chunks <= 8192) return launch_tile<Fmt, 1024, 8>(L, a);
    if (chunks <= 16384) return launch_tile<Fmt, 1024, 16>(L, a);
    return hipErrorInvalidValue;
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
