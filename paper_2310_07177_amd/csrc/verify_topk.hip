// verify_topk.hip -- verification of proposals drawn from the draft's record
// (gfx950).
//
// Method: with q the softmax over the record's slots (0 elsewhere) and p the
// target's softmax over the whole row, proposal y_i is accepted when
// u q(y_i) < p(y_i), and the first rejection at row a draws from max(0, p - q)
// (Appendix A.1, Eq. 5).  p and max(0, p - q) differ at the record's tokens only,
// so the masses of a row's cells (256 chunks: 2048 bf16 or 1024 fp32 logits), known
// from the sums that normalise p, need no more than the record's corrections to
// place the draw in a cell, and one cell of row a is read again.
//
//   cells   one wave per cell of every row 0 .. k_b: its largest logit and the
//           fp64 sum of exponentials relative to it
//   decide  one workgroup per sequence: normalisers, tests, first rejection,
//           corrections, the draw
#include "osd.h"
#include "osd_device.hpp"
#include "osd_internal.hpp"
#include "stream_device.hpp"
#include "topk_device.hpp"

namespace osd {
namespace {

constexpr int kW = 256, kNW = kW / kWave;
constexpr int kCellChunks = 256;  // chunks of a cell: one wave, four a lane
constexpr int64_t kMaxGrid = int64_t(1) << 22;

struct VerifyTopkArgs {
    const char* target;
    const int32_t* ids;
    const char* top;
    int k;
    int B, K, V, cells;
    const int32_t* tokens;
    const int32_t* draft_len;
    const float* u_accept;
    const float* u_resample;
    double c2;
    VerifyTopkRow* rows;
    int32_t* accepted_len;
    int32_t* out_tokens;
    uint8_t* reject_mask;
    int64_t first;
};

template <typename Fmt>
__device__ inline chunk_t row_chunk(const char* row, int ch, const RowCut<Fmt>& cut, int V) {
    if (V < Fmt::kPerChunk) return ch == 0 ? load_short<Fmt>(row, V) : pad_chunk<Fmt>();
    return pad_lead<Fmt>(load_off(row, cut.off(ch)), cut.lead(ch));
}

template <typename Fmt>
__global__ __launch_bounds__(kW) void cells_kernel(VerifyTopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk, kPer = kCellChunks / kWave;
    const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
    const int64_t unit = (a.first + blockIdx.x) * kNW + wid;
    const int64_t row = unit / a.cells;
    const int cell = int(unit - row * a.cells);
    const int64_t b = row / (a.K + 1);
    const int i = int(row - b * (a.K + 1));
    if (b >= a.B) return;
    const int kb = a.draft_len ? a.draft_len[b] : a.K;
    if (i > kb || kb < 1 || kb > a.K) return;
    const RowCut<Fmt> cut(a.V);
    const char* x = a.target + row * a.V * Fmt::kBytes;
    chunk_t c[kPer];
#pragma unroll
    for (int r = 0; r < kPer; ++r) c[r] = row_chunk<Fmt>(x, cell * kCellChunks + r * kWave + lane, cut, a.V);
    float m = kNegInf;
#pragma unroll
    for (int r = 0; r < kPer; ++r)
#pragma unroll
        for (int e = 0; e < EPC; ++e) m = max_nan(m, Fmt::get(c[r], e));
    m = wave_max_nan(m);
    double S = 0.0;
    if (is_finite(m)) {
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int e = 0; e < EPC; ++e) S += exp2_f64((double(Fmt::get(c[r], e)) - double(m)) * a.c2);
    }
    S = wave_sum(S);
    if (lane == 0) {
        a.rows[row].sum[cell] = S;
        a.rows[row].top[cell] = m;
    }
}

struct DecideLds {
    double sum[OSD_MAX_K + 1];          // rows: normaliser
    float top[OSD_MAX_K + 1];           //       largest logit, NaN if unusable
    double qy[OSD_MAX_K];
    int bad[OSD_MAX_K];                 // records that are none
    double q[OSD_MAX_TOPK];
    int id[OSD_MAX_TOPK];
    uint64_t fixed[kMaxCells];          // corrections by cell, 2^-62
    double cum[kMaxCells];              // mass up to and with each cell
    double dense[kCellChunks * 8];      // q over the tokens of one cell
    double wave[kNW];
    int hit[kNW], last[kNW];
    int32_t table[kNW][1024];           // ids seen, by wave
    int stop, invalid;
};

// Slot i = j * 64 + lane of the record of one position, by one wave: its
// probability in q[j] (id -1: 0), and whether the record is one.
template <typename Fmt>
__device__ inline bool record_softmax(const VerifyTopkArgs& a, int64_t pos, int32_t* table, int (&id)[4],
                                      double (&q)[4]) {
    const int lane = threadIdx.x & (kWave - 1);
    float x[4], m = kNegInf;
    bool ok = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = j * kWave + lane;
        id[j] = i < a.k ? a.ids[pos * a.k + i] : -1;
        x[j] = kNegInf;
        if (id[j] < -1 || id[j] >= a.V) {
            ok = false;
            id[j] = -1;
        }
        if (id[j] >= 0) {
            x[j] = Fmt::load_one(a.top + pos * a.k * Fmt::kBytes, i);
            if (!(x[j] < -kNegInf)) ok = false;
        }
        m = fmaxf(m, x[j]);
    }
    m = wave_max(m);
    ok = ok && m > kNegInf;
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        q[j] = x[j] > kNegInf ? exp2_f64((double(x[j]) - double(m)) * a.c2) : 0.0;
        s += q[j];
    }
    s = wave_sum(s);
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = q[j] / s;
    // An id twice: its place in the table of ids (1024 places for at most 256
    // ids) is taken by an equal one.
    int place[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        place[j] = -1;
        if (id[j] < 0) continue;
        int h = int((uint32_t(id[j]) * 2654435761u) >> 22);
        for (int t = 0; t < 1024; ++t) {
            const int old = atomicCAS(&table[h], -1, id[j]);
            if (old == -1) {
                place[j] = h;
                break;
            }
            if (old == id[j]) {
                ok = false;
                break;
            }
            h = (h + 1) & 1023;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (place[j] >= 0) table[place[j]] = -1;
    return __ballot(!ok) == 0;
}

template <typename Fmt>
__global__ __launch_bounds__(kW) void decide_kernel(VerifyTopkArgs a) {
    constexpr int EPC = Fmt::kPerChunk;
    __shared__ DecideLds s;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    const int64_t b = a.first + blockIdx.x;
    const int K = a.K;
    const int kb = a.draft_len ? a.draft_len[b] : K;
    const int32_t* y = a.tokens + b * K;
    for (int i = lane; i < 1024; i += kWave) s.table[wid][i] = -1;
    if (tid < kMaxCells) s.fixed[tid] = 0;
    if (tid == 0) s.invalid = 0;
    __syncthreads();
    if (tid < K && tid < kb && (y[tid] < 0 || y[tid] >= a.V)) s.invalid = 1;
    __syncthreads();
    bool invalid = kb < 1 || kb > K || s.invalid;
    int acc = 0, extra = -1;
    if (!invalid) {
        for (int i = wid; i <= kb; i += kNW) {
            const VerifyTopkRow& r = a.rows[b * (K + 1) + i];
            const float m = lane < a.cells ? r.top[lane] : kNegInf;
            const float top = wave_max_nan(m);
            const double v = lane < a.cells && is_finite(m) ? r.sum[lane] : 0.0;
            const double sum = wave_sum(v * exp2_f64((double(m) - double(top)) * a.c2));
            if (lane == 0) {
                s.top[i] = top;
                s.sum[i] = sum;
            }
            if (i < kb) {
                int id[4];
                double q[4];
                const bool ok = record_softmax<Fmt>(a, b * K + i, s.table[wid], id, q);
                const int want = y[i];
                double mine = 0.0;
#pragma unroll
                for (int j = 0; j < 4; ++j) mine += id[j] == want ? q[j] : 0.0;
                mine = wave_sum(mine);
                if (lane == 0) {
                    s.qy[i] = mine;
                    s.bad[i] = !ok;
                }
            }
        }
        __syncthreads();
        if (wid == 0) {
            // Lane i: the test of position i.
            bool bad = false, reject = false;
            if (lane <= kb) bad = !is_finite(s.top[lane]);
            if (lane < kb && !bad) {
                bad = s.bad[lane] != 0;
                const float t = Fmt::load_one(a.target + ((b * (K + 1) + lane) * a.V) * Fmt::kBytes, y[lane]);
                const double py = exp2_f64((double(t) - double(s.top[lane])) * a.c2) / s.sum[lane];
                reject = !(double(a.u_accept[b * K + lane]) * s.qy[lane] < (t > kNegInf ? py : 0.0));
            }
            const uint64_t stops = __ballot(lane <= kb && (bad || reject || lane == kb));
            const int at = __builtin_ctzll(stops);
            const uint64_t bads = __ballot(bad);
            if (lane == 0) {
                s.stop = at;
                s.invalid = int((bads >> at) & 1);
            }
        }
        __syncthreads();
        acc = s.stop;
        invalid = s.invalid != 0;
    }
    if (!invalid) {
        const bool rejected = acc < kb;
        const int64_t row = b * (K + 1) + acc;
        const char* x = a.target + row * a.V * Fmt::kBytes;
        const RowCut<Fmt> cut(a.V);
        const double top = double(s.top[acc]), inv = 1.0 / s.sum[acc];
        const auto place = [&](int id) {  // element of the row in chunk order
            const int ch = id / EPC;
            return id + (ch >= cut.nfull ? cut.dup : 0);
        };
        const auto prob = [&](float t) {
            return t > kNegInf ? exp2_f64((double(t) - top) * a.c2) * inv : 0.0;
        };
        if (rejected && wid == 0) {
            int id[4];
            double q[4];
            record_softmax<Fmt>(a, b * K + acc, s.table[0], id, q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = j * kWave + lane;
                s.id[i] = id[j];
                s.q[i] = q[j];
                if (id[j] < 0) continue;
                const double both = fmin(prob(Fmt::load_one(x, id[j])), q[j]);
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.fixed[place(id[j]) / (kCellChunks * EPC)]),
                          (unsigned long long)(both * 0x1p62));
            }
        }
        __syncthreads();
        // Lane c of every wave: cell c.
        const VerifyTopkRow& r = a.rows[row];
        const float m = lane < a.cells ? r.top[lane] : kNegInf;
        double mass = 0.0;
        if (lane < a.cells && is_finite(m)) mass = r.sum[lane] * exp2_f64((double(m) - top) * a.c2) * inv;
        const bool live = mass > 0.0;
        const double left = fmax(mass - double(s.fixed[lane]) * 0x1p-62, 0.0);
        double cum = wave_scan_add(left);
        bool with_q = rejected;
        if (readlane_f64(cum, kWave - 1) <= 0.0) {  // rounding left nothing: from p
            cum = wave_scan_add(mass);
            with_q = false;
        }
        const double Z = readlane_f64(cum, kWave - 1);
        const double point = double(a.u_resample[b]) * Z;
        const uint64_t lives = __ballot(live);
        // The first cell that may hold the point (the sums of the cells and of
        // their elements differ by rounding), then upwards; down from there only
        // if rounding put the point past the last token.
        const uint64_t from = __ballot(live && cum > point - 1e-14);
        int cell = from ? __builtin_ctzll(from) : 63 - __builtin_clzll(lives);
        const int start = cell;
        bool up = true;
        while (true) {
            double base = cell > 0 ? readlane_f64(cum, cell - 1) : 0.0;
            __syncthreads();
            for (int i = tid; i < kCellChunks * EPC; i += kW) s.dense[i] = 0.0;
            __syncthreads();
            if (with_q && tid < a.k && s.id[tid] >= 0) {
                const int at = place(s.id[tid]) - cell * kCellChunks * EPC;
                if (at >= 0 && at < kCellChunks * EPC) s.dense[at] = s.q[tid];
            }
            __syncthreads();
            const int ch = cell * kCellChunks + tid;
            const chunk_t c = row_chunk<Fmt>(x, ch, cut, a.V);
            double e[EPC], run = 0.0;
#pragma unroll
            for (int j = 0; j < EPC; ++j) {
                e[j] = fmax(prob(Fmt::get(c, j)) - s.dense[tid * EPC + j], 0.0);
                run += e[j];
            }
            const double upto = wave_scan_add(run);
            if (lane == kWave - 1) s.wave[wid] = upto;
            __syncthreads();
            for (int w = 0; w < wid; ++w) base += s.wave[w];
            base += upto - run;
            int hit = 0x7FFFFFFF, lastpos = -1;
#pragma unroll
            for (int j = 0; j < EPC; ++j) {
                base += e[j];
                if (e[j] > 0.0) lastpos = cut.token(ch * EPC + j);
                if (e[j] > 0.0 && base > point && hit == 0x7FFFFFFF) hit = cut.token(ch * EPC + j);
            }
            const uint64_t any = __ballot(hit != 0x7FFFFFFF), pos = __ballot(lastpos >= 0);
            const int h = any ? __shfl(hit, __builtin_ctzll(any), kWave) : 0x7FFFFFFF;
            const int l = pos ? __shfl(lastpos, 63 - __builtin_clzll(pos), kWave) : -1;
            if (lane == 0) {
                s.hit[wid] = h;
                s.last[wid] = l;
            }
            __syncthreads();
            int found = 0x7FFFFFFF, lastfound = -1;
            for (int w = 0; w < kNW; ++w) {
                found = min(found, s.hit[w]);
                lastfound = max(lastfound, s.last[w]);
            }
            if (up) {
                if (found != 0x7FFFFFFF) {
                    extra = found;
                    break;
                }
                if (lastfound >= 0) extra = lastfound;
                const uint64_t more = lives & ~((2ull << cell) - 1);
                if (cell < 63 && more) {
                    cell = __builtin_ctzll(more);
                    continue;
                }
                if (extra >= 0) break;
                up = false;
                cell = start;
            } else if (lastfound >= 0) {
                extra = lastfound;
                break;
            }
            const uint64_t fewer = lives & ((1ull << cell) - 1);
            if (!fewer) break;
            cell = 63 - __builtin_clzll(fewer);
        }
        invalid = extra < 0;
    }
    if (tid <= K) {
        const int64_t o = b * (K + 1) + tid;
        a.out_tokens[o] = invalid || tid > acc ? -1 : (tid == acc ? extra : y[tid]);
        if (tid == 0) a.accepted_len[b] = invalid ? -1 : acc;
        if (a.reject_mask && tid < K) a.reject_mask[b * K + tid] = !invalid && tid == acc && acc < kb ? 1 : 0;
    }
}

template <typename Fmt>
hipError_t launch_fmt(const VerifyTopkLaunch& L, VerifyTopkArgs a) {
    const int chunks = (L.V + Fmt::kPerChunk - 1) / Fmt::kPerChunk;
    a.cells = (chunks + kCellChunks - 1) / kCellChunks;
    if (a.cells > kMaxCells) return hipErrorInvalidValue;
    const int64_t groups = (int64_t(a.B) * (a.K + 1) * a.cells + kNW - 1) / kNW;
    for (int64_t f = 0; f < groups; f += kMaxGrid) {
        a.first = f;
        const unsigned g = unsigned(groups - f < kMaxGrid ? groups - f : kMaxGrid);
        const hipError_t e = launch_kernel(&cells_kernel<Fmt>, dim3(g), dim3(kW), 0, L.stream, a);
        if (e != hipSuccess) return e;
    }
    for (int64_t f = 0; f < a.B; f += kMaxGrid) {
        a.first = f;
        const unsigned g = unsigned(a.B - f < kMaxGrid ? a.B - f : kMaxGrid);
        const hipError_t e = launch_kernel(&decide_kernel<Fmt>, dim3(g), dim3(kW), 0, L.stream, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_verify_topk(const VerifyTopkLaunch& L) {
    VerifyTopkArgs a{};
    a.target = static_cast<const char*>(L.target);
    a.ids = L.ids;
    a.top = static_cast<const char*>(L.top);
    a.k = L.k;
    a.B = L.B;
    a.K = L.K;
    a.V = L.V;
    a.tokens = L.tokens;
    a.draft_len = L.draft_len;
    a.u_accept = L.u_accept;
    a.u_resample = L.u_resample;
    a.c2 = scaled_log2e(L.temperature);
    a.rows = L.rows;
    a.accepted_len = L.accepted_len;
    a.out_tokens = L.out_tokens;
    a.reject_mask = L.reject_mask;
    return L.dtype == 1 ? launch_fmt<BF16>(L, a) : launch_fmt<F32>(L, a);
}

}  // namespace osd
