// tree_attention.hpp -- what the two kernels of osd_tree_attention share: the
// matrix products, the softmax of a step, how work is divided, how parts are
// joined and rows written.
//
// The rows that read one kv head (all nodes, all its query heads) are the columns
// of two matrix products with each tile of keys:
//   S^T = K Q^T            A: 16 keys,          B: 16 rows of queries
//   O^T += V^T P^T         A: 16 of the values, B: the same rows
// so that the probabilities come out of the first product where the second takes
// them: a lane holds 4 keys of every 16 for one row, and as the order of keys
// within a product is free, these are its 8 (bf16) or 1 (fp32) of the second's.
// K is read as the first product's A operand, 16 bytes a lane.  Softmax in one pass:
// the exponents are relative to a reference that holds for all of a wave's keys (its
// first step's largest score), not to a running maximum, so that no step waits for the
// other lanes' scores or rescales sums.
#pragma once

#include "cache_device.hpp"

namespace osd {
namespace attention {

constexpr int kMaxGroups = 512;   // workgroups of a launch
constexpr int kMaxPieces = 64;    // workgroups that share a unit, at most, on average (a far longer one has more)

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// Maximum and sum over the four lanes that hold one row (lane, +16, +32, +48).
__device__ inline float rows_max(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float rows_sum(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// 2^(a - b), 0 where a is -inf (nothing seen yet).
__device__ inline float rescale(float a, float b) { return a == kNegInf ? 0.0f : exp2_fast(a - b); }

// x, of which the compiler computes nothing ahead: what is derived from a thread's number for the end of a
// piece would otherwise be computed before the loop over pieces and lie in scratch memory meanwhile
// (44 registers of 512 threads of 256 workgroups: 23 MB, 5 us).
__device__ inline int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The matrix products of one format.  KT tiles of 16 keys make a step.
//   K: chunk c of a key holds elements c * kChunk + group * (16 / ES) ..
//   V: a lane holds VW elements of a row for each block of 16 * VW of them.
// A value that is not finite must not reach rows that do not see its key (0 * inf
// is NaN): in steps that have keys of the tree the product takes 0 in its place, and
// the rows that see it get it when they are written.
struct Bf16Ops {
    using Fmt = BF16;
    static constexpr int kKT = 2, kChunk = 32;
    template <int VW>
    struct Value {
        typedef uint32_t reg_t __attribute__((ext_vector_type(VW / 2)));
        reg_t x;
        __device__ bool finite() const {
            bool f = true;
#pragma unroll
            for (int e = 0; e < VW / 2; ++e)
                f = f && (x[e] & 0x7F80u) != 0x7F80u && (x[e] & 0x7F800000u) != 0x7F800000u;
            return f;
        }
    };
    __device__ static f32x4_t qk(const chunk_t& k, const chunk_t& q, f32x4_t s) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q), s,
                                                       0, 0, 0);
    }
    __device__ static chunk_t negate(chunk_t q) { return q ^ 0x80008000u; }
    // A probability as two bf16 numbers, its upper half and the rest: together off by at most 2^-15 + 2^-22 of
    // it, so outputs lie 0.0017 (relative, rms) from exact ones, which is their own rounding.  One
    // number, off by 2^-8, gives 0.0024 and half of the second product's instructions: 32 even sequences
    // of 4032 tokens, 64 nodes, 195 us against 237; what memory bounds does not get slower (single tokens of
    // 64 sequences 221 and 222 us).  The rest is of p (1 + 2^-23), so above 0 wherever p is: with one of 0 an
    // infinite value would give NaN.
    struct Probs {
        chunk_t x[2];
    };
    __device__ static Probs probs(const float (&p)[8]) {
        constexpr float kUp = 1.00000011920928955078125f;  // 1 + 2^-23
        Probs r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = __float_as_uint(p[2 * i]), b = __float_as_uint(p[2 * i + 1]);
            r.x[0][i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            r.x[1][i] = pack_bf16x2(fmaf(p[2 * i], kUp, -__uint_as_float(a & 0xFFFF0000u)),
                                    fmaf(p[2 * i + 1], kUp, -__uint_as_float(b & 0xFFFF0000u)));
        }
        return r;
    }
    // Element t of the 8 keys of a lane.
    template <int VW>
    __device__ static chunk_t column(const Value<VW> (&v)[8], int t) {
        chunk_t a;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = __builtin_amdgcn_perm(v[2 * i + 1].x[t / 2], v[2 * i].x[t / 2], (t & 1) ? 0x07060302u : 0x05040100u);
        return a;
    }
    template <int VW>
    __device__ static f32x4_t pv(const Value<VW> (&v)[8], int t, const Probs& p, f32x4_t o) {
        const chunk_t a = column(v, t);
        return qk(a, p.x[1], qk(a, p.x[0], o));
    }
    static constexpr int kParts = 2;  // instructions of a product
    __device__ static f32x4_t pv_part(const chunk_t& v, const Probs& p, int i, f32x4_t o) { return qk(v, p.x[i], o); }
    // Of an operand of the second product: nonzero where a value is not finite (an exponent of all ones
    // carries into the sign's place), and those to 0.
    static constexpr uint32_t kSigns = 0x80008000u;
    __device__ static uint32_t carries(const chunk_t& v) {
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) c |= (v[i] & 0x7F807F80u) + 0x00800080u;
        return c;
    }
    __device__ static void clean(chunk_t& v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_finite(v[i]);
    }
    __device__ static uint32_t half_finite(uint32_t h) { return (h & 0x7F80u) == 0x7F80u ? 0u : h; }
    __device__ static uint32_t pair_finite(uint32_t h) { return half_finite(h & 0xFFFFu) | half_finite(h >> 16) << 16; }
    template <int VW>
    __device__ static void clean(Value<VW>& v) {
#pragma unroll
        for (int e = 0; e < VW / 2; ++e) v.x[e] = pair_finite(v.x[e]);
    }
};

struct F32Ops {
    using Fmt = F32;
    static constexpr int kKT = 1, kChunk = 16;
    template <int VW>
    struct Value {
        static_assert(VW == 4, "16 bytes");
        f32x4_t x;
        __device__ bool finite() const {
            bool f = true;
#pragma unroll
            for (int e = 0; e < 4; ++e) f = f && (__float_as_uint(x[e]) & 0x7F800000u) != 0x7F800000u;
            return f;
        }
    };
    __device__ static f32x4_t qk(const chunk_t& k, const chunk_t& q, f32x4_t s) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i]), __uint_as_float(q[i]), s, 0, 0, 0);
        return s;
    }
    __device__ static chunk_t negate(chunk_t q) { return q ^ 0x80000000u; }
    struct Probs {
        f32x4_t x;
    };
    __device__ static Probs probs(const float (&p)[4]) { return Probs{f32x4_t{p[0], p[1], p[2], p[3]}}; }
    template <int VW>
    __device__ static f32x4_t pv(const Value<VW> (&v)[4], int t, const Probs& p, f32x4_t o) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i].x[t], p.x[i], o, 0, 0, 0);
        return o;
    }
    static constexpr int kParts = 4;
    // (Element i of an operand: the lane's key i of 4.)
    __device__ static f32x4_t pv_part(const chunk_t& v, const Probs& p, int i, f32x4_t o) {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i]), p.x[i], o, 0, 0, 0);
    }
    static constexpr uint32_t kSigns = 0x80000000u;
    __device__ static uint32_t carries(const chunk_t& v) {
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) c |= (v[i] & 0x7F800000u) + 0x00800000u;
        return c;
    }
    __device__ static void clean(chunk_t& v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (v[i] & 0x7F800000u) == 0x7F800000u ? 0u : v[i];
    }
    template <int VW>
    __device__ static void clean(Value<VW>& v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v.x[e] = v.x[e] - v.x[e] == 0.0f ? v.x[e] : 0.0f;
    }
};

struct no_t {
    static constexpr bool value = false;
};
struct yes_t {
    static constexpr bool value = true;
};

struct Args {
    TreeAttentionLaunch L;
    float c2;            // |scale| * log2(e)
    int group;           // query heads of a kv head
    int blocks;          // row blocks of a kv head
    uint32_t* counters;  // [kMaxGroups, 3] zero on entry and exit: of the unit that begins in a workgroup
    float* stats;        // [2 * kMaxGroups, rows, 2] maximum (times c2) and sum
    float* parts;        // [2 * kMaxGroups, rows, DT] sums of p v
    uint32_t stats_bytes, parts_bytes;
};

// A sequence: 0 normal, 1 nothing to attend to (zeros), 2 invalid (NaN).
struct Seq {
    int len, n, state;
};
__device__ inline int state_of(const TreeAttentionLaunch& L, int len, int n) {
    return len < 0 || n == 0 ? 1 : cache_fits(L.pages, len, n, L.N) ? 0 : 2;
}
__device__ inline Seq sequence(const TreeAttentionLaunch& L, int b) {
    Seq s{L.seq_len[b], L.new_len ? L.new_len[b] : L.N, 0};
    s.state = state_of(L, s.len, s.n);
    return s;
}

__device__ inline int64_t quotient(int64_t a, int64_t b) {
    if ((uint64_t(a | b) >> 32) == 0) return int64_t(uint32_t(a) / uint32_t(b));  // a tenth of the instructions
    return a / b;
}

// A workgroup's part of one unit.
struct Piece {
    Seq seq;
    int b, h, tiles, t0, t1;
    int row0, rows, live;  // of the row block: its first row, its rows, those before padding
    int T;                 // keys
    bool whole;
    // Otherwise: the unit's first workgroup, how many there are, and where in the workspace
    // their parts are (the first's; those of the others are at 2 * workgroup) and this one's.
    int w0, count, first_slot, slot;
};
// Work is counted in tiles of keys.  A unit is one row block of one kv head of one
// sequence, all its keys.  There are two ways to divide them, neither of which asks the host for
// lengths:
//   apart     every unit is cut into equal parts, one workgroup each.  For few units;
//   in a row  units lie one after another, and every workgroup takes the same number of
//             tiles: at most two pieces of units that others share, the rest alone.
// A workgroup that ends one piece and begins another loses about 5 us (its loads run dry), so
// units are cut apart wherever that costs at most kSlack tiles of the longest.  Sequences'
// lengths are in registers of each wave (up to 64 of them; the parts, too, are counted there, so more
// sequences always lie in a row) or in LDS.
constexpr int kSlack = 4;

template <int THREADS, int TILE>
struct Division {
    int* s_before;          // [B + 1] tiles of the sequences before each, of one unit (more than 64)
    int tiles, len, n;      // (up to 64) lane b: a unit's tiles, and the sequence
    int upto;               // (up to 64) lane b: tiles (in a row) or parts (apart) up to and with sequence b
    int64_t total, each;    // tiles of all units, of a workgroup
    bool apart;

    __device__ static int tiles_of(const Seq& s) { return s.state ? 1 : (s.len + s.n - 1) / TILE + 1; }
    // Sums over the lanes up to each: within rows of 16, then across them.
    __device__ static int scan(int x) {
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);   // row_shr:1
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);   // row_shr:2
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);   // row_shr:4
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);   // row_shr:8
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1 and 3
        x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2 and 3
        return x;
    }

    __device__ void init(const Args& a, int* room) {
        const TreeAttentionLaunch& L = a.L;
        const int tid = int(threadIdx.x), lane = tid & (kWave - 1);
        const int64_t units = int64_t(L.kv_heads) * a.blocks;
        int all;
        s_before = room;
        apart = false;
        if (L.B <= kWave) {
            Seq s{-1, 0, 1};
            if (lane < L.B) s = sequence(L, lane);
            len = s.len;
            n = s.n;
            tiles = lane < L.B ? tiles_of(s) : 0;
            upto = scan(tiles);
            all = __builtin_amdgcn_readlane(upto, kWave - 1);
        } else {
            constexpr int WAVES = THREADS / kWave;
            __shared__ int s_scan[WAVES];
            const int wave = tid / kWave, share = (L.B + THREADS - 1) / THREADS, first = tid * share;
            int mine = 0;
            for (int b = first; b < first + share && b < L.B; ++b) {
                const int t = tiles_of(sequence(L, b));
                s_before[b] = t;
                mine += t;
            }
            const int sum = scan(mine);
            if (lane == kWave - 1) s_scan[wave] = sum;
            __syncthreads();
            int before = sum - mine;
            for (int w = 0; w < wave; ++w) before += s_scan[w];
            for (int b = first; b < first + share && b < L.B; ++b) {
                const int t = s_before[b];
                s_before[b] = before;
                before += t;
                if (b == L.B - 1) s_before[L.B] = before;
            }
            __syncthreads();
            all = __builtin_amdgcn_readfirstlane(s_before[L.B]);
        }
        total = all * units;
        int64_t W = int64_t(gridDim.x);
        if (W > L.B * units * kMaxPieces) W = L.B * units * kMaxPieces;
        each = quotient(total + W - 1, W);
        if (L.B <= kWave && L.B * units <= W) {
            for (int more = 0; more <= kSlack && !apart; more = more ? more * 2 : 1) {
                const int e = int(each) + more, parts = (tiles + e - 1) / e, to = scan(parts);
                if (__builtin_amdgcn_readlane(to, kWave - 1) * units > W) continue;
                apart = true;
                upto = to;
                each = e;
                break;
            }
        }
    }
    // The tiles (apart: the workgroup) that workgroup w begins with.
    __device__ int64_t begin(int64_t w) const {
        if (apart) return w;
        return w * each < total ? w * each : total;
    }
    __device__ int64_t end(const Args& a, int64_t w) const {
        if (!apart) return begin(w + 1);
        const int64_t W = int64_t(__builtin_amdgcn_readlane(upto, kWave - 1)) * a.L.kv_heads * a.blocks;
        return w < W ? w + 1 : w;
    }

    // The piece at `pos`, of a workgroup w that has the ones from `first` to `end`.
    template <int ROWS>
    __device__ Piece find(const Args& a, int64_t w, int64_t pos, int64_t first, int64_t end) const;
    // What has to be added to `pos` for the next one.
    __device__ int64_t step(const Piece& p) const { return apart ? 1 : p.t1 - p.t0; }
};

template <int THREADS, int TILE>
template <int ROWS>
__device__ inline Piece Division<THREADS, TILE>::find(const Args& a, int64_t w, int64_t pos, int64_t first, int64_t end) const {
    const TreeAttentionLaunch& L = a.L;
    const int64_t units = int64_t(L.kv_heads) * a.blocks;
    Piece p;
    int before, upto_b;
    if (L.B <= kWave) {
        const int lane = int(threadIdx.x) & (kWave - 1);
        p.b = __ffsll(static_cast<unsigned long long>(__ballot(lane < L.B && upto * units > pos))) - 1;
        before = p.b ? __builtin_amdgcn_readlane(upto, p.b - 1) : 0;
        upto_b = __builtin_amdgcn_readlane(upto, p.b);
        p.tiles = __builtin_amdgcn_readlane(tiles, p.b);
        p.seq = Seq{__builtin_amdgcn_readlane(len, p.b), __builtin_amdgcn_readlane(n, p.b), 0};
        p.seq.state = state_of(L, p.seq.len, p.seq.n);
    } else {
        int b = 0;
        for (int hi = L.B; hi - b > 1;) {
            const int mid = (b + hi) / 2;
            if (s_before[mid] * units <= pos) b = mid;
            else hi = mid;
        }
        p.b = __builtin_amdgcn_readfirstlane(b);
        before = __builtin_amdgcn_readfirstlane(s_before[p.b]);
        upto_b = __builtin_amdgcn_readfirstlane(s_before[p.b + 1]);
        p.tiles = upto_b - before;
        p.seq = sequence(L, p.b);
    }
    int unit;
    if (apart) {  // (at most kMaxGroups parts: 32 bits)
        const int length = upto_b - before, in_b = int(pos) - before * int(units);
        unit = int(uint32_t(in_b) / uint32_t(length));
        const int at = in_b - unit * length, e = int(each);
        p.t0 = at * e;
        p.t1 = p.t0 + e < p.tiles ? p.t0 + e : p.tiles;
        p.whole = length == 1;
        p.w0 = int(w) - at;
        p.count = length;
        p.first_slot = 2 * p.w0;
        p.slot = 2 * int(w);
    } else {
        const int64_t in_b = pos - before * units;
        unit = int(quotient(in_b, p.tiles));
        const int at = int(in_b - int64_t(unit) * p.tiles);
        p.t0 = at;
        p.t1 = int(end - pos < p.tiles - at ? at + (end - pos) : p.tiles);
        p.whole = p.t0 == 0 && p.t1 == p.tiles;
        p.w0 = p.count = p.first_slot = 0;
        if (!p.whole) {
            const int64_t u0 = pos - at;
            p.w0 = int(quotient(u0, each));
            p.count = int(quotient(u0 + p.tiles - 1, each)) - p.w0 + 1;
            p.first_slot = 2 * p.w0 + (p.w0 * each == u0 ? 0 : 1);
        }
        p.slot = 2 * int(w) + (pos == first ? 0 : 1);
    }
    p.h = unit / a.blocks;
    p.row0 = (unit - p.h * a.blocks) * ROWS;
    p.rows = L.N * a.group - p.row0 < ROWS ? L.N * a.group - p.row0 : ROWS;
    p.live = p.seq.state ? 0 : p.seq.n * a.group - p.row0;
    p.T = p.seq.state ? 0 : p.seq.len + p.seq.n;
    return p;
}

// Queries of 16 rows as the first product's B operand, `r` of the block this lane's.
template <typename Ops, int CHUNKS, bool FULL>
__device__ inline void load_queries(const Args& a, const Piece& p, int r, int D, chunk_t (&q)[CHUNKS]) {
    const TreeAttentionLaunch& L = a.L;
    constexpr int ES = Ops::Fmt::kBytes;
    const int grp = (here(int(threadIdx.x)) & (kWave - 1)) >> 4;
    const int node = (p.row0 + r) / a.group, g = p.row0 + r - node * a.group;
    const char* at = L.q + (int64_t(p.b) * L.N + node) * L.q_stride + int64_t(p.h * a.group + g) * D * ES + grp * 16;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        q[c] = chunk_t{0, 0, 0, 0};
        if (r < p.live && (FULL || c * Ops::kChunk + grp * (16 / ES) < D))
            q[c] = *reinterpret_cast<const chunk_t*>(at + c * Ops::kChunk * ES);
        if (L.scale < 0.0f) q[c] = Ops::negate(q[c]);
    }
}

// Elements of V that a lane reads at once where each lane reads whole pieces of rows.
template <typename Ops, int DT>
constexpr int kPiece = DT * Ops::Fmt::kBytes >= 256 ? 16 / Ops::Fmt::kBytes : DT / 16;

// 16 MT rows and what a wave has summed for them: element (col * VW + t) of block n of
// a row's values in acc[..][n][t].
template <typename Ops, int DT, int MT, int VW_>
struct Rows {
    static constexpr int ES = Ops::Fmt::kBytes, KT = Ops::kKT, KEYS = 4 * KT, CHUNKS = (DT + Ops::kChunk - 1) / Ops::kChunk;
    static constexpr int VW = VW_, BW = 16 * VW, BLOCKS = DT / BW;
    f32x4_t acc[MT][BLOCKS][VW];
    float ref[MT], sum[MT];  // every exponent's reference, and the lane's sum
    float seen[MT];          // the lane's largest score so far
    uint64_t sees[MT];       // the tree's nodes that a row sees
    bool odd;                // a value of the tree's steps that is not finite

    __device__ void clear() {
        odd = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            seen[mt] = kNegInf;
            sum[mt] = 0.0f;
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int t = 0; t < VW; ++t) acc[mt][n][t] = f32x4_t{0, 0, 0, 0};
        }
    }
    // What exponents are taken relative to: the largest of some scores (the first
    // step's), 0 where they have none.
    __device__ void refer(const float (&most)[MT], float c2) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const float m = rows_max(most[mt]);
            ref[mt] = m == kNegInf ? 0.0f : m * c2;
        }
    }
    // Whether the reference served: p up to 2^32 and sums of them are as exact as p up to
    // 1 (no scale is lost in fp32 or bf16), so steps need not agree on a maximum; only
    // where a score turned out further away are all keys taken again, now relative to
    // the largest.  So they are where a sum of p v reached 2^112 (or is not finite): relative to the largest score
    // it may be smaller, and below 2^112 those of 2^12 waves have a sum.  (Not of a row whose probabilities
    // are NaN: what only that row sees must not change its neighbours.)
    __device__ bool served(float c2) const {
        constexpr uint32_t kLarge = 0x77800000u;  // 2^112
        bool ok = true;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            uint32_t most = 0;
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int t = 0; t < VW; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = max(most, __float_as_uint(acc[mt][n][t][e]) & 0x7FFFFFFFu);
            const float m = rows_max(seen[mt]), all = rows_sum(sum[mt]);
            ok = ok && (most < kLarge || all != all);
            ok = ok && (m == kNegInf || fabsf(m * c2 - ref[mt]) <= 32.0f);
        }
        return __all(ok);
    }
    // Where keys that not every row sees begin, j0 their first step's.
    __device__ void mask(f32x4_t (&s)[MT][KT], int j0, const Seq& seq) const {
        const int grp = (int(threadIdx.x) & (kWave - 1)) >> 4;
        // The lane's first key, counted from the tree's; bit i of `on`: whether the row sees key first + i.
        // (Without branches: hipcc lost scores where lanes parted here.)
        const int first = j0 + grp * 4 - seq.len, up = first > 0 ? first : 0, down = first < 0 ? -first : 0;
        const uint32_t context = down < 32 ? (1u << (down & 31)) - 1u : ~0u;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            uint32_t on = uint32_t((sees[mt] >> (up & 63)) << (down & 31));
            on = (up < 64 && down < 32 ? on : 0u) | context;
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const uint32_t bit = 1u << ((i / 4) * 16 + (i & 3));
                s[mt][i / 4][i & 3] = (on & bit) != 0u ? s[mt][i / 4][i & 3] : kNegInf;
            }
        }
    }
    __device__ static void largest(const f32x4_t (&s)[MT][KT], float (&most)[MT]) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < KEYS; ++i) most[mt] = fmaxf(most[mt], s[mt][i / 4][i & 3]);
    }
    // Scores to probabilities (times 2^-ref).  TAIL: masked ones are -inf, and their probability is 0
    // (also with c2 = 0).
    template <bool TAIL>
    __device__ void soften(const f32x4_t (&s)[MT][KT], float c2, typename Ops::Probs (&p)[MT]) {
        largest(s, seen);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float x[KEYS];
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const float score = s[mt][i / 4][i & 3];
                x[i] = exp2_fast(fmaf(score, c2, -ref[mt]));
                if constexpr (TAIL) x[i] = score == kNegInf ? 0.0f : x[i];
                sum[mt] += x[i];
            }
            p[mt] = Ops::probs(x);
        }
    }
    // Keys behind the last may hold anything; nodes that a row does not see, too.
    template <typename Value>
    __device__ void guard(Value (&v)[BLOCKS][KEYS], int j0, int T) {
        const int grp = (int(threadIdx.x) & (kWave - 1)) >> 4;
        bool fine = true;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const bool in = j0 + (i / 4) * 16 + grp * 4 + (i & 3) < T;
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n) {
                if (!in) v[n][i].x = decltype(Value::x){};
                fine = fine && v[n][i].finite();
            }
        }
        if (__any(!fine)) {
            odd = true;
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int i = 0; i < KEYS; ++i) Ops::clean(v[n][i]);
        }
    }
    template <typename Value>
    __device__ void add(const Value (&v)[BLOCKS][KEYS], const typename Ops::Probs (&p)[MT]) {
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
            for (int t = 0; t < VW; ++t)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[mt][n][t] = Ops::pv(v[n], t, p[mt], acc[mt][n][t]);
    }
    // The sums of row tile mt, times f, to a row of LDS.
    template <int PITCH>
    __device__ void store(int mt, float f, float* row, int grp) const {
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n) {
            if constexpr (VW == 1) {
                *reinterpret_cast<f32x4_t*>(row + n * 16 + grp * 4) = acc[mt][n][0] * f;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < VW; t += 4)
                        *reinterpret_cast<f32x4_t*>(row + n * BW + (grp * 4 + e) * VW + t) =
                            f32x4_t{acc[mt][n][t][e] * f, acc[mt][n][t + 1][e] * f, acc[mt][n][t + 2][e] * f, acc[mt][n][t + 3][e] * f};
            }
        }
    }
};

// Adds the values d .. d+3 that are not finite of the keys `from` .. `to`-1 that a row sees: those of this
// workgroup's piece (one that saw none of them would post an infinity beside a maximum of -inf, and
// the join make NaN of it).
template <typename Fmt>
__device__ inline void add_odd(const TreeAttentionLaunch& L, int b, int h, int d, int len, int from, int to, uint64_t sees,
                                     f32x4_t& o) {
    for (int j = from; j < to; ++j) {
        if (j >= len && !(sees >> (j - len) & 1)) continue;
        const int64_t at = cache_place(L.pages, b, j);
        if (at < 0) continue;
        for (int e = 0; e < 4; ++e) {
            const float x = Fmt::load_one(L.v_cache + at + h * L.pages.head_bytes, d + e);
            if (x - x != 0.0f) o[e] += x;
        }
    }
}

// Where a row's values go: a byte offset in the output (a multiple of 16), 1 more for a row of zeros.
template <typename Fmt>
__device__ inline int64_t row_place(const Args& a, const Piece& p, int row, int D) {
    const TreeAttentionLaunch& L = a.L;
    const int at = p.row0 + row, node = int(uint32_t(at) / uint32_t(a.group)), g = at - node * a.group;
    const bool on = row < p.live || (p.seq.state == 2 && (p.seq.n < 0 || p.seq.n > node));
    return ((int64_t(p.b) * L.N + node) * L.q_heads + p.h * a.group + g) * (D * Fmt::kBytes) + (on ? 0 : 1);
}
// Four values of a row to the output.
template <typename Fmt>
__device__ inline void write_row(const Args& a, int64_t place, int d, f32x4_t o, float inv) {
    char* to = a.L.out + (place & ~int64_t(1)) + d * Fmt::kBytes;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (place & 1) == 0 ? o[e] * inv : 0.0f;
    if constexpr (Fmt::kBytes == 2) *reinterpret_cast<u32x2_t*>(to) = u32x2_t{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
    else *reinterpret_cast<f32x4_t*>(to) = o;
}

// Parts cross workgroups through loads and stores at device scope (sc1), which
// pass by the private caches of the dies.
constexpr int kDeviceScope = 16;
__device__ inline auto buffer_of(float* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(p, 0, int(bytes), 0x00027000);
}
template <int ROWS, int DT>
__device__ inline void post_part(const Args& a, int slot, int row, int d, f32x4_t o, float top, float sum) {
    const int64_t at = int64_t(slot) * ROWS + row;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(chunk_t, o), buffer_of(a.parts, a.parts_bytes),
                                           int(uint32_t(at * DT + d) * 4u), 0, kDeviceScope);
    if (d == 0)
        __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{__float_as_uint(top), __float_as_uint(sum)},
                                              buffer_of(a.stats, a.stats_bytes), int(uint32_t(at) * 8u), 0, kDeviceScope);
}

// Rows r0 .. r1-1 of a unit from its parts, in their order: ITEMS times four values of a
// thread, PIECES parts in flight each.
template <typename Fmt, int THREADS, int ROWS, int DT, int ITEMS, int PIECES>
__device__ inline void join_parts(const Args& a, const Piece& p, int r0, int r1, int D, const int64_t* places) {
    const auto stats = buffer_of(a.stats, a.stats_bytes), parts = buffer_of(a.parts, a.parts_bytes);
    const int items = r1 * (DT / 4), count = p.count;
    for (int i0 = r0 * (DT / 4) + here(int(threadIdx.x)); i0 < items; i0 += THREADS * ITEMS) {
        float most[ITEMS], total[ITEMS];
        f32x4_t o[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) most[k] = kNegInf, total[k] = 0.0f, o[k] = f32x4_t{0, 0, 0, 0};
        for (int x0 = 0; x0 < count; x0 += PIECES) {
            u32x2_t st[ITEMS][PIECES];
            chunk_t part[ITEMS][PIECES];
#pragma unroll
            for (int x = 0; x < PIECES; ++x)
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    const int i = i0 + k * THREADS, row = i / (DT / 4), d = i % (DT / 4) * 4;
                    const bool in = i < items && x0 + x < count && d < D;
                    const uint32_t at = uint32_t(x0 + x ? 2 * (p.w0 + x0 + x) : p.first_slot) * ROWS + row;
                    st[k][x] = u32x2_t{0, 0};
                    part[k][x] = chunk_t{0, 0, 0, 0};
                    if (in) {
                        st[k][x] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(stats, int(at * 8u), 0, kDeviceScope));
                        part[k][x] = __builtin_bit_cast(chunk_t, __builtin_amdgcn_raw_buffer_load_b128(parts, int((at * DT + d) * 4u), 0, kDeviceScope));
                    }
                }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                float now = most[k];
#pragma unroll
                for (int x = 0; x < PIECES; ++x)
                    if (x0 + x < count) now = fmaxf(now, __uint_as_float(st[k][x].x));
                const float f = rescale(most[k], now);
                o[k] *= f;
                total[k] *= f;
#pragma unroll
                for (int x = 0; x < PIECES; ++x) {
                    if (x0 + x >= count) continue;
                    const float g = rescale(__uint_as_float(st[k][x].x), now), s = __uint_as_float(st[k][x].y);
                    o[k] += __builtin_bit_cast(f32x4_t, part[k][x]) * g;
                    total[k] += s == s ? s * g : s;
                }
                most[k] = now;
            }
        }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = i0 + k * THREADS, row = i / (DT / 4), d = i % (DT / 4) * 4;
            if (i < items && d < D) write_row<Fmt>(a, places[row], d, o[k], 1.0f / total[k]);
        }
    }
}

// A workgroup has posted its part of a unit (all its threads call this).  Where the unit's
// parts are many and large, its workgroups wait for each other and join some rows each: a
// workgroup alone reads 50 GB/s.  The wait is bounded, and nothing depends on who waits: rows
// are taken from a counter, and the last to arrive does not wait and takes what is left.  (places: of
// the unit's rows, in LDS.)
constexpr int kJoinBytes = 128 << 10;  // of a unit's parts: fewer are joined by the last alone
constexpr int kJoinPolls = 64;

template <typename Fmt, int THREADS, int ROWS, int DT>
__device__ inline void join_rows(const Args& a, const Piece& p, int r0, int r1, int D, const int64_t* places) {
    // A read takes about 2 us, so as many as registers allow are in flight.
    if (p.count <= 2) join_parts<Fmt, THREADS, ROWS, DT, 8, 2>(a, p, r0, r1, D, places);
    else if (p.count <= 4) join_parts<Fmt, THREADS, ROWS, DT, 4, 4>(a, p, r0, r1, D, places);
    else if ((r1 - r0) * (DT / 4) > THREADS) join_parts<Fmt, THREADS, ROWS, DT, 2, 8>(a, p, r0, r1, D, places);
    else join_parts<Fmt, THREADS, ROWS, DT, 1, 16>(a, p, r0, r1, D, places);
}

template <typename Fmt, int THREADS, int ROWS, int DT>
__device__ inline void join(const Args& a, const Piece& p, bool together, int D, const int64_t* places) {
    __shared__ uint32_t s_word;
    const int tid = int(threadIdx.x);
    uint32_t* arrivals = a.counters + 3 * p.w0;
    uint32_t* taken = arrivals + 1;
    uint32_t* gone = arrivals + 2;
    together = together && int64_t(p.count) * p.rows * DT * 4 > kJoinBytes;
    wait_memory();
    __syncthreads();
    if (tid == 0) {
        bool all = arrive(arrivals) == uint32_t(p.count - 1);
        for (int i = 0; together && !all && i < kJoinPolls; ++i) {
            __builtin_amdgcn_s_sleep(8);
            all = load_relaxed(arrivals) == uint32_t(p.count);
        }
        s_word = all;
    }
    __syncthreads();
    const bool all = s_word != 0;
    if (!together) {
        if (!all) return;
        join_rows<Fmt, THREADS, ROWS, DT>(a, p, 0, p.rows, D, places);
        if (tid == 0) __hip_atomic_store(arrivals, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return;
    }
    const int some = (p.rows + p.count - 1) / p.count;
    while (all) {
        __syncthreads();
        if (tid == 0) s_word = arrive(taken);
        __syncthreads();
        const int r0 = int(s_word) * some;
        if (r0 >= p.rows) break;
        join_rows<Fmt, THREADS, ROWS, DT>(a, p, r0, r0 + some < p.rows ? r0 + some : p.rows, D, places);
    }
    // The last to leave clears the counters.
    if (tid == 0 && arrive(gone) == uint32_t(p.count - 1)) {
        __hip_atomic_store(arrivals, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(taken, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(gone, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// Rows of one workgroup, of the kernel that serves `rows` rows of a kv head.
inline int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// tree_attention_wide.hpp
hipError_t launch_wide_bf16(const Args& a, int rows);
hipError_t launch_wide_f32(const Args& a, int rows);

}  // namespace attention
}  // namespace osd
