// tree_attention.hip -- osd_tree_attention: drafted tokens attend to the context
// in the paged cache, to their ancestors and to themselves.
//
// The rows that read one kv head (all nodes, all its query heads) are the columns
// of two matrix products with each tile of keys:
//   S^T = K Q^T            A: 16 keys,          B: 16 rows of queries
//   O^T += V^T P^T         A: 16 of the values, B: the same rows
// so that the probabilities come out of the first product where the second takes
// them: a lane holds 4 keys of every 16 for one row, and as the order of keys
// within a product is free, these are its 8 (bf16) or 1 (fp32) of the second's.
// K comes from memory as the first product's A operand (16 bytes a lane); of V a
// lane loads whole 16-byte pieces of the keys that it holds, and picks the halves
// of each pair of keys apart in registers, which is the transposition.  Nothing
// goes through LDS on the way.  Softmax in one pass: running maximum and sum in
// fp32, rescaled when a tile raises a maximum.
#include "cache_device.hpp"

namespace osd {
namespace {

constexpr int kWaves = 4;         // of a workgroup: each takes its own keys of a tile
constexpr int kThreads = kWaves * kWave;
constexpr int kMaxGroups = 512;   // workgroups of a launch
constexpr int kMaxPieces = 64;    // workgroups that share a unit

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

// The matrix products of one format.  KT tiles of 16 keys make a step.
//   K: chunk c of a key holds elements c * kChunk + group * (16 / ES) ..
//   V: a lane holds VW elements of a row for each block of 16 * VW of them.
// A value that is not finite must not reach rows that do not see its key (0 * inf
// is NaN): in steps that have keys of the tree the product takes 0 in its place, and
// the rows that see it get it when they are written.
struct Bf16Ops {
    using Fmt = BF16;
    static constexpr int kKT = 2, kChunk = 32;
    using score_t = f32x4_t;
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
    struct Probs {
        chunk_t x;
    };
    __device__ static Probs probs(const float (&p)[8]) {
        Probs r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.x[i] = pack_bf16x2(p[2 * i], p[2 * i + 1]);
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
        return qk(column(v, t), p.x, o);
    }
    __device__ static uint32_t half_finite(uint32_t h) { return (h & 0x7F80u) == 0x7F80u ? 0u : h; }
    template <int VW>
    __device__ static void clean(Value<VW>& v) {
#pragma unroll
        for (int e = 0; e < VW / 2; ++e) v.x[e] = half_finite(v.x[e] & 0xFFFFu) | half_finite(v.x[e] >> 16) << 16;
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

struct AttentionArgs {
    TreeAttentionLaunch L;
    float c2;       // |scale| * log2(e)
    int group;      // query heads of a kv head
    int blocks;     // row blocks of a kv head
    uint32_t* counters;  // [kMaxGroups] zero on entry and exit: arrivals of the unit that begins in a workgroup
    float* stats;        // [2 * kMaxGroups, rows, 2] maximum (times c2) and sum
    float* parts;        // [2 * kMaxGroups, rows, DT] sums of p v
};

// Work is counted in tiles of kWaves steps.  A unit is one row block of one kv head
// of one sequence, all its keys; units lie one after another, and workgroup w of W
// takes the tiles from w * total / W on: equal shares whatever the lengths, at most
// two pieces of which are parts of units (the others it has alone).
struct Share {
    int64_t total;
    int64_t W;
    __device__ int64_t begin(int64_t w) const { return w * total / W; }
    __device__ int64_t owner(int64_t tile) const { return ((tile + 1) * W - 1) / total; }
};

// A sequence: 0 normal, 1 nothing to attend to (zeros), 2 invalid (NaN).
struct Seq {
    int len, n, state;
};
__device__ inline Seq sequence(const TreeAttentionLaunch& L, int b) {
    Seq s{L.seq_len[b], L.new_len ? L.new_len[b] : L.N, 0};
    if (s.len < 0 || s.n == 0) s.state = 1;
    else if (!cache_fits(L.pages, s.len, s.n, L.N)) s.state = 2;
    return s;
}

__device__ inline void post(float* p, float x, float y) {
    const u32x2_t v = {__float_as_uint(x), __float_as_uint(y)};
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float2 fetch(const float* p) {
    const uint64_t w =
        __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const u32x2_t v = __builtin_bit_cast(u32x2_t, w);
    return float2{__uint_as_float(v.x), __uint_as_float(v.y)};
}

// Adds the values d .. d+3 that are not finite of the keys from `from` on that a row sees.
template <typename Fmt>
__device__ inline void add_odd(const TreeAttentionLaunch& L, int b, int h, int d, int len, int T, int from, uint64_t sees,
                                     f32x4_t& o) {
    for (int j = from; j < T; ++j) {
        if (j >= len && !(sees >> (j - len) & 1)) continue;
        const int64_t at = cache_place(L.pages, b, j);
        if (at < 0) continue;
        for (int e = 0; e < 4; ++e) {
            const float x = Fmt::load_one(L.v_cache + at + h * L.pages.head_bytes, d + e);
            if (x - x != 0.0f) o[e] += x;
        }
    }
}

// DT: head_dim rounded up; MT: row tiles of 16; GEN: pages that end inside tiles of
// 16 keys, or head_dim < DT.
template <typename Ops, int DT, int MT, bool GEN>
__global__ __launch_bounds__(kThreads, MT * DT >= 512 ? 1 : 2) void tree_attention_kernel(AttentionArgs a) {
    using Fmt = typename Ops::Fmt;
    const TreeAttentionLaunch& L = a.L;
    constexpr int ES = Fmt::kBytes, KT = Ops::kKT, STEP = 16 * KT, TILE = STEP * kWaves;
    constexpr int CHUNKS = DT / Ops::kChunk, VW = DT * ES >= 256 ? 16 / ES : DT / 16, BW = 16 * VW, BLOCKS = DT / BW;
    constexpr int ROWS = 16 * MT, KEYS = 4 * KT, PITCH = DT + 4;
    using Value = typename Ops::template Value<VW>;
    const int tid = int(threadIdx.x), lane = tid & (kWave - 1), wave = tid / kWave, col = lane & 15, grp = lane >> 4;
    const int D = GEN ? L.head_dim : DT;
    const int row_bytes = GEN ? L.pages.row_bytes : DT * ES;

    extern __shared__ int64_t s_tiles[];  // [B + 1] tiles before each sequence (of one unit)
    __shared__ float s_acc[kWaves][16][PITCH];
    __shared__ float s_stat[kWaves][ROWS][2];
    __shared__ int64_t s_scan[kWaves];
    __shared__ uint64_t s_sees[ROWS];
    __shared__ int s_odd[kWaves];
    __shared__ uint32_t s_arrived;

    // Tiles of all sequences before each.
    {
        const int each = (L.B + kThreads - 1) / kThreads, first = tid * each;
        int64_t mine = 0;
        for (int b = first; b < first + each && b < L.B; ++b) {
            const Seq s = sequence(L, b);
            mine += s.state ? 1 : (s.len + s.n - 1) / TILE + 1;
        }
        int64_t sum = mine;
#pragma unroll
        for (int o = 1; o < kWave; o *= 2) {
            const int64_t up = __shfl_up(static_cast<long long>(sum), o);
            if (lane >= o) sum += up;
        }
        if (lane == kWave - 1) s_scan[wave] = sum;
        __syncthreads();
        int64_t before = sum - mine;
        for (int w = 0; w < wave; ++w) before += s_scan[w];
        for (int b = first; b < first + each && b < L.B; ++b) {
            s_tiles[b] = before;
            const Seq s = sequence(L, b);
            before += s.state ? 1 : (s.len + s.n - 1) / TILE + 1;
            if (b == L.B - 1) s_tiles[L.B] = before;
        }
        __syncthreads();
    }
    const int units = L.kv_heads * a.blocks;  // of a sequence
    Share share;
    share.total = s_tiles[L.B] * units;
    share.W = int64_t(gridDim.x);
    if (share.W > int64_t(L.B) * units * kMaxPieces) share.W = int64_t(L.B) * units * kMaxPieces;
    if (share.W > share.total) share.W = share.total;
    const int64_t w = int64_t(blockIdx.x);
    if (w >= share.W) return;
    const int64_t first = share.begin(w), end = share.begin(w + 1);

    for (int64_t pos = first; pos < end;) {
        // The unit that holds tile `pos`.
        int b = 0;
        for (int hi = L.B; hi - b > 1;) {
            const int mid = (b + hi) / 2;
            if (s_tiles[mid] * units <= pos) b = mid;
            else hi = mid;
        }
        b = __builtin_amdgcn_readfirstlane(b);
        const Seq seq = sequence(L, b);
        const int tiles = int(s_tiles[b + 1] - s_tiles[b]);
        const int64_t in_b = pos - s_tiles[b] * units;
        const int unit = __builtin_amdgcn_readfirstlane(int(in_b / tiles));
        const int t0 = __builtin_amdgcn_readfirstlane(int(in_b - int64_t(unit) * tiles));
        const int t1 = __builtin_amdgcn_readfirstlane(int(end - pos < tiles - t0 ? t0 + (end - pos) : tiles));
        const int h = unit / a.blocks, row0 = (unit - h * a.blocks) * ROWS;
        const int rows = L.N * a.group - row0 < ROWS ? L.N * a.group - row0 : ROWS;  // of this block
        const int live = seq.state ? 0 : seq.n * a.group - row0;                      // before padding
        const int len = seq.len, T = seq.state ? 0 : seq.len + seq.n;

        // Queries.
        chunk_t q[MT][CHUNKS];
        uint64_t sees[MT];
        bool bad = seq.state == 2;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int r = mt * 16 + col;
            const int node = (row0 + r) / a.group, g = row0 + r - node * a.group;
            const char* at = L.q + (int64_t(b) * L.N + node) * L.q_stride + int64_t(h * a.group + g) * D * ES + grp * 16;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                q[mt][c] = chunk_t{0, 0, 0, 0};
                if (r < live && (!GEN || c * Ops::kChunk + grp * (16 / ES) < D))
                    q[mt][c] = *reinterpret_cast<const chunk_t*>(at + c * Ops::kChunk * ES);
                if (L.scale < 0.0f) q[mt][c] = Ops::negate(q[mt][c]);
            }
            sees[mt] = 0;
        }
        if (t1 * TILE > len && T > 0) {
            bool tree;
            const uint64_t all = wave_ancestors(L.parent ? L.parent + int64_t(b) * L.N : nullptr, seq.n, &tree);
            bad = bad || !tree;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int node = (row0 + mt * 16 + col) / a.group;
                sees[mt] = uint64_t(__shfl(static_cast<unsigned long long>(all), node & (kWave - 1)));
            }
        }

        f32x4_t acc[MT][BLOCKS][VW];
        float top[MT], sum[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            top[mt] = kNegInf;
            sum[mt] = 0.0f;
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int t = 0; t < VW; ++t) acc[mt][n][t] = f32x4_t{0, 0, 0, 0};
        }

        // Byte offsets of the tiles of 16 keys to come (!GEN), two lanes a step, or
        // of the 32 keys of the next step (GEN); out of the cache: its first.
        const int64_t head = int64_t(h) * L.pages.head_bytes;
        int64_t ahead = 0;
        auto look = [&](int j) {
            int64_t at = 0;
            if (j < T) {
                at = cache_place(L.pages, b, j);
                bad = bad || at < 0;
                at = at < 0 ? 0 : at;
            }
            return at + head;
        };
        chunk_t k[KT][CHUNKS];
        Value v[BLOCKS][KEYS];
        const int k_lane = col * row_bytes + grp * 16, v_lane = grp * 4 * row_bytes + col * VW * ES;
        auto at_tile = [&](int step, int kt) {  // !GEN
            const int from = (step * KT + kt) & (kWave - 1);
            const uint32_t lo = __builtin_amdgcn_readlane(int(uint32_t(ahead)), from);
            const uint32_t hi = __builtin_amdgcn_readlane(int(uint32_t(uint64_t(ahead) >> 32)), from);
            return int64_t(uint64_t(hi) << 32 | lo);
        };
        auto load_k = [&](int step) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const char* at;
                if constexpr (GEN) at = L.k_cache + __shfl(static_cast<long long>(ahead), kt * 16 + col) + grp * 16;
                else at = L.k_cache + at_tile(step, kt) + k_lane;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    if constexpr (GEN) {
                        const bool in = c * Ops::kChunk + grp * (16 / ES) < D;
                        k[kt][c] = *reinterpret_cast<const chunk_t*>(in ? at + c * Ops::kChunk * ES : at - grp * 16);
                        if (!in) k[kt][c] = chunk_t{0, 0, 0, 0};
                    } else {
                        k[kt][c] = *reinterpret_cast<const chunk_t*>(at + c * Ops::kChunk * ES);
                    }
                }
            }
        };
        auto load_v = [&](int step) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const char* tile = nullptr;
                if constexpr (!GEN) tile = L.v_cache + at_tile(step, kt) + v_lane;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const char* at;
                    if constexpr (GEN) at = L.v_cache + __shfl(static_cast<long long>(ahead), kt * 16 + grp * 4 + i) + col * VW * ES;
                    else at = tile + i * row_bytes;
#pragma unroll
                    for (int n = 0; n < BLOCKS; ++n) {
                        const bool in = !GEN || n * BW + col * VW < D;
                        v[n][kt * 4 + i].x = *reinterpret_cast<const decltype(Value::x)*>(in ? at + n * BW * ES : at - col * VW * ES);
                    }
                }
            }
        };
        auto fill = [&](int step) {  // the offsets from `step` on
            if constexpr (GEN) ahead = look((t0 + step) * TILE + wave * STEP + (lane & (STEP - 1)));
            else ahead = look((t0 + step + lane / KT) * TILE + wave * STEP + (lane & (KT - 1)) * 16);
        };
        // The wave's steps: one in each tile, as long as there are keys.
        int steps = t1 - t0;
        if (steps > 0 && (t1 - 1) * TILE + wave * STEP >= T) --steps;
        steps = __builtin_amdgcn_readfirstlane(steps);
        constexpr int PERIOD = GEN ? 1 : kWave / KT;
        if (steps > 0) {
            fill(0);
            load_k(0);
            load_v(0);
        }
        bool odd = false;  // a value of these that is not finite
        // One step; TAIL: it has keys that not every row sees.
        auto take = [&](int step, auto tail) {
            constexpr bool TAIL = decltype(tail)::value;
            const int j0 = (t0 + step) * TILE + wave * STEP;
            f32x4_t s[MT][KT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    s[mt][kt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) s[mt][kt] = Ops::qk(k[kt][c], q[mt][c], s[mt][kt]);
                }
            // The next step's keys while this one's probabilities are formed.
            const bool more = step + 1 < steps;
            if (more) {
                if ((step + 1) % PERIOD == 0) fill(step + 1);
                load_k(step + 1);
            }
            typename Ops::Probs p[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                bool on[KEYS];
                float best = kNegInf;
                if constexpr (TAIL) {
#pragma unroll
                    for (int i = 0; i < KEYS; ++i) {
                        const int j = j0 + (i / 4) * 16 + grp * 4 + (i & 3) - len;
                        on[i] = j < 0 || (j < seq.n && (sees[mt] >> (j & 63) & 1));
                        if (!on[i]) s[mt][i / 4][i & 3] = kNegInf;
                    }
                }
#pragma unroll
                for (int i = 0; i < KEYS; ++i) best = fmaxf(best, s[mt][i / 4][i & 3]);
                best = fmaxf(rows_max(best) * a.c2, top[mt]);
                if (__any(best > top[mt])) {
                    const float f = rescale(top[mt], best);
                    sum[mt] *= f;
#pragma unroll
                    for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                        for (int t = 0; t < VW; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[mt][n][t][e] *= f;
                    top[mt] = best;
                }
                const float base = top[mt] == kNegInf ? 0.0f : top[mt];
                float x[KEYS];
#pragma unroll
                for (int i = 0; i < KEYS; ++i) {
                    x[i] = exp2_fast(fmaf(s[mt][i / 4][i & 3], a.c2, -base));
                    if constexpr (TAIL) x[i] = on[i] ? x[i] : 0.0f;
                    sum[mt] += x[i];
                }
                p[mt] = Ops::probs(x);
            }
            if constexpr (TAIL) {
                // Keys behind the last may hold anything; nodes that a row does not see, too.
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
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int t = 0; t < VW; ++t)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) acc[mt][n][t] = Ops::pv(v[n], t, p[mt], acc[mt][n][t]);
            if (more) load_v(step + 1);
        };
        int step = 0;
        for (; step < steps && (t0 + step) * TILE + wave * STEP + STEP <= len; ++step) take(step, no_t{});
        for (; step < steps; ++step) take(step, yes_t{});

        // The four waves' sums, relative to the largest of their maxima.
        bad = __any(bad);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            sum[mt] = rows_sum(sum[mt]);
            if (bad) sum[mt] = __builtin_nanf("");
            if (grp == 0) {
                s_stat[wave][mt * 16 + col][0] = top[mt];
                s_stat[wave][mt * 16 + col][1] = sum[mt];
                if (wave == 0) s_sees[mt * 16 + col] = sees[mt];
            }
        }
        if (lane == 0) s_odd[wave] = odd;
        __syncthreads();
        const bool whole = t0 == 0 && t1 == tiles;
        odd = false;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) odd = odd || s_odd[i];
        // Where this piece's part goes: a unit that an earlier workgroup began, or one that begins here.
        const int slot = 2 * int(w) + (pos == first ? 0 : 1);
        float* stats = a.stats + int64_t(slot) * ROWS * 2;
        float* parts = a.parts + int64_t(slot) * ROWS * DT;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int r = mt * 16 + col;
            float all = kNegInf;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) all = fmaxf(all, s_stat[i][r][0]);
            const float f = rescale(top[mt], all);
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < VW; t += 4) {
                        const f32x4_t o = {acc[mt][n][t][e] * f, acc[mt][n][t + 1][e] * f, acc[mt][n][t + 2][e] * f,
                                           acc[mt][n][t + 3][e] * f};
                        *reinterpret_cast<f32x4_t*>(&s_acc[wave][col][n * BW + (grp * 4 + e) * VW + t]) = o;
                    }
            __syncthreads();
            for (int i = tid; i < 16 * (DT / 4); i += kThreads) {
                const int rr = i / (DT / 4), d = i % (DT / 4) * 4, row = mt * 16 + rr;
                if (row >= rows || d >= D) continue;
                f32x4_t o = *reinterpret_cast<const f32x4_t*>(&s_acc[0][rr][d]);
#pragma unroll
                for (int x = 1; x < kWaves; ++x) o += *reinterpret_cast<const f32x4_t*>(&s_acc[x][rr][d]);
                if (odd && row < live) add_odd<Fmt>(L, b, h, d, len, T, len / STEP * STEP, s_sees[row], o);
                float most = kNegInf, total = 0.0f;
#pragma unroll
                for (int x = 0; x < kWaves; ++x) most = fmaxf(most, s_stat[x][row][0]);
#pragma unroll
                for (int x = 0; x < kWaves; ++x) {
                    const float s = s_stat[x][row][1];
                    total += s_stat[x][row][0] == kNegInf ? (s == s ? 0.0f : s) : s * exp2_fast(s_stat[x][row][0] - most);
                }
                if (whole) {
                    const int node = (row0 + row) / a.group, g = row0 + row - node * a.group;
                    char* to = L.out + ((int64_t(b) * L.N + node) * L.q_heads + h * a.group + g) * int64_t(D) * ES + d * ES;
                    const float inv = 1.0f / total;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = row < live || (seq.state == 2 && (seq.n < 0 || seq.n > node)) ? o[e] * inv : 0.0f;
                    if constexpr (ES == 2) *reinterpret_cast<u32x2_t*>(to) = u32x2_t{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
                    else *reinterpret_cast<f32x4_t*>(to) = o;
                } else {
                    post(parts + row * DT + d, o[0], o[1]);
                    post(parts + row * DT + d + 2, o[2], o[3]);
                    if (d == 0) post(stats + row * 2, most, total);
                }
            }
            __syncthreads();
        }
        if (!whole) {
            // The last of the unit's workgroups joins their parts, in their order.
            const int64_t u0 = pos - t0, w0 = share.owner(u0), w1 = share.owner(u0 + tiles - 1);
            wait_memory();
            __syncthreads();
            if (tid == 0) s_arrived = arrive(&a.counters[w0]);
            __syncthreads();
            if (s_arrived == uint32_t(w1 - w0)) {
                const int first_slot = 2 * int(w0) + (share.begin(w0) == u0 ? 0 : 1);
                const int count = int(w1 - w0) + 1;
                for (int i = tid; i < ROWS * (DT / 4); i += kThreads) {
                    const int row = i / (DT / 4), d = i % (DT / 4) * 4;
                    if (row >= rows || d >= D) continue;
                    float most = kNegInf, total = 0.0f;
                    f32x4_t o = {0, 0, 0, 0};
                    for (int x = 0; x < count; ++x) {
                        const int64_t at = (x ? 2 * (w0 + x) : first_slot) * ROWS + row;
                        const float2 st = fetch(a.stats + at * 2);
                        const float2 lo = fetch(a.parts + at * DT + d), hi = fetch(a.parts + at * DT + d + 2);
                        const float now = fmaxf(most, st.x), f = rescale(most, now), g = rescale(st.x, now);
                        o = o * f + f32x4_t{lo.x, lo.y, hi.x, hi.y} * g;
                        total = total * f + (st.y == st.y ? st.y * g : st.y);
                        most = now;
                    }
                    const int node = (row0 + row) / a.group, g = row0 + row - node * a.group;
                    char* to = L.out + ((int64_t(b) * L.N + node) * L.q_heads + h * a.group + g) * int64_t(D) * ES + d * ES;
                    const float inv = 1.0f / total;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = row < live ? o[e] * inv : 0.0f;
                    if constexpr (ES == 2) *reinterpret_cast<u32x2_t*>(to) = u32x2_t{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
                    else *reinterpret_cast<f32x4_t*>(to) = o;
                }
                if (tid == 0) __hip_atomic_store(&a.counters[w0], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        pos += t1 - t0;
    }
}

int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Row tiles of a workgroup.
int row_tiles(int rows, int DT) {
    const int most = DT == 256 ? 2 : 4, want = (rows + 15) / 16;
    return want <= 1 ? 1 : want <= 2 ? 2 : most;
}

struct Workspace {
    size_t stats, parts, total;
};
Workspace layout(int rows, int DT) {
    const size_t R = size_t(row_tiles(rows, DT)) * 16, slots = 2 * kMaxGroups;
    Workspace w;
    w.stats = kMaxGroups * sizeof(uint32_t);
    w.parts = w.stats + slots * R * 2 * sizeof(float);
    w.total = w.parts + slots * R * DT * sizeof(float);
    return w;
}

template <typename Ops, int DT, int MT>
hipError_t launch_tiles(const TreeAttentionLaunch& L, AttentionArgs& a) {
    a.blocks = (L.N * a.group + 16 * MT - 1) / (16 * MT);
    int grid = L.cus * 2;
    if (grid > kMaxGroups) grid = kMaxGroups;
    const size_t lds = size_t(L.B + 1) * sizeof(int64_t);
    if (L.pages.page_size % 16 || L.head_dim != DT)
        return launch_kernel(&tree_attention_kernel<Ops, DT, MT, true>, dim3(grid), dim3(kThreads), lds, L.stream, a);
    return launch_kernel(&tree_attention_kernel<Ops, DT, MT, false>, dim3(grid), dim3(kThreads), lds, L.stream, a);
}

template <typename Ops, int DT>
hipError_t launch_dim(const TreeAttentionLaunch& L, AttentionArgs& a) {
    switch (row_tiles(L.N * a.group, DT)) {
        case 1: return launch_tiles<Ops, DT, 1>(L, a);
        case 2: return launch_tiles<Ops, DT, 2>(L, a);
        default:
            if constexpr (DT < 256) return launch_tiles<Ops, DT, 4>(L, a);
            else return hipErrorInvalidValue;
    }
}

template <typename Ops>
hipError_t launch_ops(const TreeAttentionLaunch& L, AttentionArgs& a) {
    switch (padded_dim(L.head_dim)) {
        case 64: return launch_dim<Ops, 64>(L, a);
        case 128: return launch_dim<Ops, 128>(L, a);
        default: return launch_dim<Ops, 256>(L, a);
    }
}

}  // namespace

size_t tree_attention_workspace(int B, int N, int q_heads, int kv_heads, int head_dim) {
    (void)B;
    return layout(N * (q_heads / kv_heads), padded_dim(head_dim)).total;
}

hipError_t launch_tree_attention(const TreeAttentionLaunch& L) {
    AttentionArgs a{};
    a.L = L;
    a.c2 = float((L.scale < 0.0f ? -double(L.scale) : double(L.scale)) * 1.4426950408889634);
    a.group = L.q_heads / L.kv_heads;
    const Workspace w = layout(L.N * a.group, padded_dim(L.head_dim));
    a.counters = reinterpret_cast<uint32_t*>(L.workspace);
    a.stats = reinterpret_cast<float*>(L.workspace + w.stats);
    a.parts = reinterpret_cast<float*>(L.workspace + w.parts);
    return L.dtype == OSD_BF16 ? launch_ops<Bf16Ops>(L, a) : launch_ops<F32Ops>(L, a);
}

}  // namespace osd
