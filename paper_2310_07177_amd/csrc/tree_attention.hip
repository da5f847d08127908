// tree_attention.hip -- osd_tree_attention: drafted tokens attend to the context
// in the paged cache, to their ancestors and to themselves.  Up to 16 rows of a kv
// head (single tokens): keys and values go from memory to registers.  Of V a lane reads whole 16-byte
// pieces of the keys that it holds, and picks the halves of each pair of keys apart,
// which is the transposition that the second product's A operand needs.
#include "tree_attention.hpp"

namespace osd {
namespace {

using namespace attention;

constexpr int kWaves = 4;  // of a workgroup: each takes its own keys of a tile
constexpr int kThreads = kWaves * kWave;

// DT: head_dim rounded up; GEN: pages that end inside tiles of
// 16 keys, or head_dim < DT.  A step is 16 or 32 keys of a wave, a tile those of the
// workgroup's four; the next step's keys and values are on their way while one is
// worked on, 16 KB a wave of DT = 128.  Bound by memory: single tokens of 64 sequences of up to 8192
// tokens, 1.34 GB, 216 us (6.2 TB/s; 244 us with loads that stay in the caches); one token over 2048
// 11.7 us, a chain of waits (length, page, keys, the join of the parts).
template <typename Ops, int DT, bool GEN>
__global__ __launch_bounds__(kThreads, DT == 256 ? 1 : 2) void tree_attention_kernel(Args a) {
    using Fmt = typename Ops::Fmt;
    constexpr int MT = 1;
    using R = Rows<Ops, DT, MT, kPiece<Ops, DT>>;
    using Value = typename Ops::template Value<R::VW>;
    const TreeAttentionLaunch& L = a.L;
    constexpr int ES = R::ES, KT = R::KT, STEP = 16 * KT, TILE = STEP * kWaves;
    constexpr int CHUNKS = R::CHUNKS, VW = R::VW, BW = R::BW, BLOCKS = R::BLOCKS, KEYS = R::KEYS;
    constexpr int ROWS = 16 * MT, PITCH = DT + 4;
    const int tid = int(threadIdx.x), lane = tid & (kWave - 1), col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int D = GEN ? L.head_dim : DT;
    const int row_bytes = GEN ? L.pages.row_bytes : DT * ES;

    extern __shared__ int s_tiles[];  // [B + 1]
    __shared__ float s_acc[kWaves][16][PITCH];
    __shared__ float s_stat[kWaves][ROWS][2];
    __shared__ uint64_t s_sees[ROWS];
    __shared__ int s_odd[kWaves];
    __shared__ int64_t s_place[ROWS];

    Division<kThreads, TILE> share;
    share.init(a, s_tiles);
    const int64_t w = int64_t(blockIdx.x), first = share.begin(w), end = share.end(a, w);

    for (int64_t pos = first; pos < end;) {
        const Piece p = share.template find<ROWS>(a, w, pos, first, end);
        const int len = p.seq.len, T = p.T;
        chunk_t q[MT][CHUNKS];
        R rows;
        bool bad = p.seq.state == 2;

        // Byte offsets of the tiles of 16 keys to come (!GEN), KT lanes a step, or of
        // the keys of the next step (GEN); out of the cache: its first.
        const int64_t head = int64_t(p.h) * L.pages.head_bytes;
        int64_t ahead = 0;
        auto look = [&](int j) {
            int64_t at = 0;
            if (j < T) {
                at = cache_place(L.pages, p.b, j);
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
                        k[kt][c] = __builtin_nontemporal_load(reinterpret_cast<const chunk_t*>(in ? at + c * Ops::kChunk * ES : at - grp * 16));
                        if (!in) k[kt][c] = chunk_t{0, 0, 0, 0};
                    } else {
                        k[kt][c] = __builtin_nontemporal_load(reinterpret_cast<const chunk_t*>(at + c * Ops::kChunk * ES));
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
                        v[n][kt * 4 + i].x = __builtin_nontemporal_load(
                            reinterpret_cast<const decltype(Value::x)*>(in ? at + n * BW * ES : at - col * VW * ES));
                    }
                }
            }
        };
        auto fill = [&](int step) {  // the offsets from `step` on
            if constexpr (GEN) ahead = look((p.t0 + step) * TILE + wave * STEP + (lane & (STEP - 1)));
            else ahead = look((p.t0 + step + lane / KT) * TILE + wave * STEP + (lane & (KT - 1)) * 16);
        };
        // The wave's steps: one in each tile, as long as there are keys.
        int steps = p.t1 - p.t0;
        if (steps > 0 && (p.t1 - 1) * TILE + wave * STEP >= T) --steps;
        steps = __builtin_amdgcn_readfirstlane(steps);
        constexpr int PERIOD = GEN ? 1 : kWave / KT;
        auto scores = [&](f32x4_t (&s)[MT][KT]) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    s[mt][kt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) s[mt][kt] = Ops::qk(k[kt][c], q[mt][c], s[mt][kt]);
                }
        };
        auto take = [&](int step, auto tail) {
            constexpr bool TAIL = decltype(tail)::value;
            const int j0 = (p.t0 + step) * TILE + wave * STEP;
            f32x4_t s[MT][KT];
            scores(s);
            // The next step's keys while this one's probabilities are formed.
            const bool more = step + 1 < steps;
            if (more) {
                if ((step + 1) % PERIOD == 0) fill(step + 1);
                load_k(step + 1);
            }
            if constexpr (TAIL) rows.mask(s, j0, p.seq);
            typename Ops::Probs pr[MT];
            rows.template soften<TAIL>(s, a.c2, pr);
            if constexpr (TAIL) rows.guard(v, j0, T);
            rows.add(v, pr);
            if (more) load_v(step + 1);
        };
        if (steps > 0) {
            fill(0);
            load_k(0);
            load_v(0);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            load_queries<Ops, CHUNKS, !GEN>(a, p, mt * 16 + col, D, q[mt]);
            rows.sees[mt] = 0;
        }
        if (p.t1 * TILE > len && T > 0) {
            bool tree;
            const uint64_t all = wave_ancestors(L.parent ? L.parent + int64_t(p.b) * L.N : nullptr, p.seq.n, &tree);
            bad = bad || !tree;
            const uint64_t nodes = p.seq.n < kWave ? (uint64_t(1) << p.seq.n) - 1 : ~uint64_t(0);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int node = (p.row0 + mt * 16 + col) / a.group;
                rows.sees[mt] = uint64_t(__shfl(static_cast<unsigned long long>(all), node & (kWave - 1))) & nodes;
            }
        }
        rows.clear();
        for (bool again = false; steps > 0; again = true) {
            if (again) {
                fill(0);
                load_k(0);
                load_v(0);
            }
            float most[MT];
            if (!again) {
                f32x4_t s[MT][KT];
                scores(s);
                if (p.t0 * TILE + wave * STEP + STEP > len) rows.mask(s, p.t0 * TILE + wave * STEP, p.seq);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) most[mt] = kNegInf;
                R::largest(s, most);
            } else {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) most[mt] = rows.seen[mt];
                rows.clear();
            }
            rows.refer(most, a.c2);
            int step = 0;
            for (; step < steps && (p.t0 + step) * TILE + wave * STEP + STEP <= len; ++step) take(step, no_t{});
            for (; step < steps; ++step) take(step, yes_t{});
            if (again || rows.served(a.c2)) break;
        }

        // The four waves' sums, relative to the largest of their references.
        bad = __any(bad);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const float sum = bad ? __builtin_nanf("") : rows_sum(rows.sum[mt]);
            if (sum == 0.0f || steps <= 0) rows.ref[mt] = kNegInf;
            if (grp == 0) {
                s_stat[wave][mt * 16 + col][0] = rows.ref[mt];
                s_stat[wave][mt * 16 + col][1] = sum;
                if (wave == 0) s_sees[mt * 16 + col] = rows.sees[mt];
            }
        }
        if (lane == 0) s_odd[wave] = rows.odd;
        if (tid < p.rows) s_place[tid] = row_place<Fmt>(a, p, tid, D);
        __syncthreads();
        const bool odd = s_odd[0] || s_odd[1] || s_odd[2] || s_odd[3];
        // Keys of the piece in steps that took 0 in the place of values that are not finite.
        const int odd_from = max(len / STEP * STEP, p.t0 * TILE), odd_to = min(T, p.t1 * TILE);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float all = kNegInf;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) all = fmaxf(all, s_stat[i][mt * 16 + col][0]);
            rows.template store<PITCH>(mt, rescale(rows.ref[mt], all), s_acc[wave][col], grp);
            __syncthreads();
            for (int i = tid; i < 16 * (DT / 4); i += kThreads) {
                const int rr = i / (DT / 4), d = i % (DT / 4) * 4, row = mt * 16 + rr;
                if (row >= p.rows || d >= D) continue;
                f32x4_t o = *reinterpret_cast<const f32x4_t*>(&s_acc[0][rr][d]);
#pragma unroll
                for (int x = 1; x < kWaves; ++x) o += *reinterpret_cast<const f32x4_t*>(&s_acc[x][rr][d]);
                if (odd && row < p.live) add_odd<Fmt>(L, p.b, p.h, d, len, odd_from, odd_to, s_sees[row], o);
                float most = kNegInf, total = 0.0f;
#pragma unroll
                for (int x = 0; x < kWaves; ++x) most = fmaxf(most, s_stat[x][row][0]);
#pragma unroll
                for (int x = 0; x < kWaves; ++x) {
                    const float s = s_stat[x][row][1];
                    total += s == s ? s * rescale(s_stat[x][row][0], most) : s;
                }
                if (p.whole) write_row<Fmt>(a, s_place[row], d, o, 1.0f / total);
                else post_part<ROWS, DT>(a, p.slot, row, d, o, most, total);
            }
            __syncthreads();
        }
        if (!p.whole) {
            join<Fmt, kThreads, ROWS, DT>(a, p, share.apart, D, s_place);
            __syncthreads();  // the places are free
        }
        pos += share.step(p);
    }
}

template <typename Ops, int DT>
hipError_t launch_dim(Args& a) {
    const TreeAttentionLaunch& L = a.L;
    a.blocks = 1;
    int grid = L.cus * 2;
    if (grid > kMaxGroups) grid = kMaxGroups;
    const size_t lds = size_t(L.B + 1) * sizeof(int);
    if (L.pages.page_size % 16 || L.head_dim != DT)
        return launch_kernel(&tree_attention_kernel<Ops, DT, true>, dim3(grid), dim3(kThreads), lds, L.stream, a);
    return launch_kernel(&tree_attention_kernel<Ops, DT, false>, dim3(grid), dim3(kThreads), lds, L.stream, a);
}

// Rows of a workgroup.
int block_rows(int rows, int DT, int dtype) {
    if (rows <= 16) return 16;
    if (rows <= 64 || (dtype != OSD_BF16 && DT == 256)) return 64;
    return rows <= 128 || DT == 256 || dtype != OSD_BF16 ? 128 : 256;
}

struct Workspace {
    size_t stats, parts, total;
};
Workspace layout(int rows, int DT, int dtype) {
    const size_t R = size_t(block_rows(rows, DT, dtype)), slots = 2 * kMaxGroups / (R > 16 ? 2 : 1);
    Workspace w;
    w.stats = kMaxGroups * 3 * sizeof(uint32_t);
    w.parts = w.stats + slots * R * 2 * sizeof(float);
    w.total = w.parts + slots * R * DT * sizeof(float);
    return w;
}

template <typename Ops>
hipError_t launch_ops(Args& a) {
    switch (padded_dim(a.L.head_dim)) {
        case 64: return launch_dim<Ops, 64>(a);
        case 128: return launch_dim<Ops, 128>(a);
        default: return launch_dim<Ops, 256>(a);
    }
}

}  // namespace

size_t tree_attention_workspace(int N, int q_heads, int kv_heads, int head_dim) {
    const int rows = N * (q_heads / kv_heads), DT = padded_dim(head_dim);
    const size_t bf16 = layout(rows, DT, OSD_BF16).total, f32 = layout(rows, DT, OSD_F32).total;
    return bf16 > f32 ? bf16 : f32;
}

hipError_t launch_tree_attention(const TreeAttentionLaunch& L) {
    Args a{};
    a.L = L;
    a.c2 = float((L.scale < 0.0f ? -double(L.scale) : double(L.scale)) * 1.4426950408889634);
    a.group = L.q_heads / L.kv_heads;
    const int DT = padded_dim(L.head_dim), R = block_rows(L.N * a.group, DT, L.dtype);
    const Workspace w = layout(L.N * a.group, DT, L.dtype);
    a.counters = reinterpret_cast<uint32_t*>(L.workspace);
    a.stats = reinterpret_cast<float*>(L.workspace + w.stats);
    a.parts = reinterpret_cast<float*>(L.workspace + w.parts);
    a.stats_bytes = uint32_t(w.parts - w.stats);
    a.parts_bytes = uint32_t(w.total - w.parts);
    if (R > 16) return L.dtype == OSD_BF16 ? launch_wide_bf16(a, R) : launch_wide_f32(a, R);
    return L.dtype == OSD_BF16 ? launch_ops<Bf16Ops>(a) : launch_ops<F32Ops>(a);
}

}  // namespace osd
