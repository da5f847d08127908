// tree_attention_wide.hpp -- osd_tree_attention of many rows: eight waves read keys
// and values from LDS, where they arrive directly from memory.  (Compiled once for each
// type.)
#pragma once

#include "tree_attention.hpp"

namespace osd {
namespace attention {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kPageWindow = 512;  // pages looked up at once

// 16 bytes a lane from memory to LDS at `to` (uniform) + 16 * lane, without a register on
// the way.  Counted in vmcnt; the compiler does not know of it, so that reads of LDS
// wait for it only where wait_stage() says so.  (hipcc warns that M0, which it names itself where it needs it, is no
// register that it keeps for others: nothing here does.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_lds(const char* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(from), "s"(to) : "m0", "memory");
}
#pragma clang diagnostic pop
// All but the wave's LEFT newest loads are there, then those of all waves.
template <int LEFT>
__device__ inline void wait_stage() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}
// The transposing read: 16 lanes give the places of 4 keys' pieces of 16 elements (8 bytes
// a lane, four lanes a key) and get an element of the 4 keys each.
typedef short s16x4_t __attribute__((ext_vector_type(4)));
__device__ inline u32x2_t transposed(const char* at) {
    return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                           (__attribute__((address_space(3))) s16x4_t*)(const_cast<char*>(at))));
}

// WR waves share the rows, 16 MT each, WK = 8 / WR the keys of a stage.  The ring of
// stages in LDS is filled NST - 1 ahead.  32 sequences of 4032 to 4080 tokens, 8 kv heads of 128 bf16
// values: 64 rows 97 us (5.5 TB/s), 128 rows 143 us, 256 rows 240 us (859 TFLOP/s of executed products),
// which as two blocks of 128 would take 286.  Few rows are bound by memory, many by products and exponentials in
// turn.  Eight waves of 32 rows: sixteen of 16 rows read K and V from LDS twice as often, and spilled.  (Of DT = 128
// waves of 32 rows keep 22 to 34 registers in scratch, those of DT = 256 11 to 52.)
template <typename Ops, int DT, int WR, int MT>
struct Shape {
    static constexpr int ES = Ops::Fmt::kBytes, STEP = 16 * Ops::kKT, ROW = DT * ES;
    static constexpr int WK = kWaves / WR, FIT = 16384 / ROW < 64 ? 16384 / ROW : 64;
    static constexpr int STAGE = FIT > STEP * WK ? FIT : STEP * WK;
    static constexpr int ROWS = 16 * MT * WR, PITCH = DT + 4;
    static constexpr int TILE_BYTES = STAGE * ROW;  // of K, and of V
    static constexpr int NST = TILE_BYTES > 16384 ? 2 : 4;
    static constexpr int RING = NST * 2 * TILE_BYTES, MERGE = kWaves * 16 * PITCH * 4;
    static constexpr int LDS = RING > MERGE ? RING : MERGE;
    static constexpr int LOADS = TILE_BYTES / 1024 / kWaves;  // of K, and of V, of a wave for a stage
    static constexpr int CPR = ROW / 16;                      // 16-byte chunks of a row
};

// DT: head_dim rounded up to a power of two, as rows lie in LDS; NC: tiles of 16 of its
// values that are computed; FULL: all DT of them.
template <typename Ops, int DT, int WR, int MT, int NC, bool FULL>
__global__ __launch_bounds__(kThreads, 2) void tree_attention_wide(Args a) {
    using Fmt = typename Ops::Fmt;
    using S = Shape<Ops, DT, WR, MT>;
    using R = Rows<Ops, NC * 16, MT, 1>;
    constexpr int ES = S::ES, CHUNKS = R::CHUNKS, KT = R::KT, STEP = S::STEP, STAGE = S::STAGE, ROWS = S::ROWS;
    constexpr int PITCH = S::PITCH, CPR = S::CPR, ROW = S::ROW;
    // Tiles that lie in the head whole, whatever its size (of those that launch_shape sends here).
    constexpr int WHOLE = FULL ? NC : DT == 64 ? 0 : DT == 256 ? 8 : NC == 8 ? 6 : NC - 1;
    static_assert(WR == 4 || WR == kWaves, "two waves share keys, or one, or two with half of the rows");
    const TreeAttentionLaunch& L = a.L;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    const int D = FULL ? DT : L.head_dim;

    extern __shared__ int s_tiles[];  // [B + 1]
    __shared__ __attribute__((aligned(1024))) char s_ring[S::LDS];
    __shared__ float s_stat[kWaves][16 * MT][2];
    __shared__ uint64_t s_sees[ROWS];
    __shared__ int s_flags[kWaves];
    __shared__ int s_page[kPageWindow];
    __shared__ int64_t s_place[ROWS];
    __shared__ float s_total[ROWS][2];  // maximum; sum, or its reciprocal
    float(*s_acc)[16][PITCH] = reinterpret_cast<float(*)[16][PITCH]>(s_ring);
    const uint32_t ring = uint32_t(uintptr_t((__attribute__((address_space(3))) char*)s_ring));

    Division<kThreads, STAGE> share;
    share.init(a, s_tiles);
    const int64_t w = int64_t(blockIdx.x), first = share.begin(w), end = share.end(a, w);

    // A row's chunks lie permuted (chunk ^ key, of period 16; rows of 128 bytes lie two to
    // 64 banks), so that 16 lanes that read one chunk of 16 keys meet 16 different
    // places; the DMA writes lanes one after another, so the permutation is in what they read.
    const auto swizzle = [](int key) { return CPR == 8 ? (key >> 1) & 7 : key & 15; };
    // Of each of the wave's loads: its first key in the stage (of 1024 / ROW), and the lane's place from there.
    int lane_key[S::LOADS], lane_chunk[S::LOADS];
#pragma unroll
    for (int x = 0; x < S::LOADS; ++x) {
        const int lane = int(threadIdx.x) & (kWave - 1), at = (wave * S::LOADS + x) * kWave + lane, key = at / CPR;
        lane_key[x] = lane / CPR;
        lane_chunk[x] = (at % CPR) ^ swizzle(key);
    }
    const bool even_pages = L.pages.page_size % 8 == 0;  // a load's keys (8 at most) lie on one page

    for (int64_t pos = first; pos < end;) {
        const int tid = here(int(threadIdx.x)), lane = tid & (kWave - 1), col = lane & 15, grp = lane >> 4;
        const Piece p = share.template find<ROWS>(a, w, pos, first, end);
        const int len = p.seq.len, T = p.T;
        bool bad = p.seq.state == 2;
        const int64_t head = int64_t(p.h) * L.pages.head_bytes;

        // The pages from page0 on; a stage's keys behind the last stand for the last.
        const int stages = T > 0 ? p.t1 - p.t0 : 0;
        int page0 = 0, page_end = 0;
        const auto page_of = [&](int j) { return int((uint64_t(uint32_t(j)) * L.pages.magic) >> L.pages.shift); };
        auto look = [&](int st) {  // uniform: the stage's pages are in the window
            int j1 = (p.t0 + st + 1) * STAGE - 1;
            j1 = j1 < T ? j1 : T - 1;
            if (page_of(j1) < page_end) return;
            page0 = page_of((p.t0 + st) * STAGE);
            page_end = page0 + kPageWindow;
            __syncthreads();
            const int last = page_of(T - 1);
            if (page0 + tid <= last) {
                int page = L.pages.table[int64_t(p.b) * L.pages.table_len + page0 + tid];
                if (uint32_t(page) >= uint32_t(L.pages.pages)) {
                    bad = true;
                    page = 0;
                }
                s_page[tid] = page;
            }
            __syncthreads();
        };
        static_assert(kThreads == kPageWindow, "a page for each thread");
        auto issue = [&](int st) {
            look(st);
            const uint32_t to = ring + uint32_t(st % S::NST) * (2 * S::TILE_BYTES);
            constexpr int KEYS_OF = 1024 / ROW > 0 ? 1024 / ROW : 1;  // keys of a load
            int64_t from[S::LOADS];
            if (even_pages) {
                int page[S::LOADS], slot[S::LOADS];
#pragma unroll
                for (int x = 0; x < S::LOADS; ++x) {
                    const int key = (p.t0 + st) * STAGE + (wave * S::LOADS + x) * KEYS_OF, last = (T - 1) / KEYS_OF * KEYS_OF;
                    const int j = key < last ? key : last, in = page_of(j);
                    page[x] = s_page[in - page0];
                    slot[x] = j - in * L.pages.page_size;
                }
#pragma unroll
                for (int x = 0; x < S::LOADS; ++x)
                    from[x] = int64_t(__builtin_amdgcn_readfirstlane(page[x])) * L.pages.page_bytes + head +
                              int64_t(slot[x]) * (D * ES) + (lane_key[x] * (D * ES) + lane_chunk[x] * 16);
            } else {
#pragma unroll
                for (int x = 0; x < S::LOADS; ++x) {
                    int j = (p.t0 + st) * STAGE + (wave * S::LOADS + x) * KEYS_OF + lane_key[x];
                    j = j < T ? j : T - 1;
                    const int in = page_of(j);
                    from[x] = int64_t(s_page[in - page0]) * L.pages.page_bytes + head +
                              int64_t(j - in * L.pages.page_size) * (D * ES) + lane_chunk[x] * 16;
                }
            }
#pragma unroll
            for (int x = 0; x < S::LOADS; ++x) {
                const uint32_t unit = to + uint32_t(wave * S::LOADS + x) * 1024u;
                if (FULL || lane_chunk[x] * 16 < D * ES) {  // (what lies behind a row in LDS is not used)
                    load_lds(L.k_cache + from[x], unit);
                    load_lds(L.v_cache + from[x], unit + S::TILE_BYTES);
                }
            }
        };
        for (int st = 0; st < S::NST - 1 && st < stages; ++st) issue(st);

        // Half of the rows in use (a batch's smaller trees): the waves without rows take half of the keys.
        constexpr bool HALVES = WR == kWaves && STAGE / STEP % 2 == 0;
        const int half = HALVES && p.live * 2 <= ROWS ? 1 : 0;
        const int row_waves = WR >> half, key_waves = S::WK << half;
        // (Waves that share rows are neighbours, so that few rows, too, are spread over all SIMDs.)
        const int wr = wave / key_waves, wk = wave & (key_waves - 1);
        const bool alive = wr * MT * 16 < p.live;  // (of padding alone: a wave helps to fill the ring)
        chunk_t q[MT][CHUNKS];
        R rows;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            load_queries<Ops, CHUNKS, FULL>(a, p, (wr * MT + mt) * 16 + col, D, q[mt]);
            rows.sees[mt] = 0;
        }
        if (p.t1 * STAGE > len && T > 0) {
            bool tree;
            const uint64_t all = wave_ancestors(L.parent ? L.parent + int64_t(p.b) * L.N : nullptr, p.seq.n, &tree);
            bad = bad || !tree;
            const uint64_t nodes = p.seq.n < kWave ? (uint64_t(1) << p.seq.n) - 1 : ~uint64_t(0);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int node = (p.row0 + (wr * MT + mt) * 16 + col) / a.group;
                rows.sees[mt] = uint64_t(__shfl(static_cast<unsigned long long>(all), node & (kWave - 1))) & nodes;
            }
        }

        auto scores = [&](const char* k_row, int k_lane, f32x4_t (&s)[MT][KT]) {
            // All of K's operands are read before the first product, V's a batch ahead of theirs and the first
            // before the exponentials.  (The compiler would read each where it is used, and every
            // one of the 24 reads of a step would wait for LDS.)
            chunk_t k[CHUNKS][KT];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
                    k[c][kt] = *reinterpret_cast<const chunk_t*>(k_row + kt * 16 * ROW + (k_lane ^ c * 64));
            __builtin_amdgcn_sched_barrier(0);
            f32x4_t odd_chunks[MT][KT];  // (fp32: two sums in turn)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) s[mt][kt] = odd_chunks[mt][kt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    if (!FULL && c * Ops::kChunk + grp * (16 / ES) >= D) k[c][kt] = chunk_t{0, 0, 0, 0};
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        f32x4_t& sum = ES == 4 && (c & 1) ? odd_chunks[mt][kt] : s[mt][kt];
                        sum = Ops::qk(k[c][kt], q[mt][c], sum);
                    }
                }
            if constexpr (ES == 4) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) s[mt][0] += odd_chunks[mt][0];
            }
        };
        auto take = [&](int st, int k0, auto tail) {
            constexpr bool TAIL = decltype(tail)::value;
            const int j0 = (p.t0 + st) * STAGE + k0;
            const char* k_row = s_ring + (st % S::NST) * (2 * S::TILE_BYTES) + (k0 + col) * ROW;
            // (A chunk's place is a XOR of the lane's part and a constant; computed each time, as all of
            // them together would hold 30 registers.)
            int k_lane = (grp ^ swizzle(col)) * 16;
            const char* v_row;
            int v_lane;
            if constexpr (ES == 2) {  // the key whose piece of V this lane reads for the others
                const int from = grp * 4 + (col >> 2);
                v_row = k_row + S::TILE_BYTES + (from - col) * ROW + (col & 1) * 8;
                v_lane = (((col & 3) >> 1) ^ swizzle(from)) * 16;
            } else {
                v_row = k_row + S::TILE_BYTES + (grp * 4 - col) * ROW + (col & 3) * 4;
                v_lane = ((col >> 2) ^ swizzle(grp * 4)) * 16;
            }
            asm volatile("" : "+v"(k_lane), "+v"(v_lane));
            f32x4_t s[MT][KT];
            scores(k_row, k_lane, s);
            constexpr int BATCH = 4, BATCHES = (NC + BATCH - 1) / BATCH;  // tiles of V
            chunk_t v[2][BATCH];
            auto read_v = [&](int batch) {
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    const int t = batch * BATCH + u;
                    if (t >= NC) continue;
                    if constexpr (ES == 2) {
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) {
                            const u32x2_t half_of = transposed(v_row + kt * 16 * ROW + (v_lane ^ t * 32));
                            v[batch & 1][u][2 * kt] = half_of.x;
                            v[batch & 1][u][2 * kt + 1] = half_of.y;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[batch & 1][u][i] = *reinterpret_cast<const uint32_t*>(v_row + i * ROW + (v_lane ^ (i * 16) ^ t * 64));
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            read_v(0);
            if constexpr (TAIL) rows.mask(s, j0, p.seq);
            typename Ops::Probs pr[MT];
            rows.template soften<TAIL>(s, a.c2, pr);
            // The lane's keys that are keys.
            chunk_t in;
            if constexpr (TAIL) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + (ES == 2 ? (i / 2) * 16 + grp * 4 + (i & 1) * 2 : grp * 4 + i);
                    in[i] = ES == 2 ? (j < T ? 0xFFFFu : 0u) | (j + 1 < T ? 0xFFFF0000u : 0u) : j < T ? ~0u : 0u;
                }
            }
#pragma unroll
            for (int batch = 0; batch < BATCHES; ++batch) {
                if (batch + 1 < BATCHES) read_v(batch + 1);
                if constexpr (TAIL) {
                    uint32_t carries = 0;
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        if (batch * BATCH + u >= NC) continue;
                        v[batch & 1][u] &= in;
                        const int t = batch * BATCH + u;
                        if (t < WHOLE || t * 16 + col < D) carries |= Ops::carries(v[batch & 1][u]);
                    }
                    if (__any((carries & Ops::kSigns) != 0)) {
                        rows.odd = true;
#pragma unroll
                        for (int u = 0; u < BATCH; ++u)
                            if (batch * BATCH + u < NC) Ops::clean(v[batch & 1][u]);
                    }
                }
                // (Products of several tiles in turn: each of fp32 would wait for the one before it.)
#pragma unroll
                for (int i = 0; i < Ops::kParts; ++i)
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        const int t = batch * BATCH + u;
                        if (t >= NC) continue;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) rows.acc[mt][t][0] = Ops::pv_part(v[batch & 1][u], pr[mt], i, rows.acc[mt][t][0]);
                    }
            }
        };
        rows.clear();
        for (bool again = false;; again = true) {
            if (again) {
                float most[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) most[mt] = rows.seen[mt];
                rows.clear();
                rows.refer(most, a.c2);
                page_end = 0;
                for (int st = 0; st < S::NST - 1 && st < stages; ++st) issue(st);
            }
            auto arrive_at = [&](int st) {
                // This stage is there; the ones behind it may be on their way.
                if (S::NST > 2 && st + 2 < stages) wait_stage<(S::NST > 2 ? 4 * S::LOADS : 0)>();
                else if (S::NST > 2 && st + 1 < stages) wait_stage<(S::NST > 2 ? 2 * S::LOADS : 0)>();
                else wait_stage<0>();
            };
            auto stage = [&](int st, auto tail) {
                arrive_at(st);
                if (S::NST == 2 && st + 1 < stages) issue(st + 1);
                if (alive) {
#pragma unroll
                    for (int sub = 0; sub < STAGE / STEP / S::WK; ++sub) {
                        const int k0 = (sub * key_waves + wk) * STEP;
                        if (HALVES && k0 >= STAGE) continue;
                        if (!decltype(tail)::value || (p.t0 + st) * STAGE + k0 < T) take(st, k0, tail);
                    }
                }
                // (Sent for here, where the waves have drifted apart, rather than by all at once above.)
                if (S::NST > 2 && st + S::NST - 1 < stages) issue(st + S::NST - 1);
            };
            if (!again) {  // the reference: the wave's first step
                float most[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) most[mt] = kNegInf;
                if (stages > 0) {
                    arrive_at(0);
                    if (alive) {
                        f32x4_t s[MT][KT];
                        scores(s_ring + (wk * STEP + col) * ROW, (grp ^ swizzle(col)) * 16, s);
                        if (p.t0 * STAGE + wk * STEP + STEP > len) rows.mask(s, p.t0 * STAGE + wk * STEP, p.seq);
                        R::largest(s, most);
                    }
                }
                rows.refer(most, a.c2);
            }
            // Stages of the context alone, then those with keys that not every row sees.  (Two loops: where the
            // two kinds of step met, all sums went through a copy.)
            int st = 0;
            for (const int plain = len / STAGE - p.t0 < stages ? len / STAGE - p.t0 : stages; st < plain; ++st) stage(st, no_t{});
            for (; st < stages; ++st) stage(st, yes_t{});
            // Columns behind the head's last hold what LDS held, which says nothing about the sums (nor, above, about
            // values that are not finite: with those counted, heads of 72 took 148 us instead of 44).
#pragma unroll
            for (int t = WHOLE; t < NC; ++t)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) rows.acc[mt][t][0][e] = t * 16 + grp * 4 + e < D ? rows.acc[mt][t][0][e] : 0.0f;
            // All waves share the stages, so that one that needs them again has all go through them.
            const bool ok = again || rows.served(a.c2);
            if (lane == 0) s_flags[wave] = ok;
            __syncthreads();
            int all = 1;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) all &= s_flags[i];
            if (all) break;
        }

        // The sums of the waves that share rows, relative to the largest of their references.
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const float sum = rows_sum(rows.sum[mt]);
            if (sum == 0.0f) rows.ref[mt] = kNegInf;
            if (grp == 0) {
                s_stat[wave][mt * 16 + col][0] = rows.ref[mt];
                s_stat[wave][mt * 16 + col][1] = sum;
                if (wk == 0) s_sees[(wr * MT + mt) * 16 + col] = rows.sees[mt];
            }
        }
        bad = __any(bad);
        __syncthreads();
        if (lane == 0) s_flags[wave] = (bad ? 1 : 0) | (rows.odd ? 2 : 0);
        __syncthreads();
        int flags = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) flags |= s_flags[i];
        // What all values of a row share, once for each: its sums (with half of the rows in use the other
        // half is padding: zeros), where it goes.
        const int t0 = here(tid), col0 = t0 & 15, grp0 = (t0 & (kWave - 1)) >> 4;
        if (t0 < ROWS) {
            const int x = t0 / (16 * MT), at = t0 % (16 * MT);
            float most = kNegInf, total = 0.0f;
            if (x < row_waves) {
                for (int y = 0; y < key_waves; ++y) most = fmaxf(most, s_stat[x * key_waves + y][at][0]);
                for (int y = 0; y < key_waves; ++y) {
                    const float s = s_stat[x * key_waves + y][at][1];
                    total += s == s ? s * rescale(s_stat[x * key_waves + y][at][0], most) : s;
                }
            }
            if (flags & 1) total = __builtin_nanf("");
            s_total[t0][0] = most;
            s_total[t0][1] = p.whole ? 1.0f / total : total;
            s_place[t0] = t0 < p.rows ? row_place<Fmt>(a, p, t0, D) : -1;
        }
        // (A thread's values of ITEMS rows at once: one after another they would wait for LDS.)
        constexpr int EACH = WR * 16 * (DT / 4) / kThreads, ITEMS = EACH < 4 ? EACH : 4;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float all = kNegInf;
            for (int i = 0; i < key_waves; ++i) all = fmaxf(all, s_stat[wr * key_waves + i][mt * 16 + col0][0]);
            rows.template store<PITCH>(mt, rescale(rows.ref[mt], all), s_acc[wave][col0], grp0);
            __syncthreads();
#pragma nounroll
            for (int i0 = 0; i0 < EACH; i0 += ITEMS) {
                f32x4_t o[ITEMS];
                float most[ITEMS], total[ITEMS];
                int64_t place[ITEMS];
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    const int i = (i0 + k) * kThreads + t0, x = i / (16 * (DT / 4)), r = i / (DT / 4) % 16, d = i % (DT / 4) * 4;
                    const int row = (x * MT + mt) * 16 + r;
                    place[k] = s_place[row];
                    most[k] = s_total[row][0];
                    total[k] = s_total[row][1];
                    const bool sums = x < row_waves;
                    o[k] = *reinterpret_cast<const f32x4_t*>(&s_acc[sums ? x * key_waves : 0][r][d]);
                    if (WR < kWaves || half) o[k] += *reinterpret_cast<const f32x4_t*>(&s_acc[sums ? x * key_waves + 1 : 0][r][d]);
                    if (!sums) o[k] = f32x4_t{0, 0, 0, 0};
                }
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    const int i = (i0 + k) * kThreads + t0, x = i / (16 * (DT / 4)), r = i / (DT / 4) % 16, d = i % (DT / 4) * 4;
                    const int row = (x * MT + mt) * 16 + r;
                    if (place[k] < 0 || (!FULL && d >= D)) continue;
                    // (The piece's keys in stages that took 0 in the place of values that are not finite.)
                    if ((flags & 2) && row < p.live)
                        add_odd<Fmt>(L, p.b, p.h, d, len, max(len / STAGE * STAGE, p.t0 * STAGE), min(T, p.t1 * STAGE), s_sees[row], o[k]);
                    if (p.whole) write_row<Fmt>(a, place[k], d, o[k], total[k]);
                    else post_part<ROWS, DT>(a, p.slot, row, d, o[k], most[k], total[k]);
                }
            }
            __syncthreads();
        }
        if (!p.whole) join<Fmt, kThreads, ROWS, DT>(a, p, share.apart, D, s_place);
        pos += share.step(p);
        __syncthreads();  // the ring and the pages are free
    }
}

template <typename Ops, int DT, int WR, int MT>
hipError_t launch_shape(Args& a) {
    const TreeAttentionLaunch& L = a.L;
    constexpr int ROWS = Shape<Ops, DT, WR, MT>::ROWS;
    a.blocks = (L.N * a.group + ROWS - 1) / ROWS;
    const int grid = L.cus < kMaxGroups / 2 ? L.cus : kMaxGroups / 2;
    const size_t lds = size_t(L.B + 1) * sizeof(int);
    if (L.head_dim == DT)
        return launch_kernel(&tree_attention_wide<Ops, DT, WR, MT, DT / 16, true>, dim3(grid), dim3(kThreads), lds, L.stream, a);
    if constexpr (DT == 128) {  // heads of 80 and 96 without the products of what they lack
        if (L.head_dim <= 80)
            return launch_kernel(&tree_attention_wide<Ops, DT, WR, MT, 5, false>, dim3(grid), dim3(kThreads), lds, L.stream, a);
        if (L.head_dim <= 96)
            return launch_kernel(&tree_attention_wide<Ops, DT, WR, MT, 6, false>, dim3(grid), dim3(kThreads), lds, L.stream, a);
    }
    return launch_kernel(&tree_attention_wide<Ops, DT, WR, MT, DT / 16, false>, dim3(grid), dim3(kThreads), lds, L.stream, a);
}

// (Waves of 32 rows: their sums of DT = 256 are 128 registers.  In fp32 sums and queries of DT = 128 are 64 each, of heads
// up to 96 48 each; whether waves of 32 fp32 rows are faster is not measured.)
template <typename Ops, int DT>
hipError_t launch_dim(Args& a, int rows) {
    if (rows <= 64) return launch_shape<Ops, DT, 4, 1>(a);
    if constexpr (Ops::Fmt::kBytes == 2 && DT < 256)
        return rows <= 128 ? launch_shape<Ops, DT, 4, 2>(a) : launch_shape<Ops, DT, 8, 2>(a);
    else if constexpr (Ops::Fmt::kBytes == 2 || DT < 256) return launch_shape<Ops, DT, 8, 1>(a);
    else return hipErrorInvalidValue;
}

template <typename Ops>
hipError_t launch_ops(Args& a, int rows) {
    switch (padded_dim(a.L.head_dim)) {
        case 64: return launch_dim<Ops, 64>(a, rows);
        case 128: return launch_dim<Ops, 128>(a, rows);
        default: return launch_dim<Ops, 256>(a, rows);
    }
}

}  // namespace
}  // namespace attention
}  // namespace osd
