// cache.hip -- osd_cache_append and osd_cache_keep: new tokens into the paged
// cache, accepted paths to where the context ends.  Both only move rows; what
// bounds them is memory, and for the smallest calls the chain of dependent loads
// (length, table, page) that stands before the first store.
#include "cache_device.hpp"

namespace osd {
namespace {

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

// CH values of a head: 16 bytes where the sizes allow.
template <typename Fmt, int CH>
struct Values;
template <int CH>
struct Values<BF16, CH> {
    typedef uint16_t bits_t __attribute__((ext_vector_type(CH)));
    bits_t x;
    __device__ float get(int e) const { return __uint_as_float(uint32_t(x[e]) << 16); }
    __device__ void set(int e, float v) { x[e] = uint16_t(pack_bf16x2(v, v)); }
};
template <int CH>
struct Values<F32, CH> {
    typedef float bits_t __attribute__((ext_vector_type(CH)));
    bits_t x;
    __device__ float get(int e) const { return x[e]; }
    __device__ void set(int e, float v) { x[e] = v; }
};

struct AppendArgs {
    AppendLaunch L;
    int items;      // of a head: two chunks each
    int per_token;  // items of all heads
};

// A launch has at most 2^32 - 1 threads in a dimension: more tokens go to the second.
constexpr int64_t kAppendTokens = 1 << 21;

// One workgroup per token.  A thread takes two chunks of a head: with halves
// rotated the two that form pairs (so that a pair's values are read and written
// once, by one thread), otherwise two of equal distance.  Products and sums of the
// rotation are fp32, rounded once to the cache's type.
// Bound by memory: 8 prompts of 4096 tokens, 48 heads of 128 bf16 values, 822 MB read and
// written in 144 us (5.7 TB/s; a plain copy reaches 4.9), trees of 32 nodes of 64
// sequences 51 MB in 11.7 us.  One token takes 3.0 us, the chain of its dependent loads.
template <typename Fmt, int CH, bool PAIRS>
__global__ __launch_bounds__(1024) void append_kernel(AppendArgs a) {
    const AppendLaunch& L = a.L;
    constexpr int ES = Fmt::kBytes;
    using V = Values<Fmt, CH>;
    const int64_t at = int64_t(blockIdx.y) * kAppendTokens + blockIdx.x;
    if (at >= int64_t(L.B) * L.N) return;
    const int token = int(at), b = token / L.N, n = token - b * L.N;
    const int tid = int(threadIdx.x), lane = tid & (kWave - 1);
    const int D = L.head_dim, R = L.rotary_dim;
    const int len = L.seq_len[b], nb = L.new_len ? L.new_len[b] : L.N;
    // Its position, and where it goes.
    int depth = n;
    bool ok = nb >= 0 && nb <= L.N;
    if (L.parent) {
        bool tree;
        const uint64_t up = wave_ancestors(L.parent + int64_t(b) * L.N, ok ? nb : 0, &tree);
        depth = __popcll(__shfl(static_cast<unsigned long long>(up), n)) - 1;
        ok = ok && tree;
    }
    const bool none = len < 0 || (nb >= 0 && nb <= n);
    int64_t place = -1;
    if (!none && ok && len <= L.pages.capacity - 1 - n) place = cache_place(L.pages, b, len + n);
    ok = ok && place >= 0 && (!L.rotation || depth < L.rotation_rows - len);
    const float* turn = L.rotation + (ok && !none ? int64_t(len + depth) * R : 0);

    for (int i = tid; i < a.per_token; i += int(blockDim.x)) {
        const int head = i / a.items, j = i - head * a.items;
        const bool is_q = head < L.q_heads, is_v = head >= L.q_heads + L.kv_heads;
        if (!is_q && (none || !ok)) continue;
        const int h = is_q ? head : is_v ? head - L.q_heads - L.kv_heads : head - L.q_heads;
        const char* src = is_q ? L.q + at * L.q_stride : is_v ? L.v + at * L.v_stride : L.k + at * L.k_stride;
        char* dst = is_q ? L.q_out + at * L.q_out_stride + int64_t(h) * D * ES
                         : (is_v ? L.v_cache : L.k_cache) + place + h * L.pages.head_bytes;
        src += int64_t(h) * D * ES;
        // The chunks' first elements; the second may be none.
        int x = j * CH, y = (j + a.items) * CH;
        const bool half = !PAIRS && !is_v && x < R / 2;
        if (!PAIRS && !is_v && R > 0) {
            const int rest = (D - R + CH - 1) / CH, r = j - R / 2 / CH;
            x = half ? x : R + r * CH;
            y = half ? x + R / 2 : R + (r + (rest + 1) / 2) * CH;
        }
        const bool second = y < D;
        V u, w{};
        u.x = *reinterpret_cast<const typename V::bits_t*>(src + x * ES);
        if (second) w.x = *reinterpret_cast<const typename V::bits_t*>(src + y * ES);
        if (none || !ok) {
            const float f = none ? 0.0f : __builtin_nanf("");
#pragma unroll
            for (int e = 0; e < CH; ++e) u.set(e, f), w.set(e, f);
        } else if (half) {
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                const float c = turn[x + e], s = turn[R / 2 + x + e], p = u.get(e), q = w.get(e);
                u.set(e, fmaf(p, c, -(q * s)));
                w.set(e, fmaf(q, c, p * s));
            }
        } else if (PAIRS && !is_v) {
#pragma unroll
            for (int e = 0; e + 1 < CH; e += 2) {
                if (x < R) {
                    const float c = turn[(x + e) / 2], s = turn[R / 2 + (x + e) / 2], p = u.get(e), q = u.get(e + 1);
                    u.set(e, fmaf(p, c, -(q * s)));
                    u.set(e + 1, fmaf(q, c, p * s));
                }
                if (y < R) {
                    const float c = turn[(y + e) / 2], s = turn[R / 2 + (y + e) / 2], p = w.get(e), q = w.get(e + 1);
                    w.set(e, fmaf(p, c, -(q * s)));
                    w.set(e + 1, fmaf(q, c, p * s));
                }
            }
        }
        *reinterpret_cast<typename V::bits_t*>(dst + x * ES) = u.x;
        if (second) *reinterpret_cast<typename V::bits_t*>(dst + y * ES) = w.x;
    }
}

template <typename Fmt, int CH, bool PAIRS>
hipError_t launch_append_chunks(const AppendLaunch& L) {
    AppendArgs a{L, 0, 0};
    a.items = (L.head_dim / CH + 1) / 2;
    a.per_token = a.items * (L.q_heads + 2 * L.kv_heads);
    int threads = (a.per_token + kWave - 1) / kWave * kWave;
    if (threads > 1024) threads = 1024;
    const int64_t tokens = int64_t(L.B) * L.N;
    const dim3 grid(unsigned(tokens < kAppendTokens ? tokens : kAppendTokens),
                    unsigned((tokens + kAppendTokens - 1) / kAppendTokens));
    return launch_kernel(&append_kernel<Fmt, CH, PAIRS>, grid, dim3(threads), 0, L.stream, a);
}

// Chunks divide what is rotated (of halves, each half) and what is not.
template <typename Fmt>
hipError_t launch_append_fmt(const AppendLaunch& L) {
    constexpr int C = Fmt::kPerChunk;
    const bool pairs = L.style == OSD_ROTATE_PAIRS;
    const int r = pairs || !L.rotation ? L.rotary_dim : L.rotary_dim / 2;
    if (pairs) {
        if (r % C == 0) return launch_append_chunks<Fmt, C, true>(L);
        return launch_append_chunks<Fmt, 2, true>(L);
    }
    if (r % C == 0) return launch_append_chunks<Fmt, C, false>(L);
    if (r % 2 == 0) return launch_append_chunks<Fmt, 2, false>(L);
    return launch_append_chunks<Fmt, 1, false>(L);
}

// ---------------------------------------------------------------------------
// Keep
// ---------------------------------------------------------------------------

struct KeepArgs {
    KeepLaunch L;
    int chunks;  // of 16 bytes in a row
    int columns; // of all layers, both caches, all heads
};

// Bound by memory: paths of 64 sequences in 32 layers of 8 heads of 128 bf16 values, 52 MB read
// and written in 10.3 us (5.0 TB/s, the rate of a copy); one sequence's 3.6 us.
// A thread holds one 16-byte column of a head and moves the path's rows of it
// in order.  A node's place on the path is never behind the node itself
// (path[i] >= i + 1, ascending), so what a thread writes it has read before,
// and no two threads share a column.
constexpr int kKeepThreads = 256;
constexpr int kKeepBatch = 8;  // rows in flight (32 registers)

__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KeepArgs a) {
    const KeepLaunch& L = a.L;
    const int b = int(blockIdx.y), tid = int(threadIdx.x), lane = tid & (kWave - 1);
    __shared__ int64_t s_from[kWave], s_to[kWave];
    __shared__ int s_moves;
    const int len = L.seq_len[b], kept = L.accepted_len[b];
    if (tid < kWave) {
        // Lane i: node i of the path.
        bool ok = len >= 0 && kept >= 0 && kept < L.N && len < L.pages.capacity - kept;
        const int64_t row = int64_t(b) * L.N;
        const int node = ok && lane < kept ? L.path_nodes[row + lane] : 0;
        const int before = __shfl_up(node, 1);
        const bool on = ok && lane < kept;
        bool good = !on || (node > (lane ? before : 0) && node < L.N && len < L.pages.capacity - node);
        int64_t from = 0, to = 0;
        if (on && good) {
            from = cache_place(L.pages, b, len + node);
            to = cache_place(L.pages, b, len + 1 + lane);
            good = from >= 0 && to >= 0;
        }
        if (ok && lane == kWave - 1 && kept < kWave) good = good && cache_place(L.pages, b, len) >= 0;  // the root
        ok = ok && __ballot(!good) == 0;
        // Rows in place need no move.
        const bool moves = ok && on && from != to;
        const uint64_t set = __ballot(moves);
        if (moves) {
            const int k = __popcll(set & ((uint64_t(1) << lane) - 1));
            s_from[k] = from;
            s_to[k] = to;
        }
        if (lane == 0) {
            s_moves = __popcll(set);
            if (blockIdx.x == 0) L.new_seq_len[b] = ok ? len + 1 + kept : len;
        }
    }
    __syncthreads();
    const int moves = s_moves;
    const int col = int(blockIdx.x) * kKeepThreads + tid;
    if (moves == 0 || col >= a.columns) return;
    int rest = col / a.chunks;
    const int chunk = col - rest * a.chunks, layer = rest / (2 * L.kv_heads);
    rest -= layer * 2 * L.kv_heads;
    const bool is_v = rest >= L.kv_heads;
    const int h = is_v ? rest - L.kv_heads : rest;
    char* base = (is_v ? L.v_cache : L.k_cache) + layer * L.layer_bytes + h * L.pages.head_bytes + chunk * 16;
    for (int i = 0; i < moves; i += kKeepBatch) {
        chunk_t c[kKeepBatch];
#pragma unroll
        for (int k = 0; k < kKeepBatch; ++k)
            if (i + k < moves) c[k] = *reinterpret_cast<const chunk_t*>(base + s_from[i + k]);
#pragma unroll
        for (int k = 0; k < kKeepBatch; ++k)
            if (i + k < moves) *reinterpret_cast<chunk_t*>(base + s_to[i + k]) = c[k];
    }
}

}  // namespace

hipError_t launch_append(const AppendLaunch& L) {
    return L.dtype == OSD_BF16 ? launch_append_fmt<BF16>(L) : launch_append_fmt<F32>(L);
}

hipError_t launch_keep(const KeepLaunch& L) {
    KeepArgs a{L, L.pages.row_bytes / 16, 0};
    const int64_t columns = int64_t(L.layers) * 2 * L.kv_heads * a.chunks;
    if (columns > 0x7FFFFF00ll) return hipErrorInvalidValue;
    a.columns = int(columns);
    return launch_kernel(&keep_kernel, dim3(unsigned((columns + kKeepThreads - 1) / kKeepThreads), unsigned(L.B)),
                         dim3(kKeepThreads), 0, L.stream, a);
}

}  // namespace osd
