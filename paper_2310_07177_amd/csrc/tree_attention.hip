// tree_attention.hip -- osd_tree_attention: drafted tokens attend to the context
// in the paged cache, to their ancestors and to themselves.
#include "cache_device.hpp"

namespace osd {
namespace {

struct AttentionArgs {
    TreeAttentionLaunch L;
    float c2;  // scale * log2(e)
};

// One wave per row (sequence, node, query head): 64 keys at a time, a lane for
// each, then the lanes take the head's values.  Softmax in one pass with the
// running maximum and sum.
template <typename Fmt>
__global__ __launch_bounds__(kWave) void tree_attention_rows(AttentionArgs a) {
    const TreeAttentionLaunch& L = a.L;
    constexpr int ES = Fmt::kBytes;
    __shared__ float s_q[OSD_MAX_HEAD_DIM], s_p[kWave];
    __shared__ int64_t s_at[kWave];
    const int lane = int(threadIdx.x), D = L.head_dim;
    const int hq = int(blockIdx.x), n = int(blockIdx.y), b = int(blockIdx.z), h = hq / (L.q_heads / L.kv_heads);
    const int len = L.seq_len[b], nb = L.new_len ? L.new_len[b] : L.N;
    const int64_t token = int64_t(b) * L.N + n;
    char* out = L.out + (token * L.q_heads + hq) * D * ES;
    bool ok = cache_fits(L.pages, len, nb, L.N), tree = true;
    const uint64_t all = wave_ancestors(L.parent ? L.parent + int64_t(b) * L.N : nullptr, ok ? nb : 0, &tree);
    const uint64_t sees = uint64_t(__shfl(static_cast<unsigned long long>(all), n));
    ok = ok && tree;
    for (int d = lane; d < D; d += kWave) s_q[d] = Fmt::load_one(L.q + token * L.q_stride + int64_t(hq) * D * ES, d);
    __syncthreads();
    float acc[OSD_MAX_HEAD_DIM / kWave] = {}, m = kNegInf, sum = 0.0f;
    const bool none = len < 0 || (nb >= 0 && nb <= n);
    const int T = none || !ok ? 0 : len + nb;
    for (int j0 = 0; j0 < T; j0 += kWave) {
        const int j = j0 + lane;
        int64_t at = 0;
        bool on = j < T;
        if (on) {
            at = cache_place(L.pages, b, j);
            ok = ok && at >= 0;
            at += h * L.pages.head_bytes;
            on = ok && (j < len || (sees >> (j - len) & 1));
        }
        float x = 0.0f;
        if (on)
            for (int d = 0; d < D; ++d) x = fmaf(s_q[d], Fmt::load_one(L.k_cache + at, d), x);
        x = on ? x * a.c2 : kNegInf;
        float top = x;
        for (int s = 1; s < kWave; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
        top = fmaxf(top, m);
        const float base = top == kNegInf ? 0.0f : top;
        const float p = on ? exp2_fast(x - base) : 0.0f, scale = exp2_fast(m - base);
        m = top;
        float ps = p;
        for (int s = 1; s < kWave; s *= 2) ps += __shfl_xor(ps, s);
        sum = sum * scale + ps;
        s_p[lane] = p;
        s_at[lane] = on ? at : -1;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < OSD_MAX_HEAD_DIM / kWave; ++i) {
            const int d = lane + i * kWave;
            if (d < D) {
                float o = acc[i] * scale;
                for (int k = 0; k < kWave; ++k)
                    if (s_at[k] >= 0) o = fmaf(s_p[k], Fmt::load_one(L.v_cache + s_at[k], d), o);
                acc[i] = o;
            }
        }
        __syncthreads();
    }
    ok = __ballot(!ok) == 0;
#pragma unroll
    for (int i = 0; i < OSD_MAX_HEAD_DIM / kWave; ++i) {
        const int d = lane + i * kWave;
        if (d >= D) continue;
        const float o = none ? 0.0f : ok ? acc[i] / sum : __builtin_nanf("");
        if (ES == 2) reinterpret_cast<uint16_t*>(out)[d] = uint16_t(pack_bf16x2(o, o));
        else reinterpret_cast<float*>(out)[d] = o;
    }
}

}  // namespace

size_t tree_attention_workspace(int B, int N, int q_heads, int kv_heads, int head_dim) { return 256; }

hipError_t launch_tree_attention(const TreeAttentionLaunch& L) {
    AttentionArgs a{L, float(double(L.scale) * 1.4426950408889634)};
    const dim3 grid(L.q_heads, L.N, L.B);
    return L.dtype == OSD_BF16 ? launch_kernel(&tree_attention_rows<BF16>, grid, dim3(kWave), 0, L.stream, a)
                               : launch_kernel(&tree_attention_rows<F32>, grid, dim3(kWave), 0, L.stream, a);
}

}  // namespace osd
