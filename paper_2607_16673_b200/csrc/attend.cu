// Verification by an attention layer: draft nodes attend the committed rows of a paged cache and their own ancestors.
#include "attn.cuh"

namespace speca {
namespace {

constexpr int kWarps = 4;

// One warp a row (node, query head): keys one at a time, running maximum and sum.
template <int D>
__global__ void __launch_bounds__(kWarps * 32)
attend_kernel(AttnParams p)
{
    after_previous_kernel();
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    const long task = long(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    if (task >= long(p.L) * p.T * p.H) return;
    const int h = int(task % p.H), t = int(task / p.H % p.T), l = int(task / p.H / p.T), hk = h / (p.H / p.HK);
    int b = 0;
    for (int i = lane; i < p.B; i += 32) b += p.node_offsets[i + 1] <= t;
    b = __reduce_add_sync(0xffffffffu, b);
    int base = 0, n = 0, fault = b >= p.B ? SPECA_STATUS_BAD_OFFSETS : sequence_nodes(p, b, base, n);
    if (!fault && t < base) fault = SPECA_STATUS_BAD_OFFSETS;
    const int page = 1 << p.page_shift;
    const int32_t *table = nullptr;
    int len = 0;
    if (!fault) {
        table = p.page_table + size_t(b) * p.max_pages;
        len = p.kv_len[b];
        int bad = len < 0 || len > (p.max_pages << p.page_shift);
        if (!bad)
            for (int i = lane; i < (len + page - 1) >> p.page_shift; i += 32) bad |= table[i] < 0 || table[i] >= p.n_pages;
        if (__any_sync(0xffffffffu, bad)) fault |= SPECA_STATUS_BAD_PAGE;
        bad = 0;
        if (p.parent != nullptr)
            for (int i = lane; i < n; i += 32) bad |= p.parent[base + i] < -1 || p.parent[base + i] >= i;
        if (__any_sync(0xffffffffu, bad)) fault |= SPECA_STATUS_BAD_PARENT;
    }
    if (fault) {
        if (lane == 0 && l == 0 && h == 0) atomicOr(p.status, fault);
        return;
    }
    float q[E], o[E], m = -INFINITY, sum = 0.f;
    const size_t row = (size_t(l) * p.T + t) * p.H + h;
    for (int i = 0; i < E; ++i) { q[i] = __bfloat162float(p.q[row * D + lane + 32 * i]) * p.scale; o[i] = 0.f; }
    auto take = [&](const __nv_bfloat16 *k, const __nv_bfloat16 *v) {
        float s = 0.f;
        for (int i = 0; i < E; ++i) s = fmaf(q[i], __bfloat162float(k[lane + 32 * i]), s);
        for (int w = 16; w > 0; w /= 2) s += __shfl_xor_sync(0xffffffffu, s, w);
        const float top = fmaxf(m, s), old = m == top ? 1.f : expf(m - top), e = expf(s - top);
        sum = sum * old + e;
        for (int i = 0; i < E; ++i) o[i] = o[i] * old + e * __bfloat162float(v[lane + 32 * i]);
        m = top;
    };
    for (int j = 0; j < len; ++j) {
        const size_t at = (((size_t(l) * p.n_pages + table[j >> p.page_shift]) * p.HK + hk) << p.page_shift) + (j & (page - 1));
        take(p.k_cache + at * D, p.v_cache + at * D);
    }
    for (int a = t - base; a >= 0; a = p.parent != nullptr ? p.parent[base + a] : a - 1) {
        const size_t at = (size_t(l) * p.T + base + a) * p.HK + hk;
        take(p.k + at * D, p.v + at * D);
    }
    for (int i = 0; i < E; ++i) p.o[row * D + lane + 32 * i] = __float2bfloat16_rn(o[i] / sum);
}

}  // namespace

size_t attend_workspace_bytes(const speca_attn_dims *d)
{
    (void)d;
    return 16;
}

int launch_attend(const AttnParams &p, int d_head, cudaStream_t st)
{
    const long blocks = (long(p.L) * p.T * p.H + kWarps - 1) / kWarps;
    if (blocks > 0x7fffffffL) return int(cudaErrorInvalidConfiguration);
    if (d_head == 64) launch(attend_kernel<64>, unsigned(blocks), kWarps * 32, 0, st, p);
    else if (d_head == 128) launch(attend_kernel<128>, unsigned(blocks), kWarps * 32, 0, st, p);
    else launch(attend_kernel<256>, unsigned(blocks), kWarps * 32, 0, st, p);
    return int(cudaGetLastError());
}

}  // namespace speca
