// Attention layers, everything but the attention: norm and rotation of queries and keys, commit of accepted records to
// the paged cache, copies of pages.  All three move bytes and compute next to nothing.
#include "attn.cuh"

namespace speca {
namespace {

// ---------------------------------------------------------------------------------------------------------------
// Norm and rotation.  A warp takes a share of one token's head rows over all layers: a lane has 8 consecutive elements (16
// bytes) of a row, D / 8 lanes a row, so its angles are the same for every row of the token and are formed once.
// ---------------------------------------------------------------------------------------------------------------
constexpr int kNormWarps = 8;

__device__ __forceinline__ void unpack8(const uint4 &x, float (&f)[8])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sequence of packed node t, whole warp: the number of sequences that end at or before it (B if there is none).
__device__ __forceinline__ int sequence_of(const int32_t *node_offsets, int B, int t, int lane)
{
    int before = 0;
    for (int b = lane; b < B; b += 32) before += node_offsets[b + 1] <= t;
    return __reduce_add_sync(0xffffffffu, before);
}

template <int D>
__global__ void __launch_bounds__(kNormWarps * 32)
norm_rope_kernel(AttnParams p, NormParams np, int32_t parts)
{
    after_previous_kernel();
    constexpr int LPH = D / 8, HPW = 32 / LPH;             // lanes of a row, rows a warp has at a time
    const int lane = threadIdx.x & 31;
    const long task = long(blockIdx.x) * kNormWarps + (threadIdx.x >> 5);
    const int t = int(task / parts), part = int(task % parts);
    if (t >= p.T) return;
    const int b = sequence_of(p.node_offsets, p.B, t, lane);
    int base, n, fault = 0;
    if (b >= p.B) fault = SPECA_STATUS_BAD_OFFSETS;        // behind the last sequence
    else fault = sequence_nodes(p, b, base, n);
    if (!fault && t < base) fault = SPECA_STATUS_BAD_OFFSETS;
    int depth = 0, len = 0;
    if (!fault) {
        len = p.kv_len[b];
        if (len < 0) fault = SPECA_STATUS_BAD_PAGE;
        if (p.parent == nullptr) depth = t - base + 1;
        else {
            int bad = 0;
            for (int i = lane; i < n; i += 32) {
                const int up = p.parent[base + i];
                bad |= up < -1 || up >= i;
            }
            if (__any_sync(0xffffffffu, bad)) fault |= SPECA_STATUS_BAD_PARENT;
            else
                for (int a = t - base; a >= 0; a = p.parent[base + a]) ++depth;
        }
    }
    if (fault) {
        if (lane == 0 && part == 0) atomicOr(p.status, fault);
        return;
    }

    // this lane's 8 elements of a row, and for each the element it is rotated with
    const int e0 = (lane % LPH) * 8, half = np.rot / 2;
    const bool turned = e0 < np.rot;
    int mate = lane;                                        // lane that has the other elements of the pairs (itself: interleaved)
    if (turned && !np.interleaved) mate = e0 < half ? lane + half / 8 : lane - half / 8;
    float c[8], s[8];                                       // element <- element * c + partner * s
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
    if (turned) {
        const double pos = double(len) + double(depth - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = e0 + i;
            const int j = np.interleaved ? e / 2 : (e < half ? e : e - half);
            const bool first = np.interleaved ? (e & 1) == 0 : e < half;
            // the angle in turns, whole ones taken off in 64 bits: far positions leave fp32 no digits behind the point
            const double turns = pos * double(np.inv_freq[j]) * 0.15915494309189533577;
            float sn, cs;
            sincospif(2.f * float(turns - rint(turns)), &sn, &cs);
            c[i] = cs * np.rope_scale;
            s[i] = (first ? -sn : sn) * np.rope_scale;
        }
    }

    const int rows = p.H + p.HK, steps = (rows + HPW - 1) / HPW;
    const long total = long(p.L) * steps, per = (total + parts - 1) / parts;
    const long end = min(total, (part + 1) * per);
    for (long it = part * per; it < end; ++it) {
        const int l = int(it / steps), r = int(it % steps) * HPW + lane / LPH;
        const bool on = r < rows, is_q = r < p.H;
        const int h = is_q ? r : r - p.H;
        uint4 raw = make_uint4(0u, 0u, 0u, 0u);
        if (on) {
            const __nv_bfloat16 *row = is_q ? p.q + l * np.q_layer + t * np.q_token : p.k + l * np.k_layer + t * np.k_token;
            raw = *reinterpret_cast<const uint4 *>(row + h * D + e0);
        }
        float x[8], y[8];
        unpack8(raw, x);
        const float *w = is_q ? np.q_weight : np.k_weight;
        float rs = 1.f;
        if (np.q_weight != nullptr || np.k_weight != nullptr) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
            for (int m = LPH / 2; m > 0; m /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            if (w != nullptr) rs = rsqrtf(sum * (1.f / D) + np.eps);
        }
        if (w != nullptr && on) {
            const float4 *w4 = reinterpret_cast<const float4 *>(w + size_t(l) * D + e0);
            const float4 a = w4[0], d = w4[1];
            const float ww[8] = {a.x, a.y, a.z, a.w, d.x, d.y, d.z, d.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * rs * ww[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl_sync(0xffffffffu, x[i], mate);
            y[i] = np.interleaved ? x[i ^ 1] : other;
        }
        if (turned)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i] + y[i] * s[i];
        if (on) {
            __nv_bfloat16 *out = is_q ? np.q_out + (size_t(l) * p.T + t) * p.H * D : np.k_out + (size_t(l) * p.T + t) * p.HK * D;
            *reinterpret_cast<uint4 *>(out + size_t(h) * D + e0) = pack8(x);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Commit of records to the cache: a CTA takes a share of what one sequence appends to one layer, 16 bytes a thread at a
// time.  Rows of the records are [token][head], rows of the cache [page][head][row].
// ---------------------------------------------------------------------------------------------------------------
constexpr int kCommitThreads = 256;

__global__ void __launch_bounds__(kCommitThreads)
commit_kv_kernel(AttnParams p, int32_t vec, int32_t parts, int32_t *kv_len_out)
{
    after_previous_kernel();
    __shared__ int32_t node[16];
    const int part = blockIdx.x % parts, b = blockIdx.x / parts % p.B, l = blockIdx.x / parts / p.B, tid = threadIdx.x;
    const int len = p.kv_len[b];
    int base, n, A, fault = 0;
    if (p.path_idx != nullptr) {
        A = p.path_len[b];
        base = p.node_offsets[b];
        const int end = p.node_offsets[b + 1];
        n = end - base;
        if (A < 0 || A > p.max_depth) fault = SPECA_STATUS_TOO_DEEP;
        else if (A > 0 && (base < 0 || end < base || end > p.T)) fault = SPECA_STATUS_BAD_OFFSETS;
        else if (tid < A) {
            const int e = p.path_idx[size_t(b) * p.max_depth + tid];
            node[tid] = e;
            if (e < 0 || e >= n) fault = SPECA_STATUS_BAD_PATH;
            else if (p.parent != nullptr &&
                     p.parent[base + e] != (tid == 0 ? -1 : p.path_idx[size_t(b) * p.max_depth + tid - 1]))
                fault = SPECA_STATUS_BAD_PATH;
        }
    } else {
        fault = sequence_nodes(p, b, base, n);
        A = n;
    }
    const int page = 1 << p.page_shift;
    const int32_t *table = p.page_table + size_t(b) * p.max_pages;
    if (!fault && (len < 0 || (A > 0 && 1LL * len + A > 1LL * p.max_pages * page))) fault = SPECA_STATUS_BAD_PAGE;
    if (!fault && A > 0)
        for (int i = (len >> p.page_shift) + tid; i <= (len + A - 1) >> p.page_shift; i += kCommitThreads)
            if (table[i] < 0 || table[i] >= p.n_pages) fault = SPECA_STATUS_BAD_PAGE;
    const bool lead = l == 0 && part == 0;
    if (fault && lead) atomicOr(p.status, fault);
    if (__syncthreads_or(fault)) {
        if (lead && tid == 0 && kv_len_out != nullptr) kv_len_out[b] = len;
        return;
    }
    if (lead && tid == 0 && kv_len_out != nullptr) kv_len_out[b] = len + A;
    const int row = p.HK * vec, page_vec = page * vec;       // 16-byte pieces of a token's row, of a page of one head
    const long total = long(A) * row;
    const uint4 *ks = reinterpret_cast<const uint4 *>(p.k), *vs = reinterpret_cast<const uint4 *>(p.v);
    uint4 *kc = reinterpret_cast<uint4 *>(p.k_cache), *vc = reinterpret_cast<uint4 *>(p.v_cache);
    for (long i = long(part) * kCommitThreads + tid; i < total; i += long(parts) * kCommitThreads) {
        const int a = int(i / row), r = int(i % row), h = r / vec, e = r % vec;
        const int from = base + (p.path_idx != nullptr ? node[a] : a), at = len + a;
        const size_t src = (size_t(l) * p.T + from) * row + r;
        const size_t dst = ((size_t(l) * p.n_pages + table[at >> p.page_shift]) * p.HK + h) * page_vec + size_t(at & (page - 1)) * vec + e;
        const uint4 x = ks[src], y = vs[src];
        kc[dst] = x;
        vc[dst] = y;
    }
}

// New lengths where they replace the old ones: the kernel above reads those in every CTA, so they change behind it.
__global__ void __launch_bounds__(256) grow_kernel(AttnParams p, int32_t *kv_len)
{
    after_previous_kernel();
    const int b = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (b >= p.B) return;
    const int len = kv_len[b], page = 1 << p.page_shift;
    int base, n, A, bad = 0;
    if (p.path_idx != nullptr) {
        A = p.path_len[b];
        base = p.node_offsets[b];
        const int end = p.node_offsets[b + 1];
        n = end - base;
        bad = A < 0 || A > p.max_depth || (A > 0 && (base < 0 || end < base || end > p.T));
        if (!bad && lane < A) {
            const int e = p.path_idx[size_t(b) * p.max_depth + lane];
            bad = e < 0 || e >= n;
            if (!bad && p.parent != nullptr)
                bad = p.parent[base + e] != (lane == 0 ? -1 : p.path_idx[size_t(b) * p.max_depth + lane - 1]);
        }
    } else {
        bad = sequence_nodes(p, b, base, n) != 0;
        A = n;
    }
    if (!bad && (len < 0 || (A > 0 && 1LL * len + A > 1LL * p.max_pages * page))) bad = 1;
    if (!bad && A > 0)
        for (int i = (len >> p.page_shift) + lane; i <= (len + A - 1) >> p.page_shift; i += 32) {
            const int id = p.page_table[size_t(b) * p.max_pages + i];
            bad |= id < 0 || id >= p.n_pages;
        }
    if (!__any_sync(0xffffffffu, bad) && lane == 0) kv_len[b] = len + A;
}

// ---------------------------------------------------------------------------------------------------------------
// Copies of pages: a CTA has a share of one page of one layer, keys and values.  Every CTA looks its pair up among all
// others, so that what is copied does not depend on the order in which CTAs run.
// ---------------------------------------------------------------------------------------------------------------
constexpr int kCopyThreads = 256, kCopyPieces = 8;           // 16-byte pieces of keys and of values a thread moves

__global__ void __launch_bounds__(kCopyThreads)
copy_pages_kernel(AttnParams p, int32_t page_vec, int32_t parts, int32_t n, const int32_t *src, const int32_t *dst)
{
    after_previous_kernel();
    const int part = blockIdx.x % parts, j = blockIdx.x / parts % n, l = blockIdx.x / parts / n, tid = threadIdx.x;
    const int from = src[j], to = dst[j];
    int bad = from < 0 || from >= p.n_pages || to < 0 || to >= p.n_pages;
    for (int i = tid; i < n; i += kCopyThreads) bad |= (i != j && dst[i] == to) || src[i] == to;
    if (__syncthreads_or(bad)) {
        if (tid == 0 && l == 0 && part == 0) atomicOr(p.status, SPECA_STATUS_BAD_PAGE);
        return;
    }
    const size_t a = (size_t(l) * p.n_pages + from) * page_vec, c = (size_t(l) * p.n_pages + to) * page_vec;
    uint4 *kc = reinterpret_cast<uint4 *>(p.k_cache), *vc = reinterpret_cast<uint4 *>(p.v_cache);
    const int first = part * (kCopyThreads * kCopyPieces) + tid;
    uint4 x[kCopyPieces], y[kCopyPieces];
#pragma unroll
    for (int i = 0; i < kCopyPieces; ++i)
        if (first + i * kCopyThreads < page_vec) {
            x[i] = kc[a + first + i * kCopyThreads];
            y[i] = vc[a + first + i * kCopyThreads];
        }
#pragma unroll
    for (int i = 0; i < kCopyPieces; ++i)
        if (first + i * kCopyThreads < page_vec) {
            kc[c + first + i * kCopyThreads] = x[i];
            vc[c + first + i * kCopyThreads] = y[i];
        }
}

inline int grid_of(long blocks, unsigned &grid)
{
    grid = unsigned(blocks);
    return blocks < 1 || blocks > 0x7fffffffL ? int(cudaErrorInvalidConfiguration) : 0;
}

}  // namespace

int launch_norm_rope(const AttnParams &p, const NormParams &n, int d_head, cudaStream_t st)
{
    const long sms = sm_count_of_current_device();
    if (sms <= 0) return int(cudaErrorInvalidDevice);
    const long steps = long(p.L) * ((p.H + p.HK) * (d_head / 8) + 31) / 32, most = sms * 64;
    long parts = p.T >= most ? 1 : most / p.T;
    if (parts > steps) parts = steps;
    unsigned grid;
    const int rc = grid_of((p.T * parts + kNormWarps - 1) / kNormWarps, grid);
    if (rc != 0) return rc;
    if (d_head == 64) launch(norm_rope_kernel<64>, grid, kNormWarps * 32, 0, st, p, n, int(parts));
    else if (d_head == 128) launch(norm_rope_kernel<128>, grid, kNormWarps * 32, 0, st, p, n, int(parts));
    else launch(norm_rope_kernel<256>, grid, kNormWarps * 32, 0, st, p, n, int(parts));
    return int(cudaGetLastError());
}

int launch_commit_kv(const AttnParams &p, int d_head, int32_t *kv_len_out, cudaStream_t st)
{
    const int vec = d_head / 8;
    const long most = long(p.path_idx != nullptr ? p.max_depth : p.max_nodes) * p.HK * vec;
    long parts = (most + kCommitThreads * 4 - 1) / (kCommitThreads * 4);
    const bool in_place = kv_len_out == p.kv_len;
    unsigned grid;
    const int rc = grid_of(parts * p.B * p.L, grid);
    if (rc != 0) return rc;
    launch(commit_kv_kernel, grid, kCommitThreads, 0, st, p, vec, int(parts), in_place ? nullptr : kv_len_out);
    const int e = int(cudaGetLastError());
    if (e != 0 || !in_place) return e;
    launch(grow_kernel, (p.B + 7) / 8, 256, 0, st, p, kv_len_out);
    return int(cudaGetLastError());
}

int launch_copy_pages(const AttnParams &p, int d_head, const int32_t *src, const int32_t *dst, int32_t n, cudaStream_t st)
{
    const int page_vec = (p.HK << p.page_shift) * (d_head / 8);
    const long parts = (long(page_vec) + kCopyThreads * kCopyPieces - 1) / (kCopyThreads * kCopyPieces);
    unsigned grid;
    const int rc = grid_of(parts * n * p.L, grid);
    if (rc != 0) return rc;
    launch(copy_pages_kernel, grid, kCopyThreads, 0, st, p, page_vec, int(parts), n, src, dst);
    return int(cudaGetLastError());
}

}  // namespace speca
