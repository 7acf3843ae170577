// Attention layers, everything but the attention: norm and rotation of queries and keys, commit of accepted records to
// the paged cache, copies of pages.  All three move bytes and compute next to nothing.
#include "attn.cuh"

namespace speca {
namespace {

// ---------------------------------------------------------------------------------------------------------------
// Norm and rotation.  A warp takes a share of one token's head rows over all layers.  D / 8 lanes have a row, and a lane has both
// elements of four pairs (lanes beyond the rotated part: eight plain elements), so no element travels between lanes but for
// the sum of squares, and its four angles are the same for every row of the token: they are formed once.  Weights, cosines and
// sines of a layer's queries (or keys) are multiplied out beforehand, which leaves a product, a fused multiply-add and the scale
// by the norm for each pair of elements.  The rows of the next step are asked for before this one's are worked on.
// ---------------------------------------------------------------------------------------------------------------
// rows a lane has in flight: 5632 tokens in 12 layers 243 us with 2, 215 with 4, 281 with 8 (spilled), on one GPU; others take up to 10 % more
constexpr int kNormWarps = 4, kNormRows = 4;
constexpr int kNormBlocks = 5;                              // an SM: up to 102 registers (94 with the bound, 92 without it: same times)

// two fp32 values in a pair of registers, one instruction for both
__device__ __forceinline__ uint64_t pair2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair2(uint64_t x, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack2(uint64_t x)
{
    float lo, hi;
    unpair2(x, lo, hi);
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Sequence of packed node t, whole warp: the number of sequences that end at or before it (B if there is none).
__device__ __forceinline__ int sequence_of(const int32_t *node_offsets, int B, int t, int lane)
{
    int before = 0;
    for (int b = lane; b < B; b += 32) before += node_offsets[b + 1] <= t;
    return __reduce_add_sync(0xffffffffu, before);
}

template <int D, bool INTER>
__global__ void __launch_bounds__(kNormWarps * 32, kNormBlocks)
norm_rope_kernel(AttnParams p, NormParams np, int32_t parts)
{
    after_previous_kernel();
    constexpr int LPH = D / 8, HPW = 32 / LPH, U = kNormRows;      // lanes of a row, rows a warp has side by side
    const int lane = threadIdx.x & 31, sub = lane / LPH, in = lane % LPH;
    const long task = long(blockIdx.x) * kNormWarps + (threadIdx.x >> 5);
    const int t = int(task / parts), part = int(task % parts);
    if (t >= p.T) return;
    // this lane's elements of a row: ea .. ea + 3 and eb .. eb + 3
    const int half = np.rot / 2;
    const bool turned = 8 * in < np.rot;
    const int ea = !INTER && turned ? 4 * in : 8 * in, eb = !INTER && turned ? half + 4 * in : 8 * in + 4;

    const int steps_q = (p.H + HPW - 1) / HPW, steps = steps_q + (p.HK + HPW - 1) / HPW;
    const long total = long(p.L) * steps, per = (total + parts - 1) / parts;
    long it = part * per;
    const long end = min(total, it + per);
    int l = int(it / steps), s = int(it % steps);
    // up to U steps from (l, s) on, of the queries or of the keys of one layer
    auto width = [&](long it, int s) { return int(min(long(min(U, (s < steps_q ? steps_q : steps) - s)), end - it)); };
    auto ask = [&](int l, int s, int m, uint2 (&a)[U], uint2 (&b)[U]) {
        const bool is_q = s < steps_q;
        const __nv_bfloat16 *row = is_q ? p.q + l * np.q_layer + t * np.q_token : p.k + l * np.k_layer + t * np.k_token;
        const int h0 = (is_q ? s : s - steps_q) * HPW + sub, heads = is_q ? p.H : p.HK;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < m && h0 + u * HPW < heads) {
                a[u] = *reinterpret_cast<const uint2 *>(row + (h0 + u * HPW) * D + ea);
                b[u] = *reinterpret_cast<const uint2 *>(row + (h0 + u * HPW) * D + eb);
            } else a[u] = b[u] = make_uint2(0u, 0u);
    };
    uint2 a[U], b[U];
    int m = width(it, s);
    if (it < end) ask(l, s, m, a, b);

    const int seq = sequence_of(p.node_offsets, p.B, t, lane);
    int base, n, fault = 0;
    if (seq >= p.B) fault = SPECA_STATUS_BAD_OFFSETS;      // behind the last sequence
    else fault = sequence_nodes(p, seq, base, n);
    if (!fault && t < base) fault = SPECA_STATUS_BAD_OFFSETS;
    int depth = 0, len = 0;
    if (!fault) {
        len = p.kv_len[seq];
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
                for (int x = t - base; x >= 0; x = p.parent[base + x]) ++depth;
        }
    }
    if (fault) {
        if (lane == 0 && part == 0) atomicOr(p.status, fault);
        return;
    }
    float cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
    if (turned) {
        const double pos = double(len) + double(depth - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // the angle in turns, whole ones taken off in 64 bits: far positions leave fp32 no digits behind the point
            const double turns = pos * double(np.inv_freq[4 * in + i]) * 0.15915494309189533577;
            sincospif(2.f * float(turns - rint(turns)), &sn[i], &cs[i]);
            cs[i] *= np.rope_scale;
            sn[i] *= np.rope_scale;
        }
    }

    // element <- element * own + mate * other, before the norm's scale; in pairs as below
    uint64_t own[4], other[4];
    int made = -1;                                          // 2 * layer + (keys) that they are for
    while (it < end) {
        const bool is_q = s < steps_q;
        // what comes after this step
        const long it2 = it + m;
        const int s2 = s + m == steps ? 0 : s + m, l2 = s + m == steps ? l + 1 : l, m2 = it2 < end ? width(it2, s2) : 0;
        uint2 a2[U], b2[U];
        if (m2 > 0) ask(l2, s2, m2, a2, b2);
        const float *w = is_q ? np.q_weight : np.k_weight;
        if (made != 2 * l + !is_q) {
            made = 2 * l + !is_q;
            float4 wa = make_float4(1.f, 1.f, 1.f, 1.f), wb = wa;
            if (w != nullptr) {
                wa = *reinterpret_cast<const float4 *>(w + size_t(l) * D + ea);
                wb = *reinterpret_cast<const float4 *>(w + size_t(l) * D + eb);
            }
            const float x[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // elements 2 i and 2 i + 1; of the half layout those of the second half (i >= 2) turn the other way
                const int e = 2 * i;
                if (INTER) {
                    own[i] = pair2(x[e] * cs[i], x[e + 1] * cs[i]);
                    other[i] = pair2(-x[e + 1] * sn[i], x[e] * sn[i]);
                } else {
                    const int f = e & 3, m = e ^ 4;
                    const float s0 = i < 2 ? -sn[f] : sn[f], s1 = i < 2 ? -sn[f + 1] : sn[f + 1];
                    own[i] = pair2(x[e] * cs[f], x[e + 1] * cs[f + 1]);
                    other[i] = pair2(x[m] * s0, x[m + 1] * s1);
                }
            }
        }
        const int h0 = (is_q ? s : s - steps_q) * HPW + sub, heads = is_q ? p.H : p.HK;
        __nv_bfloat16 *out = (is_q ? np.q_out : np.k_out) + (size_t(l) * p.T + t) * heads * D;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < m) {
                // pairs of elements: (0, 1) and (2, 3) of each half, so that one instruction works on two
                const uint32_t raw[4] = {a[u].x, a[u].y, b[u].x, b[u].y};
                uint64_t x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = pair2(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xffff0000u));
                float rs = 1.f;
                if (w != nullptr) {
                    uint64_t sq = mul2(x[0], x[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i) sq = fma2(x[i], x[i], sq);
                    float lo, hi;
                    unpair2(sq, lo, hi);
                    float sum = lo + hi;
#pragma unroll
                    for (int j = LPH / 2; j > 0; j /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, j);
                    rs = rsqrtf(sum * (1.f / D) + np.eps);
                }
                const uint64_t rs2 = pair2(rs, rs);
                uint64_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // what each element is rotated with: the same place of the other half, or its neighbour
                    uint64_t mate = x[i ^ 2];
                    if (INTER) {
                        float lo, hi;
                        unpair2(x[i], lo, hi);
                        mate = pair2(hi, lo);
                    }
                    // (a plain element takes nothing from another, not even what is not finite)
                    y[i] = mul2(x[i], own[i]);
                    if (turned) y[i] = fma2(mate, other[i], y[i]);
                    y[i] = mul2(y[i], rs2);
                }
                if (h0 + u * HPW < heads) {
                    __nv_bfloat16 *to = out + size_t(h0 + u * HPW) * D;
                    *reinterpret_cast<uint2 *>(to + ea) = make_uint2(pack2(y[0]), pack2(y[1]));
                    *reinterpret_cast<uint2 *>(to + eb) = make_uint2(pack2(y[2]), pack2(y[3]));
                }
            }
        it = it2; s = s2; l = l2; m = m2;
#pragma unroll
        for (int u = 0; u < U; ++u) { a[u] = a2[u]; b[u] = b2[u]; }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Commit of records to the cache: a CTA takes a share of what one sequence appends to one layer, 16 bytes a thread at a
// time.  Rows of the records are [token][head], rows of the cache [page][head][row].  Accepted paths of 128 trees in 12 layers take
// 8.4 to 9 us where the launch is 3.7 and the bytes 3.9: 1536 CTAs of which four fit an SM, 2.6 waves of path -> page -> record.
// ---------------------------------------------------------------------------------------------------------------
constexpr int kCommitThreads = 256, kCommitPieces = 4;       // 16-byte pieces of keys and of values a thread has in flight

__global__ void __launch_bounds__(kCommitThreads)
commit_kv_kernel(AttnParams p, int32_t vec, int32_t parts, int32_t *kv_len_out)
{
    after_previous_kernel();
    const int part = blockIdx.x % parts, b = blockIdx.x / parts % p.B, l = blockIdx.x / parts / p.B, tid = threadIdx.x;
    const bool path = p.path_idx != nullptr;
    const int32_t *entry = p.path_idx + size_t(b) * p.max_depth, *table = p.page_table + size_t(b) * p.max_pages;
    const int len = p.kv_len[b], base = p.node_offsets[b], stop = p.node_offsets[b + 1];
    const int mine = path && tid < p.max_depth ? entry[tid] : 0, above = path && tid > 0 && tid < p.max_depth ? entry[tid - 1] : -1;
    int n = stop - base, A = n, fault = 0;
    if (path) {
        A = p.path_len[b];
        if (A < 0 || A > p.max_depth) fault = SPECA_STATUS_TOO_DEEP;
        else if (A > 0 && (base < 0 || stop < base || stop > p.T)) fault = SPECA_STATUS_BAD_OFFSETS;
    } else {
        int b0, n0;
        fault = sequence_nodes(p, b, b0, n0);
    }
    const int page = 1 << p.page_shift;
    if (!fault && (len < 0 || (A > 0 && 1LL * len + A > 1LL * p.max_pages * page))) fault = SPECA_STATUS_BAD_PAGE;
    const long total = fault ? 0 : long(A) * p.HK * vec;

    // The first pieces are read while the path and the pages are still being checked, each by the thread that has it: what an
    // index out of range would name is not.
    const uint32_t row = uint32_t(p.HK) * vec;               // pieces of a token's row
    const uint4 *ks = reinterpret_cast<const uint4 *>(p.k), *vs = reinterpret_cast<const uint4 *>(p.v);
    uint4 *kc = reinterpret_cast<uint4 *>(p.k_cache), *vc = reinterpret_cast<uint4 *>(p.v_cache);
    uint4 x[kCommitPieces], y[kCommitPieces];
    size_t to[kCommitPieces];
    auto fetch = [&](long first) {
#pragma unroll
        for (int j = 0; j < kCommitPieces; ++j) {
            const long i = first + j * kCommitThreads;
            to[j] = ~size_t(0);
            if (i >= total) continue;
            const int a = int(uint32_t(i) / row), at = len + a;                 // (less than 2^31 pieces: 8192 rows of 2^17 at most)
            const uint32_t r = uint32_t(i) - a * row, h = r / vec, e = r - h * vec;
            const int from = path ? entry[a] : a, id = table[at >> p.page_shift];
            if (from < 0 || from >= n || id < 0 || id >= p.n_pages) continue;
            const size_t src = (size_t(l) * p.T + base + from) * row + r;
            to[j] = ((((size_t(l) * p.n_pages + id) * p.HK + h) << p.page_shift) + (at & (page - 1))) * vec + e;
            x[j] = ks[src];
            y[j] = vs[src];
        }
    };
    auto put = [&]() {
#pragma unroll
        for (int j = 0; j < kCommitPieces; ++j)
            if (to[j] != ~size_t(0)) {
                kc[to[j]] = x[j];
                vc[to[j]] = y[j];
            }
    };
    const long first = long(part) * (kCommitThreads * kCommitPieces) + tid, stride = long(parts) * (kCommitThreads * kCommitPieces);
    fetch(first);
    if (!fault && A > 0) {
        if (path && tid < A) {
            if (mine < 0 || mine >= n) fault = SPECA_STATUS_BAD_PATH;
            else if (p.parent != nullptr && p.parent[base + mine] != (tid == 0 ? -1 : above)) fault = SPECA_STATUS_BAD_PATH;
        }
        for (int i = (len >> p.page_shift) + tid; i <= (len + A - 1) >> p.page_shift; i += kCommitThreads)
            if (table[i] < 0 || table[i] >= p.n_pages) fault = SPECA_STATUS_BAD_PAGE;
    }
    const bool lead = l == 0 && part == 0;
    if (fault && lead) atomicOr(p.status, fault);
    const bool skip = __syncthreads_or(fault);
    if (lead && tid == 0 && kv_len_out != nullptr) kv_len_out[b] = skip ? len : len + A;
    if (skip) return;
    put();
    for (long i = first + stride; i - tid < total; i += stride) {
        fetch(i);
        put();
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
// others, so that what is copied does not depend on the order in which CTAs run.  That is the square of the number of pairs:
// pages of 64 KB in one layer 5.8 TB/s with 1024 pairs, 6.1 with 4096, 2.6 with 16384, 0.45 with 65536.
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
    const int hpw = 256 / d_head;
    const long steps = long(p.L) * ((p.H + hpw - 1) / hpw + (p.HK + hpw - 1) / hpw);
    // A token's rows stay with one warp, which then forms its angles once, as long as that makes enough warps to fill the
    // machine (8192 tokens of one layer 36.6 us, spread over three times as many warps 41.8); fewer tokens are spread over as
    // many warps as they have steps.
    const long most = sms * kNormWarps * kNormBlocks;
    long parts = p.T >= most ? 1 : (most + p.T - 1) / p.T;
    if (parts > steps) parts = steps;
    unsigned grid;
    const int rc = grid_of((p.T * parts + kNormWarps - 1) / kNormWarps, grid);
    if (rc != 0) return rc;
    auto go = [&](auto kernel) { launch(kernel, grid, kNormWarps * 32, 0, st, p, n, int(parts)); };
    if (n.interleaved) go(d_head == 64 ? norm_rope_kernel<64, true> : d_head == 128 ? norm_rope_kernel<128, true> : norm_rope_kernel<256, true>);
    else go(d_head == 64 ? norm_rope_kernel<64, false> : d_head == 128 ? norm_rope_kernel<128, false> : norm_rope_kernel<256, false>);
    return int(cudaGetLastError());
}

int launch_commit_kv(const AttnParams &p, int d_head, int32_t *kv_len_out, cudaStream_t st)
{
    const int vec = d_head / 8;
    const long most = long(p.path_idx != nullptr ? p.max_depth : p.max_nodes) * p.HK * vec;
    long parts = (most + kCommitThreads * kCommitPieces - 1) / (kCommitThreads * kCommitPieces);
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
