// Verification by an attention layer where a key head has few rows: single tokens, short chains, small trees.
//
// The 128-row products of the other kernel would be padding for the most part; it is fast enough for the bytes all the same,
// but 64 single tokens over long contexts then run into the power limit (1000 W, 1.55 GHz; 420 to 437 us against 360 here) and a
// single chain waits for TMEM, products and softmax in turn (16.8 us against 12.7).  Weights are rounded to bf16 as there.  Here eight warps share a tile: each has the 16 rows, an
// eighth of the tile's keys and all columns of O (D <= 128; a quarter and half of them at 256), with a maximum and sums of its own, and warp-level products (m16n8k16) whose
// operands come out of the same swizzled tiles by ldmatrix.  S stays in registers, where it becomes P.  Nothing is exchanged
// before a unit's end, where 64 columns of all warps fit into shared memory together (32 columns at a time the end took four
// more barriers and half as long again).  A warp has 128 columns: with 64, every score is formed by twice as many warps, and 64
// single tokens over long contexts took a tenth longer (398 us against 363 on one GPU).
#include "attend_common.cuh"

namespace speca {

using namespace attend;

namespace {

constexpr int kConsumers = 8;            // warps that compute; then keys, schedule, values
constexpr int kRows = 16;
constexpr float kSlack = 8.f;            // binary digits a maximum may grow by before O is scaled

// A warp has KW of the tile's N keys and OC columns.
template <int DH> struct Few {
    static constexpr int D = DH;
    static constexpr int N = D == 256 ? 64 : 128;
    static constexpr int MT = kRows, kEnds = 3, kPiece = 1, kWhole = kFewWhole;
    static constexpr bool kMend = false;
    static constexpr int THREADS = (kConsumers + 3) * 32;
    static constexpr int OC = D < 128 ? D : 128, CH = D / OC;
    static constexpr int KB = kConsumers / CH, KW = N / KB;
    static constexpr int TILE = N * D * 2;
    static constexpr int KS = D == 64 ? 6 : 3, VS = KS;
    static constexpr int OffRing = 0;
    static constexpr int OffQ = (KS + VS) * TILE;            // queries; at a unit's end the warps' sums, float [warp][row][64]
    static constexpr int OffPar = OffQ + kConsumers * kRows * 64 * 4;        // int16 parent[kRows]
    static constexpr int OffMl = OffPar + 128;               // float2 [warp][row]
    static constexpr int OffRec = OffMl + kConsumers * kRows * 8;
    static constexpr int OffBars = OffRec + 64 * kRecords;
    static constexpr int kKFull = 0, kKEmpty = KS, kVFull = 2 * KS, kVEmpty = kVFull + VS, kVRaw = 0, kRecFull = kVEmpty + VS,
                         kRecEmpty = kRecFull + kRecords, kBars = kRecEmpty + kRecords;
    static constexpr int OffMisc = OffBars + 8 * kBars;
    static constexpr int OffFlags = OffMisc + 64;
    static constexpr int Bytes = OffFlags + 8 * kFlagRing;
    static_assert(KW % 16 == 0 && KB * KW == N && OffQ % 1024 == 0 && kRows * D * 2 <= kConsumers * kRows * 64 * 4 && Bytes <= 232448, "layout");
};
// four sums of a row, spread over the banks
__device__ __forceinline__ int stage_offset(int warp, int row, int col) { return (warp * kRows + row) * 64 + (col ^ ((row & 7) << 3)); }

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&x)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&x)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16_sync(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the pair without what is not finite in it; whether there was any
__device__ __forceinline__ bool strip(uint32_t &pair)
{
    const bool lo = (pair & 0x7f80u) == 0x7f80u, hi = (pair & 0x7f800000u) == 0x7f800000u;
    if (lo) pair &= 0xffff0000u;
    if (hi) pair &= 0x0000ffffu;
    return lo || hi;
}

template <int D>
__global__ void __launch_bounds__(Few<D>::THREADS, 1)
attend_few_kernel(const __grid_constant__ Maps maps, AttnParams p, Plan plan, int32_t box_rows)
{
    after_previous_kernel();
    using C = Few<D>;
    constexpr int KB = C::KB, KW = C::KW, OC = C::OC, KS = C::KS, VS = C::VS;
    extern __shared__ __align__(1024) uint8_t smem[];
    Cta<C> x(p, plan, smem);
    if ((x.sbase & 1023u) != 0u || p.misplaced) {            // never expected; refuse to run rather than corrupt
        x.refuse();
        return;
    }
    const int warp = x.warp, lane = x.lane, cta = blockIdx.x;
    const Group group = x.group;
    if (warp == 0) {
        x.init(kConsumers + 2, kConsumers);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    x.begin();

    if (warp == kConsumers) x.template load<0>(maps, box_rows);
    else if (warp == kConsumers + 2) x.template load<1>(maps, box_rows);
    else if (warp == kConsumers + 1) x.schedule();
    else {
        const int kb = warp % KB, ch = warp / KB;
        const int k0 = kb * KW;                              // this warp's first key of a tile
        const float c2 = p.scale * 1.4426950408889634f;
        const uint32_t q_at = x.sbase + C::OffQ;
        int16_t *par = reinterpret_cast<int16_t *>(smem + C::OffPar);
        float2 *ml = reinterpret_cast<float2 *>(smem + C::OffMl);
        float *stage = reinterpret_cast<float *>(smem + C::OffQ);
        uint32_t keys = 0;                                   // tiles of the segments before
        auto sync = [&]() { return x.ok = all_well<kConsumers * 32>(x.ok); };
        Rec r;
        for (uint32_t seg = 0;; ++seg) {
            const bool more = x.record(seg, r);
            if (!sync() || !more) break;                     // everyone is through with the last segment
            const bool tree = p.parent != nullptr && r.t1 > r.ct;
            if (threadIdx.x == 0) x.topo_bad[(seg & 1) ^ 1] = 0;
            for (int i = threadIdx.x; i < r.rows * (D / 8); i += kConsumers * 32) {
                const int row = i / (D / 8), c = i % (D / 8), at = r.row0 + row, node = group.over(at), g = at - node * group.n;
                copy16(q_at + tile_offset<D>(row, c), p.q + ((size_t(r.l) * p.T + r.base + node) * p.H + r.hk * group.n + g) * D + c * 8);
            }
            if (tree) {                                      // (at most as many nodes as rows)
                int bad = 0;
                for (int i = threadIdx.x; i < r.n; i += kConsumers * 32) {
                    const int up = p.parent[r.base + i];
                    bad |= up < -1 || up >= i;
                    par[i] = int16_t(up < -1 || up >= i ? -1 : up);
                }
                if (__any_sync(0xffffffffu, bad) && lane == 0) {
                    x.topo_bad[seg & 1] = 1;
                    atomicOr(p.status, SPECA_STATUS_BAD_PARENT);
                }
            }
            copy16_wait();
            if (!sync()) break;
            // this lane's rows of the unit, and the draft nodes they attend (no more nodes than rows)
            const int row0 = lane >> 2;
            uint32_t seen[2] = {0u, 0u};
            bool live[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                live[h] = row0 + 8 * h < r.rows;
                if (!live[h] || r.t1 <= r.ct) continue;
                for (int a = group.over(r.row0 + row0 + 8 * h); a >= 0; a = tree ? int(par[a]) : a - 1) seen[h] |= 1u << a;
            }
            float o[OC / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < OC / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
            bool mend = false;

#pragma unroll 1
            for (int t = r.t0; t < r.t1; ++t, ++keys) {
                const int valid = x.valid_of(r, t);
                const bool draft = t >= r.ct, mine = k0 < valid;                 // (a warp whose keys are past the end only keeps step)
                const uint32_t ks = keys % KS, vs = keys % VS;
                if (!(x.ok = wait_fast(x.bar(C::kKFull + ks), (keys / KS) & 1, x.abort_flag))) break;
                float s[KW / 8][4];
#pragma unroll
                for (int j = 0; j < KW / 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
                if (mine) {
                    const uint32_t kt = x.sbase + C::OffRing + ks * C::TILE;
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        uint32_t a[4];
                        ldmatrix4(q_at + tile_offset<D>(lane & 15, 2 * k + (lane >> 4)), a);
#pragma unroll
                        for (int j = 0; j < KW / 16; ++j) {
                            uint32_t b[4];
                            ldmatrix4(kt + tile_offset<D>(k0 + 16 * j + (lane & 7) + (lane >> 4) * 8, 2 * k + (lane >> 3 & 1)), b);
                            mma_bf16_sync(s[2 * j], a, b[0], b[1]);
                            mma_bf16_sync(s[2 * j + 1], a, b[2], b[3]);
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(x.bar(C::kKEmpty + ks));
                const bool masked = draft || k0 + KW > valid;
                if (mine) {
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < KW / 8; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int key = k0 + 8 * j + (lane & 3) * 2 + (e & 1);
                                if (key >= valid || (draft && !(seen[e >> 1] >> (key & 31) & 1u))) s[j][e] = -INFINITY;
                            }
                    }
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < KW / 8; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) top[e >> 1] = fmaxf(top[e >> 1], s[j][e]);
                    bool grow = false;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
                        top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
                        grow |= live[h] && ((top[h] - m[h]) * c2 > kSlack || (m[h] == -INFINITY && top[h] > m[h]));
                    }
                    if (__any_sync(0xffffffffu, grow)) {
                        float f[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float now = fmaxf(m[h], top[h]);
                            // (before its first key a row's sums are zero, in whatever scale)
                            f[h] = m[h] == now || m[h] == -INFINITY ? 1.f : exp2_approx((m[h] - now) * c2);
                            m[h] = now;
                            l[h] *= f[h];
                        }
#pragma unroll
                        for (int j = 0; j < OC / 8; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[j][e] *= f[e >> 1];
                    }
                    float mc[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) mc[h] = m[h] == -INFINITY ? 0.f : m[h] * c2;
#pragma unroll
                    for (int j = 0; j < KW / 8; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[j][e] = exp2_approx(fmaf(s[j][e], c2, -mc[e >> 1]));
                            l[e >> 1] += s[j][e];
                        }
                }
                if (!(x.ok = wait_fast(x.bar(C::kVFull + vs), (keys / VS) & 1, x.abort_flag))) break;
                if (mine) {
                    const uint32_t vt = x.sbase + C::OffRing + (KS + vs) * C::TILE;
#pragma unroll
                    for (int g = 0; g < KW / 16; ++g) {
                        const uint32_t a[4] = {pack_bf16(s[2 * g][0], s[2 * g][1]), pack_bf16(s[2 * g][2], s[2 * g][3]),
                                               pack_bf16(s[2 * g + 1][0], s[2 * g + 1][1]), pack_bf16(s[2 * g + 1][2], s[2 * g + 1][3])};
                        const int key = k0 + 16 * g;
                        if (key >= valid) continue;
#pragma unroll
                        for (int j = 0; j < OC / 16; ++j) {
                            uint32_t b[4];
                            ldmatrix4_trans(vt + tile_offset<D>(key + (lane & 15), ch * (OC / 8) + 2 * j + (lane >> 4)), b);
                            if (masked) {
                                // A weight of zero does not take a value that is not finite out of a product.  Rows past the end (what
                                // was there before, or never written) are left out; draft values that are not finite, which only some
                                // rows attend, are put back at the end.
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int at = key + (lane & 3) * 2 + (e & 1) * 8;
                                    b[e] &= (at < valid ? 0x0000ffffu : 0u) | (at + 1 < valid ? 0xffff0000u : 0u);
                                    if (draft) mend |= strip(b[e]);
                                }
                            }
                            mma_bf16_sync(o[2 * j], a, b[0], b[1]);
                            mma_bf16_sync(o[2 * j + 1], a, b[2], b[3]);
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(x.bar(C::kVEmpty + vs));
            }

            // ---- end of the segment: the warps' sums are joined in the order of their keys
            if (__any_sync(0xffffffffu, mend) && lane == 0) x.value_bad[seg % kFlagRing] = int(seg) + 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
                if ((lane & 3) == 0) ml[warp * kRows + row0 + 8 * h] = make_float2(m[h], l[h]);
            }
            if (!sync()) break;                              // (the queries have been used by all)
            const bool skip = (x.topo_bad[seg & 1] != 0 && tree) || x.page_bad[seg % kFlagRing] == int(seg) + 1;
            const bool put_back = x.value_bad[seg % kFlagRing] == int(seg) + 1;
            float *sums = r.slot >= 0 ? slot_sums(plan, cta, r.slot) : nullptr;
            auto out_of = [&](int row) {
                const int at = r.row0 + row, node = group.over(at), g = at - node * group.n;
                return p.o + ((size_t(r.l) * p.T + r.base + node) * p.H + r.hk * group.n + g) * D;
            };
            if (sums != nullptr && threadIdx.x == 0) reinterpret_cast<int *>(sums + size_t(plan.rows_cap) * (D + 2))[0] = skip;
#pragma unroll
            for (int turn = 0; turn < OC / 64; ++turn) {
                if (turn > 0 && !sync()) break;
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *reinterpret_cast<float2 *>(stage + stage_offset(warp, row0 + 8 * h, 8 * j + (lane & 3) * 2)) =
                            make_float2(o[8 * turn + j][2 * h], o[8 * turn + j][2 * h + 1]);
                if (!sync()) break;
                // four columns of a row a thread, of the 64 that each group of warps has put there
#pragma unroll 1
                for (int u = threadIdx.x; u < r.rows * (C::CH * 16) && !skip; u += kConsumers * 32) {
                    const int row = u / (C::CH * 16), part = u / 16 % C::CH, e = u % 16 * 4, first = part * KB, col = part * OC + 64 * turn + e;
                    float mm = -INFINITY, ll = 0.f;
#pragma unroll
                    for (int i = 0; i < KB; ++i) mm = fmaxf(mm, ml[(first + i) * kRows + row].x);
                    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int i = 0; i < KB; ++i) {
                        const float2 w = ml[(first + i) * kRows + row];
                        // (a warp without a key of this row has zeros)
                        const float f = w.x == mm || w.x == -INFINITY ? 1.f : exp2_approx((w.x - mm) * c2);
                        const float4 y = *reinterpret_cast<const float4 *>(stage + stage_offset(first + i, row, e));
                        ll = fmaf(w.y, f, ll);
                        sum.x = fmaf(y.x, f, sum.x); sum.y = fmaf(y.y, f, sum.y); sum.z = fmaf(y.z, f, sum.z); sum.w = fmaf(y.w, f, sum.w);
                    }
                    if (sums == nullptr) {
                        const float inv = 1.f / ll;
                        *reinterpret_cast<uint2 *>(out_of(row) + col) = make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
                    } else {
                        *reinterpret_cast<float4 *>(sums + size_t(row) * D + col) = sum;
                        if (col == 0) reinterpret_cast<float2 *>(sums + size_t(plan.rows_cap) * D)[row] = make_float2(mm, ll);
                    }
                }
            }
            if (!x.ok) break;
            // (what other threads wrote is read back)
            if (put_back && !skip && !sync()) break;
            if (put_back && !skip)
                for (int u = threadIdx.x; u < r.rows * D; u += kConsumers * 32) {
                    // (column u % D of a row; what other threads have written of it is behind the last sync)
                    const int row = u / D, col = u % D;
                    for (int a = group.over(r.row0 + row); a >= 0; a = tree ? int(par[a]) : a - 1) {
                        const float y = __bfloat162float(p.v[((size_t(r.l) * p.T + r.base + a) * p.HK + r.hk) * D + col]);
                        if (isfinite(y)) continue;
                        if (sums == nullptr) out_of(row)[col] = __float2bfloat16_rn(__bfloat162float(out_of(row)[col]) + y);
                        else sums[size_t(row) * D + col] += y;
                    }
                }
        }
    }
    if ((warp == kConsumers || warp == kConsumers + 2) && *x.abort_flag) {
        // let copies still in flight land before the CTA's shared memory goes away
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    __syncthreads();
    if (*x.abort_flag) x.refuse();
}

std::atomic<bool> g_opted_in[64];                            // per device: shared memory of every instantiation

template <int D> int launch_few(const AttnParams &p, const Maps &maps, const Plan &plan, int box_rows, int grid, cudaStream_t st)
{
    using C = Few<D>;
    launch(attend_few_kernel<D>, unsigned(grid), C::THREADS, C::Bytes, st, maps, p, plan, int32_t(box_rows));
    return int(cudaGetLastError());
}

}  // namespace

// A chain of n tokens, 32 sequences over 500..8000 tokens, 32 heads over 8 of 128 columns, this kernel / the other one: 4 rows 97 /
// 104 us, 16 rows 102 / 106; of two blocks of 16 rows 156 / 107, of four 273 / 116.
int attend_few_rows(long rows) { return rows <= kRows ? kRows : 0; }

int launch_attend_few(const AttnParams &p, int d_head, const Maps &maps, const Plan &plan, int box_rows, int grid, cudaStream_t st)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return int(cudaErrorInvalidDevice);
    if (!g_opted_in[dev].load(std::memory_order_acquire)) {
        cudaError_t e = cudaSuccess;
        auto opt_in = [&](const void *k, int bytes) {
            if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        };
        opt_in(reinterpret_cast<const void *>(attend_few_kernel<64>), Few<64>::Bytes);
        opt_in(reinterpret_cast<const void *>(attend_few_kernel<128>), Few<128>::Bytes);
        opt_in(reinterpret_cast<const void *>(attend_few_kernel<256>), Few<256>::Bytes);
        if (e != cudaSuccess) return int(e);
        g_opted_in[dev].store(true, std::memory_order_release);
    }
    if (d_head == 64) return launch_few<64>(p, maps, plan, box_rows, grid, st);
    if (d_head == 128) return launch_few<128>(p, maps, plan, box_rows, grid, st);
    return launch_few<256>(p, maps, plan, box_rows, grid, st);
}

}  // namespace speca
