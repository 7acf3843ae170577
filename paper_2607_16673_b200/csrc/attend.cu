// Verification by an attention layer: draft nodes attend the committed rows of a paged cache and their own ancestors.
//
// For a key head the rows of a product are the (node, query head) pairs of a sequence that share it, up to 128 a tile; the
// columns are keys.  Per tile of N keys:  S = Q K^T (both operands in shared memory, K as its pages lie), the weights
// P = exp2((S - m) scale log2 e) with a running maximum m, rounded to bf16 and written over S in TMEM, and O += P V with P
// from TMEM and V as its pages lie (keys along the rows: an MN-major operand).  The rounding of P is the tensor core's: both operands
// of a product have one type, and V is bf16.  It adds 1.5e-3 of the output's norm to the 1.7e-3 of the output's own rounding
// (2.2e-3 in all against 64 bits); the remainder of P in a second product would take it away for half as many products again.
// The sum of weights is of the unrounded ones.  O stays in TMEM; it is scaled down only when
// a row's maximum has grown by more than kSlack, so that a weight is at most 2^kSlack and the sum of weights, kept in fp32,
// and O are in the same scale whatever that scale is.
//
// Work: the tiles of all (sequence, layer, key head, row tile) units stand in one list, and every CTA takes an equal piece of
// it, so the batch's lengths do not matter and a single long context occupies every SM.  A unit cut by the border of two
// pieces leaves unnormalised sums with their maxima in the workspace, which a second kernel joins in the order of the pieces.
#include "attend_common.cuh"

namespace speca {

using namespace attend;

namespace {

constexpr float kSlack = 8.f;            // binary digits a maximum may grow by before O is scaled

// D <= 128: two softmax groups of 128 rows, each with an O of its own.  A unit of at most 128 rows has its even key tiles in one
// and the odd ones in the other, joined at the end; a larger one has a row tile in each, over the same keys.  D = 256: O alone
// takes half of TMEM, and there is one group; its queries have a quarter of TMEM, so that a tile's scores do not read 64 KB of
// shared memory once more and the rings have room for one tile more.  Of the 1880 cycles of a tile (16 trees of 40..64 nodes behind
// 2001..30000) the softmax warps work 1310, one on each scheduler; the product warp waits 920 for weights and 640 for values, the
// score warp 540 for keys.  P takes the first half of the columns of its S.  One warp asks for scores, another
// for the products with V, so that neither's waits hold the other up (a loop over one item takes 1200 cycles beside its 12
// products where one warp does both).
// MANY: units of more than 128 rows.  Products and softmax bound these: tiles of 64 keys leave room for a second buffer of S in
// each group, formed while it works on the first (1024 prompt tokens behind 1500 and 4096: 166 us, tiles of 128 180).  Up to
// 128 rows it is the keys' bytes: tiles of 128, and the second row tile's queries make room for one more of each ring (32 trees
// of 64 rows 115 us, tiles of 64 125).
template <int DH, bool MANY> struct Cfg {
    static constexpr int D = DH;
    static constexpr int LANES = D == 256 ? 1 : 2;
    static constexpr int N = MANY || D == 256 ? 64 : 128;
    static constexpr int BUFS = LANES == 2 && MANY ? 4 : 2;
    static constexpr int MT = MANY && LANES == 2 ? 256 : 128;
    static constexpr int kEnds = N == 128 ? 5 : D == 256 ? 8 : 10;          // a unit's beginning and end in tiles: some 15000 cycles
    // 384 keys (512) and 768: 20 trees of 9..40 nodes behind 10..300 tokens 26.7 -> 18.9 us, one tree of 64 at 256 columns behind 3000
    // 55.5 -> 37.7, of 32 at 128 columns behind 1000 24.2 -> 20.4, large calls as they were
    static constexpr int kPiece = D == 256 ? 8 : 3 * (128 / N), kWhole = 6 * (128 / N);
    static constexpr bool kMend = true;
    static constexpr int SOFT = 4 * LANES;                   // softmax warps; then keys, scores, products with V, mending of V, schedule, values
    static constexpr int THREADS = (SOFT + 6) * 32;
    static constexpr int Q_BYTES = 128 * D * 2;              // queries of a row tile; at a unit's end sums on their way, 4096 bytes a warp
    static constexpr int Q_ALL = D < 256 && Q_BYTES * (MT / 128) > 4096 * SOFT ? Q_BYTES * (MT / 128) : 4096 * SOFT;
    static constexpr int TILE = N * D * 2;                   // keys or values of a tile
    static constexpr int FIT = (228 * 1024 - Q_ALL) / TILE - (D == 64 ? 1 : 0);                  // tiles in flight or in use
    static constexpr int VS = FIT / 2, KS = FIT - VS;
    static constexpr int OffQ = 0;
    static constexpr int OffRing = Q_ALL;
    static constexpr int OffPar = OffRing + (KS + VS) * TILE;    // int16 parent[kAttnMaxTree]
    static constexpr int OffRec = OffPar + 2 * kAttnMaxTree;
    static constexpr int OffBars = OffRec + 64 * kRecords;
    static constexpr int kKFull = 0, kKEmpty = KS, kVFull = 2 * KS, kVEmpty = kVFull + VS, kVRaw = kVEmpty + VS, kSFull = kVRaw + VS, kPReady = kSFull + BUFS, kODone = kPReady + BUFS,
                         kQFull = kODone + BUFS, kRecFull = kQFull + 1, kRecEmpty = kRecFull + kRecords,
                         kDrain = kRecEmpty + kRecords, kBars = kDrain + 1;
    static constexpr int OffMisc = OffBars + 8 * kBars;      // abort, TMEM base, bad topology [2]
    static constexpr int OffFlags = OffMisc + 64;            // segment numbers: bad page [8], values that are not finite [8]
    static constexpr int Bytes = OffFlags + 8 * kFlagRing;
};
template <class C> constexpr bool fits() { return C::Bytes <= 232448 && C::KS >= 2 && C::VS >= 2; }
static_assert(fits<Cfg<64, false>>() && fits<Cfg<64, true>>() && fits<Cfg<128, false>>() && fits<Cfg<128, true>>() && fits<Cfg<256, true>>(),
              "shared memory of a CTA");

constexpr int kTmemCols = 512, kQCol = 128, kOCol = 256;     // S (P) buffers from 0, N columns each, at D = 256 the queries, O

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *r)
{
    uint32_t x[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]),
          "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(x[16]), "=r"(x[17]), "=r"(x[18]),
          "=r"(x[19]), "=r"(x[20]), "=r"(x[21]), "=r"(x[22]), "=r"(x[23]), "=r"(x[24]), "=r"(x[25]), "=r"(x[26]), "=r"(x[27]),
          "=r"(x[28]), "=r"(x[29]), "=r"(x[30]), "=r"(x[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __uint_as_float(x[i]);
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float *r)
{
    uint32_t x[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]),
          "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __uint_as_float(x[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&x)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]),
          "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st2(uint32_t taddr, float x, float y)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};" ::"r"(taddr), "f"(x), "f"(y) : "memory");
}
__device__ __forceinline__ void tmem_ld2(uint32_t taddr, float2 &x)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// kind::f16 (bf16) with the A operand in TMEM: a 32-bit column holds two consecutive K elements, the even one low
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                            uint32_t lead)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(lead)
        : "memory");
}
// operand whose rows are M or N (keys of S = Q K^T), `group` bytes between groups of eight rows
__device__ __forceinline__ uint64_t make_desc_k(uint32_t smem_addr, uint32_t group)
{
    return (make_desc(smem_addr) & ~(uint64_t(0x3fff) << 32)) | uint64_t((group >> 4) & 0x3fffu) << 32;
}
// operand whose rows are K (values of O = P V): 1024 bytes from one 64-wide block of columns to the next, `group` between
// groups of eight rows
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t smem_addr, uint32_t group)
{
    return (make_desc_k(smem_addr, group) & ~(uint64_t(0x3fff) << 16)) | uint64_t(1024 >> 4) << 16;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
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
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
template <int D, bool MANY>
__global__ void __launch_bounds__(Cfg<D, MANY>::THREADS, 1)
attend_kernel(const __grid_constant__ Maps maps, AttnParams p, Plan plan, int32_t box_rows)
{
    after_previous_kernel();
    using C = Cfg<D, MANY>;
    constexpr int N = C::N, LANES = C::LANES, BUFS = C::BUFS, SOFT = C::SOFT, KS = C::KS, VS = C::VS;
    extern __shared__ __align__(1024) uint8_t smem[];
    Cta<C> x(p, plan, smem);
    const uint32_t sbase = x.sbase;
    if ((sbase & 1023u) != 0u || p.misplaced) {              // never expected; refuse to run rather than corrupt
        x.refuse();
        return;
    }
    auto bar = [&](int i) { return x.bar(i); };
    volatile int *const abort_flag = x.abort_flag, *const topo_bad = x.topo_bad;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + C::OffMisc + 4);
    const int warp = x.warp, lane = x.lane, cta = blockIdx.x;
    const Group group = x.group;

    if (warp == 0) {
        x.init(SOFT + 5, 1);
        if (lane < VS) mbar_init(bar(C::kVRaw + lane), 1);
        if (lane < BUFS) { mbar_init(bar(C::kSFull + lane), 1); mbar_init(bar(C::kPReady + lane), 4); mbar_init(bar(C::kODone + lane), 1); }
        if (lane == 0) {
            mbar_init(bar(C::kQFull), SOFT);
            mbar_init(bar(C::kDrain), 2);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == SOFT + 1) tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), kTmemCols);

    x.begin();
    const uint32_t tmem = *tmem_slot, lead = x.lead;
    bool &ok = x.ok;
    auto record = [&](uint32_t s, Rec &r) { return x.record(s, r); };
    auto valid_of = [&](const Rec &r, int t) { return x.valid_of(r, t); };
    // Buffer of item i of a segment.  Every use of a buffer is one phase of its three barriers (scores there, weights there,
    // weights used); a role keeps the parity of the next one, a bit a buffer.
    auto buffer = [](int i) { return i & (BUFS - 1); };
    Rec r;

    if (warp == SOFT) {
        // ------------------------------------------------------------------------------- keys and values, by TMA
        x.template load<0>(maps, box_rows);
    } else if (warp == SOFT + 1) {
        // ------------------------------------------------------------------------------- scores
        const uint32_t id_s = make_idesc_bf16(N);
        uint32_t loads = 0, phase = 0;                       // tiles of the segments before; next parities
        for (uint32_t seg = 0; ok && record(seg, r); ++seg) {
            const bool two = C::MT == 256 && r.rows > 128;     // two row tiles over the same keys
            const int tiles = r.t1 - r.t0, items = tiles << (two ? 1 : 0);
            if (!(ok = wait_fast(bar(C::kQFull), seg & 1, abort_flag))) break;
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < items; ++i) {
                const uint32_t kt = loads + (two ? i >> 1 : i), s = kt % KS;
                const int buf = buffer(i);
                if ((!two || !(i & 1)) && !(ok = wait_fast(bar(C::kKFull + s), (kt / KS) & 1, abort_flag))) break;
                // the weights that were in the same columns have been used
                if (i >= BUFS && !(ok = wait_fast(bar(C::kODone + buf), ((phase >> buf) & 1) ^ 1, abort_flag))) break;
                phase ^= 1u << buf;
                tc_fence_after();
                const uint64_t qd = make_desc(sbase + C::OffQ + (two ? (i & 1) * C::Q_BYTES : 0)), kd = make_desc_k(sbase + C::OffRing + s * C::TILE, 16 * D);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    if constexpr (D == 256)
                        mma_bf16_ts(tmem + buf * N, tmem + kQCol + 8 * k, kd + uint64_t(((k >> 2) * 1024 + (k & 3) * 32) >> 4), id_s, k != 0, lead);
                    else
                        mma_bf16(tmem + buf * N, qd + uint64_t(((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4),
                             kd + uint64_t(((k >> 2) * 1024 + (k & 3) * 32) >> 4), id_s, k != 0, lead);
                mma_commit(bar(C::kSFull + buf), lead);
                if (!two || (i & 1)) mma_commit(bar(C::kKEmpty + s), lead);
            }
            loads += tiles;
        }
    } else if (warp == SOFT + 2) {
        // ------------------------------------------------------------------------------- products with V
        const uint32_t id_o = make_idesc_bf16(D) | (1u << 16);   // (B is MN-major)
        uint32_t loads = 0, phase = 0;
        for (uint32_t seg = 0; ok && record(seg, r); ++seg) {
            const bool two = C::MT == 256 && r.rows > 128;
            const int tiles = r.t1 - r.t0, items = tiles << (two ? 1 : 0);
#pragma unroll 1
            for (int i = 0; i < items; ++i) {
                const int buf = buffer(i), ti = two ? i >> 1 : i, valid = valid_of(r, r.t0 + ti);
                const uint32_t vt = loads + ti, s = vt % VS;
                if ((!two || !(i & 1)) && !(ok = wait_fast(bar(C::kVFull + s), (vt / VS) & 1, abort_flag))) break;
                if (!(ok = wait_fast(bar(C::kPReady + buf), (phase >> buf) & 1, abort_flag))) break;
                phase ^= 1u << buf;
                tc_fence_after();
                const int oc = LANES == 2 ? kOCol + (i & 1) * D : kOCol, steps = (valid + 15) >> 4;
                const uint64_t vd = make_desc_mn(sbase + C::OffRing + (KS + s) * C::TILE, 16 * D);
#pragma unroll
                for (int k = 0; k < N / 16; ++k)
                    if (k < steps)
                        mma_bf16_ts(tmem + oc, tmem + buf * N + 8 * k, vd + uint64_t(k * (2 * 16 * D >> 4)), id_o, !(i < LANES && k == 0), lead);
                mma_commit(bar(C::kODone + buf), lead);
                if (!two || (i & 1)) mma_commit(bar(C::kVEmpty + s), lead);
            }
            loads += tiles;
        }
    } else if (warp == SOFT + 3) {
        // ------------------------------------------------------------------------------- mending of V
        // A weight of zero does not take a value that is not finite out of a product: rows past the end of a tile's keys (what
        // was there before, another sequence's, or never written) are set to zero, and so are draft values that are not finite,
        // which only some rows attend; those get them back at the end.
        uint32_t loads = 0, phase = 0;                       // phase: a bit a slot
        for (uint32_t seg = 0; ok && record(seg, r); loads += r.t1 - r.t0, ++seg) {
#pragma unroll 1
            for (int t = r.t0; t < r.t1; ++t) {
                if (!x.to_mend(r, t)) continue;
                const int valid = valid_of(r, t);
                const bool draft = !x.all_seen(r, t);
                const uint32_t s = (loads + (t - r.t0)) % VS;
                if (!(ok = wait_fast(bar(C::kVRaw + s), (phase >> s) & 1, abort_flag))) break;
                phase ^= 1u << s;
                uint8_t *v = smem + C::OffRing + (KS + s) * C::TILE;
                const int end = (valid + 15) & ~15;
                for (int i = valid * (D / 8) + lane; i < end * (D / 8); i += 32) {
                    const int row = i / (D / 8), c = i % (D / 8);
                    *reinterpret_cast<uint4 *>(v + tile_offset<D>(row, c)) = make_uint4(0u, 0u, 0u, 0u);
                }
                if (draft) {
                    bool bad = false;
#pragma unroll 4
                    for (int i = lane; i < valid * (D / 8); i += 32) {
                        const int row = i / (D / 8), c = i % (D / 8);
                        uint4 *at = reinterpret_cast<uint4 *>(v + tile_offset<D>(row, c));
                        const uint4 x = *at;
                        if (not_finite(x.x) || not_finite(x.y) || not_finite(x.z) || not_finite(x.w)) {
                            uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
                                if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu;
                            }
                            *at = make_uint4(w[0], w[1], w[2], w[3]);
                            bad = true;
                        }
                    }
                    if (bad) x.value_bad[seg % kFlagRing] = int(seg) + 1;
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::kVFull + s));
            }
        }
    } else if (warp == SOFT + 4) {
        // ------------------------------------------------------------------------------- schedule
        x.schedule();
    } else if (warp == SOFT + 5) {
        x.template load<1>(maps, box_rows);
    } else {
        // ------------------------------------------------------------------------------- softmax, and what is written
        const int wg = warp >> 2, quad = warp & 3, trow = quad * 32 + lane;      // lane of TMEM: row of this group's tile
        const uint32_t tq = tmem + (uint32_t(quad * 32) << 16);
        const float c2 = p.scale * 1.4426950408889634f;
        uint32_t phase = 0;
        int16_t *par = reinterpret_cast<int16_t *>(smem + C::OffPar);
        auto sync = [&]() { return ok = all_well<SOFT * 32>(ok); };
        for (uint32_t seg = 0;; ++seg) {
            const bool more = record(seg, r);
            if (!sync() || !more) break;                     // everyone is through with the last segment: its queries, its parents
            const bool two = C::MT == 256 && r.rows > 128;
            const int tiles = r.t1 - r.t0;
            const int all = tiles << (two ? 1 : 0);          // items of both groups
            if (threadIdx.x == 0) topo_bad[(seg & 1) ^ 1] = 0;
            const int first = group.over(r.row0), ahead = r.row0 - first * group.n;
            const __nv_bfloat16 *queries = p.q + ((size_t(r.l) * p.T + r.base) * p.H + r.hk * group.n) * D;
            if constexpr (D == 256) {
                if (quad * 32 < r.rows) {
                    const int at = ahead + trow, past = group.over(at);
                    const uint4 *from = reinterpret_cast<const uint4 *>(queries + (size_t(first + past) * p.H + (at - past * group.n)) * D);
#pragma unroll 1
                    for (int c = 0; c < 4; c += 2) {
                        uint4 y[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = trow < r.rows ? from[8 * c + e] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const uint32_t z[16] = {y[4 * h].x, y[4 * h].y, y[4 * h].z, y[4 * h].w, y[4 * h + 1].x, y[4 * h + 1].y, y[4 * h + 1].z,
                                                    y[4 * h + 1].w, y[4 * h + 2].x, y[4 * h + 2].y, y[4 * h + 2].z, y[4 * h + 2].w,
                                                    y[4 * h + 3].x, y[4 * h + 3].y, y[4 * h + 3].z, y[4 * h + 3].w};
                            tmem_st16(tq + kQCol + 32 * c + 16 * h, z);
                        }
                    }
                    tmem_st_wait();
                    tc_fence_before();
                }
            } else {
                const int chunks = r.rows * (D / 8);
#pragma unroll 2
                for (int i = threadIdx.x; i < chunks; i += SOFT * 32) {
                    const int row = i / (D / 8), c = i % (D / 8), at = ahead + row, past = group.over(at);
                    const int tile = row >> 7, tr = row & 127;
                    copy16(sbase + C::OffQ + tile * C::Q_BYTES + (c >> 3) * (128 * 128) + tr * 128 + (((c & 7) ^ (tr & 7)) << 4),
                           queries + (size_t(first + past) * p.H + (at - past * group.n)) * D + c * 8);
                }
                copy16_wait();
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::kQFull));
            if (p.parent != nullptr && r.t1 > r.ct) {        // (a piece without draft keys is joined with one that looks)
                int bad = 0;
                for (int i = threadIdx.x; i < r.n; i += SOFT * 32) {
                    const int up = p.parent[r.base + i];
                    bad |= up < -1 || up >= i;
                    par[i] = int16_t(up < -1 || up >= i ? -1 : up);
                }
                if (__any_sync(0xffffffffu, bad) && lane == 0) {
                    topo_bad[seg & 1] = 1;
                    atomicOr(p.status, SPECA_STATUS_BAD_PARENT);
                }
                if (!sync()) break;
            }
            const int row = (two ? wg * 128 : 0) + trow;     // row of the unit
            const bool live = (two ? wg * 128 : 0) + quad * 32 < r.rows;     // the warp has rows
            const int at = r.row0 + (row < r.rows ? row : 0), node = group.over(at), g = at - node * group.n;
            float m = -INFINITY, l = 0.f;
            const int mine = LANES == 2 ? (all + 1 - wg) / 2 : all;          // items of this group
            uint32_t uses = phase;                           // parities that its own items have turned
#pragma unroll 1
            for (int i = 0; i < mine; ++i) {
                const int item = LANES == 2 ? 2 * i + wg : i, buf = buffer(item), t = r.t0 + (two ? i : item);
                if (!(ok = wait_fast(bar(C::kSFull + buf), (uses >> buf) & 1, abort_flag))) break;
                uses ^= 1u << buf;
                tc_fence_after();
                if (live) {
                    const uint32_t ta = tq + buf * N;
                    const int valid = valid_of(r, t);
                    const bool masked = valid < N || !x.all_seen(r, t);
                    uint32_t mask[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
                    if (masked) {
                        const int first = (t - r.ct) * N;    // first node of a draft tile
                        if (t < r.ct || p.parent == nullptr) {
                            const int upto = t < r.ct ? valid : node + 1 - first;
#pragma unroll
                            for (int w = 0; w < N / 32; ++w) {
                                const int x = upto - 32 * w;
                                mask[w] = x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u;
                            }
                        } else {
#pragma unroll
                            for (int w = 0; w < N / 32; ++w) mask[w] = 0u;
                            for (int a = node; a >= first; a = par[a]) {
                                const int x = a - first;
#pragma unroll
                                for (int w = 0; w < N / 32; ++w) mask[w] |= (x >> 5) == w ? 1u << (x & 31) : 0u;
                            }
                        }
                    }
                    // Scores are read twice, for the maximum and for the weights, 32 at a time: these loops and what stands around
                    // them have to stay in the instruction cache together (unrolled over the tile, the end of every segment
                    // was fetched anew, at 6000 to 11000 cycles for a few hundred instructions).
                    float s[32];
                    auto load = [&](int c) {
                        tmem_ld32(ta + 32 * c, s);
                        tmem_ld_wait();
                        if (masked) {
                            const uint32_t w = c == 0 ? mask[0] : c == 1 ? mask[1] : c == 2 ? mask[2] : mask[3];
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(w >> e & 1u)) s[e] = -INFINITY;
                        }
                    };
                    float top = -INFINITY, other = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < N / 32; ++c) {
                        load(c);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            top = max3(top, s[e], s[e + 1]);
                            other = max3(other, s[e + 2], s[e + 3]);
                        }
                    }
                    top = fmaxf(top, other);
                    if (i == 0) m = top;
                    // (rows past the unit's last hold whatever was there: they have no say)
                    else if (__any_sync(0xffffffffu, row < r.rows && ((top - m) * c2 > kSlack || (m == -INFINITY && top > m)))) {
                        // the last item's product must have been added before O is scaled (where that item had this
                        // buffer too, its parity is two turns old)
                        const int pb = buffer(item - LANES);
                        if (!(ok = wait_fast(bar(C::kODone + pb), ((uses >> pb) & 1) ^ (pb != buf), abort_flag))) break;
                        tc_fence_after();
                        const float now = fmaxf(m, top);
                        // (before its first key a row's sums are zero, in whatever scale)
                        const float f = m == now || m == -INFINITY ? 1.f : exp2_approx((m - now) * c2);
                        m = now;
                        l *= f;
                        const uint32_t to = tq + kOCol + (LANES == 2 ? wg * D : 0);
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            float o[16];
                            uint32_t x[16];
                            tmem_ld16(to + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(o[e] * f);
                            tmem_st16(to + c, x);
                        }
                        tmem_st_wait();
                    }
                    const float mc = m == -INFINITY ? 0.f : m * c2;
                    const uint64_t scale2 = pair2(c2, c2), shift2 = pair2(-mc, -mc);
                    uint64_t add[2] = {0u, 0u};
#pragma unroll 1
                    for (int c = 0; c < N / 32; ++c) {
                        load(c);
                        uint32_t x[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float a, b;
                            unpair2(fma2(pair2(s[2 * e], s[2 * e + 1]), scale2, shift2), a, b);
                            a = exp2_approx(a);
                            b = exp2_approx(b);
                            add[e & 1] = add2(add[e & 1], pair2(a, b));
                            x[e] = pack_bf16(a, b);
                        }
                        tmem_st16(ta + 16 * c, x);           // (over scores that have been read)
                    }
                    float a0, a1, a2, a3;
                    unpair2(add[0], a0, a1);
                    unpair2(add[1], a2, a3);
                    l += (a0 + a1) + (a2 + a3);
                    tmem_st_wait();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::kPReady + buf));
            }

            // ---- end of the segment: this group's last product covers those before it
            const bool merge = LANES == 2 && !two;
            if (mine > 0 && ok) {
                const int last = buffer(LANES == 2 ? 2 * (mine - 1) + wg : mine - 1);
                ok = wait_fast(bar(C::kODone + last), ((uses >> last) & 1) ^ 1, abort_flag);
            }
            if (!ok) { sync(); break; }
#pragma unroll
            for (int b = 0; b < BUFS; ++b) phase ^= uint32_t((all + BUFS - 1 - b) / BUFS & 1) << b;      // items of all groups in buffer b
            tc_fence_after();
            float f0 = 1.f, f1 = 0.f, mm = m, ll = l;
            if (merge) {
                // Sums of even and odd tiles: both groups read both, half of the columns each.  Maxima and sums of weights go through
                // the columns of the group's last weights.
                tmem_st2(tq + wg * N, m, l);
                tmem_st_wait();
                tc_fence_before();
                if (!sync()) break;
                tc_fence_after();
                float2 a, b;
                tmem_ld2(tq, a);
                tmem_ld2(tq + N, b);
                tmem_ld_wait();
                mm = fmaxf(a.x, b.x);
                const float base = mm == -INFINITY ? 0.f : mm;
                f0 = a.x == mm ? 1.f : exp2_approx((a.x - base) * c2);
                f1 = b.x == mm ? 1.f : exp2_approx((b.x - base) * c2);
                // (a maximum that is not a number belongs to sums that are not either)
                ll = a.y * f0 + (all > 1 ? b.y * f1 : 0.f);
            }
            const bool bad = topo_bad[seg & 1] != 0 && p.parent != nullptr && r.t1 > r.ct;
            const bool skip = bad || x.page_bad[seg % kFlagRing] == int(seg) + 1;
            const bool mend = x.value_bad[seg % kFlagRing] == int(seg) + 1;
            if (live) {
                const uint32_t o0 = tq + kOCol + (LANES == 2 && two ? wg * D : 0), o1 = tq + kOCol + D;
                const bool both = merge && all > 1;
                const int c_lo = merge ? wg * (D / 2) : 0, c_hi = merge ? c_lo + D / 2 : D;
                const float inv = 1.f / ll;
                float *sums = r.slot >= 0 ? slot_sums(plan, cta, r.slot) : nullptr;
                __nv_bfloat16 *out = p.o + ((size_t(r.l) * p.T + r.base + node) * p.H + r.hk * group.n + g) * D;
                const bool write = row < r.rows && !skip;
                if (sums == nullptr) { f0 *= inv; f1 *= inv; }
                // Through shared memory (this group's queries have been used), so that a row is written in whole lines: straight
                // from the lanes, a row each, a store touched 32 lines, and 128 rows took 9000 cycles.
                uint8_t *stage = smem + C::OffQ + (two ? wg * C::Q_BYTES : wg * 16384) + quad * 4096;
                const uint64_t out_at = reinterpret_cast<uint64_t>(out);
                const int rows_here = min(32, r.rows - (row - lane));
#pragma unroll 1
                for (int c = c_lo; c < c_hi; c += 32) {
                    float o[32];
                    tmem_ld32(o0 + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] *= f0;
                    if (both) {
                        float x[32];
                        tmem_ld32(o1 + c, x);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = fmaf(x[e], f1, o[e]);
                    }
                    if (skip) continue;
                    __syncwarp();
                    if (sums == nullptr) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            *reinterpret_cast<uint4 *>(stage + lane * 64 + ((e ^ (lane >> 1 & 3)) << 4)) =
                                make_uint4(pack_bf16(o[8 * e], o[8 * e + 1]), pack_bf16(o[8 * e + 2], o[8 * e + 3]),
                                           pack_bf16(o[8 * e + 4], o[8 * e + 5]), pack_bf16(o[8 * e + 6], o[8 * e + 7]));
                        __syncwarp();
                        for (int i = 0; i < rows_here; i += 8) {
                            const int rr = i + (lane >> 2);
                            uint8_t *to = reinterpret_cast<uint8_t *>(__shfl_sync(0xffffffffu, out_at, rr)) + c * 2 + (lane & 3) * 16;
                            const uint4 x = *reinterpret_cast<const uint4 *>(stage + rr * 64 + (((lane & 3) ^ (rr >> 1 & 3)) << 4));
                            if (rr < rows_here) *reinterpret_cast<uint4 *>(to) = x;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            *reinterpret_cast<float4 *>(stage + lane * 128 + ((e ^ (lane & 7)) << 4)) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        __syncwarp();
                        for (int i = 0; i < rows_here; i += 4) {
                            const int rr = i + (lane >> 3);
                            const uint4 x = *reinterpret_cast<const uint4 *>(stage + rr * 128 + (((lane & 7) ^ (rr & 7)) << 4));
                            if (rr < rows_here) *reinterpret_cast<uint4 *>(sums + size_t(row - lane + rr) * D + c + (lane & 7) * 4) = x;
                        }
                    }
                }
                __syncwarp();
                if (mend && write) {
                    // draft values that are not finite, of the nodes that this row attends, go on top of what was written
                    const int lo = r.t0 < r.ct ? 0 : (r.t0 - r.ct) * N, hi = (r.t1 - r.ct) * N;
                    for (int a = node; a >= lo; a = p.parent != nullptr ? int(par[a]) : a - 1)
                        if (a < hi) {
                            const __nv_bfloat16 *v = p.v + ((size_t(r.l) * p.T + r.base + a) * p.HK + r.hk) * D;
#pragma unroll 1
                            for (int c = c_lo; c < c_hi; ++c) {
                                const float x = __bfloat162float(v[c]);
                                if (isfinite(x)) continue;
                                if (sums == nullptr) out[c] = __float2bfloat16_rn(__bfloat162float(out[c]) + x);
                                else sums[size_t(row) * D + c] += x;
                            }
                        }
                }
                if (sums != nullptr) {
                    float *tail = sums + size_t(plan.rows_cap) * D;
                    if (row < r.rows && c_lo == 0) reinterpret_cast<float2 *>(tail)[row] = make_float2(mm, ll);
                    if (row == 0 && c_lo == 0) reinterpret_cast<int *>(tail + 2 * plan.rows_cap)[0] = skip;
                }
            }
            tc_fence_before();
        }
    }

    if (warp == SOFT + 1 || warp == SOFT + 2) {
        // everything these warps issued must have completed before TMEM is released
        mma_commit(bar(C::kDrain), lead);
        mbar_wait(bar(C::kDrain), 0, abort_flag);
    }
    if ((warp == SOFT || warp == SOFT + 5) && *abort_flag) {
        // let copies still in flight land before the CTA's shared memory goes away
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) x.refuse();
    if (warp == SOFT + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Units that several CTAs have a piece of: a warp some rows at a time, pieces in order, so that the result does not depend on
// which CTA was ready first.  No more blocks than fit at once, and the sums of several rows and pieces asked for together: it is
// round trips to L2 that this takes (a block for every eight rows of every CTA, six waves of them, took 20 us behind 141 of
// prompt chunks).  FEW: units of few rows, which are few units if they are cut at all, and then into many pieces; larger ones
// are cut into two or three.
// ---------------------------------------------------------------------------------------------------------------
constexpr int kJoinWarps = 8, kJoinBlocks = 4;               // blocks a CTA of the other kernel at most

template <int D, bool FEW>
__global__ void __launch_bounds__(kJoinWarps * 32, kJoinBlocks)
join_kernel(AttnParams p, Plan plan, int32_t blocks)
{
    after_previous_kernel();
    constexpr int E = D / 32, PARTS = !FEW ? 2 : D == 256 ? 4 : 8, ROWS = FEW ? 1 : D == 256 ? 2 : 4;   // asked for together
    const int cta = blockIdx.x / blocks, lane = threadIdx.x & 31;
    const Join j = plan.join[cta];
    if (j.parts <= 1) return;
    const float c2 = p.scale * 1.4426950408889634f;
    const int group = p.H / p.HK, step = blocks * kJoinWarps;
    auto part = [&](int i) { return slot_sums(plan, cta + i, i == 0 ? 1 : 0); };
#pragma unroll 1
    for (int first = (blockIdx.x % blocks) * kJoinWarps + (threadIdx.x >> 5); first < j.rows; first += ROWS * step) {
        float o[ROWS][E], l[ROWS], m[ROWS];
        int skip = 0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            l[r] = 0.f;
            m[r] = -INFINITY;
#pragma unroll
            for (int e = 0; e < E; ++e) o[r][e] = 0.f;
        }
#pragma unroll 1
        for (int i0 = 0; i0 < j.parts; i0 += PARTS) {
            float2 ml = make_float2(-INFINITY, 0.f);         // lane r * PARTS + i: of part i of row r
            float x[ROWS][PARTS][E];
            if (lane < ROWS * PARTS && i0 + lane % PARTS < j.parts) {
                const float *tail = part(i0 + lane % PARTS) + size_t(plan.rows_cap) * D;
                const int row = first + lane / PARTS * step;
                if (row < j.rows) ml = reinterpret_cast<const float2 *>(tail)[row];
                skip |= reinterpret_cast<const int *>(tail + 2 * plan.rows_cap)[0];
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[r][i][e] = 0.f;
                    if (i0 + i < j.parts && first + r * step < j.rows) {
                        const float *at = part(i0 + i) + size_t(first + r * step) * D + lane * E;
                        if constexpr (E == 2) *reinterpret_cast<float2 *>(x[r][i]) = *reinterpret_cast<const float2 *>(at);
                        else
#pragma unroll
                            for (int e = 0; e < E; e += 4) *reinterpret_cast<float4 *>(x[r][i] + e) = *reinterpret_cast<const float4 *>(at + e);
                    }
                }
            float top = ml.x;
#pragma unroll
            for (int w = PARTS / 2; w > 0; w /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float now = fmaxf(m[r], __shfl_sync(0xffffffffu, top, r * PARTS));
                // (what has nothing yet is zero in whatever scale)
                const float old = m[r] == now || m[r] == -INFINITY ? 1.f : exp2_approx((m[r] - now) * c2);
                m[r] = now;
                l[r] *= old;
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= old;
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    const float mi = __shfl_sync(0xffffffffu, ml.x, r * PARTS + i), li = __shfl_sync(0xffffffffu, ml.y, r * PARTS + i);
                    const float f = mi == now || mi == -INFINITY ? 1.f : exp2_approx((mi - now) * c2);
                    l[r] = fmaf(li, f, l[r]);
#pragma unroll
                    for (int e = 0; e < E; ++e) o[r][e] = fmaf(x[r][i][e], f, o[r][e]);
                }
            }
        }
        if (__any_sync(0xffffffffu, skip)) return;           // (the same for every row)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (first + r * step >= j.rows) break;
            const int at = j.row0 + first + r * step, node = at / group, g = at - node * group;
            __nv_bfloat16 *to = p.o + ((size_t(j.l) * p.T + j.base + node) * p.H + j.hk * group + g) * D + lane * E;
            const float inv = 1.f / l[r];
            uint32_t y[E / 2];
#pragma unroll
            for (int e = 0; e < E; e += 2) y[e / 2] = pack_bf16(o[r][e] * inv, o[r][e + 1] * inv);
            if constexpr (E == 2) *reinterpret_cast<uint32_t *>(to) = y[0];
            else if constexpr (E == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(y[0], y[1]);
            else *reinterpret_cast<uint4 *>(to) = make_uint4(y[0], y[1], y[2], y[3]);
        }
    }
}

// rows of a unit at most
inline int unit_rows(int max_nodes, int group, int d)
{
    const long rows = long(max_nodes) * group;
    const int few = attend_few_rows(rows), mt = few > 0 ? few : d == 256 ? Cfg<256, true>::MT : Cfg<128, true>::MT;
    return rows < mt ? int(rows) : mt;
}

std::atomic<bool> g_opted_in[64];                            // per device: shared memory of every instantiation

int opt_in()
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return int(cudaErrorInvalidDevice);
    if (g_opted_in[dev].load(std::memory_order_acquire)) return 0;
    cudaError_t e = cudaSuccess;
    auto one = [&](const void *k, int bytes) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    };
    one(reinterpret_cast<const void *>(attend_kernel<64, false>), Cfg<64, false>::Bytes);
    one(reinterpret_cast<const void *>(attend_kernel<64, true>), Cfg<64, true>::Bytes);
    one(reinterpret_cast<const void *>(attend_kernel<128, false>), Cfg<128, false>::Bytes);
    one(reinterpret_cast<const void *>(attend_kernel<128, true>), Cfg<128, true>::Bytes);
    one(reinterpret_cast<const void *>(attend_kernel<256, true>), Cfg<256, true>::Bytes);
    if (e == cudaSuccess) g_opted_in[dev].store(true, std::memory_order_release);
    return int(e);
}

template <int D> int launch_width(const AttnParams &p, cudaStream_t st)
{
    const int sms = sm_count_of_current_device();
    if (sms <= 0) return int(cudaErrorInvalidDevice);
    const int rows_cap = unit_rows(p.max_nodes, p.H / p.HK, D), page = 1 << p.page_shift, grid = sms < kMaxCtas ? sms : kMaxCtas;
    const Plan plan = make_plan(p, rows_cap, D);
    Maps maps;
    // `keys` a tile: a box of the cache is a page, or a tile's part of one
    auto go = [&](int keys, auto launch_it) {
        const int box_rows = page < keys ? page : keys, rc = encode_maps<D>(p, box_rows, maps);
        return rc != 0 ? rc : launch_it(box_rows);
    };
    int e = opt_in();
    if (e != 0) return e;
    // whether no unit can be cut, as far as the host can tell: the table holds too little
    bool whole;
    auto never_cut = [&](int keys, int most, int weight) {
        return ((long(p.max_pages) * page + keys - 1) / keys + (p.max_nodes + keys - 1) / keys) * weight <= most;
    };
    if (attend_few_rows(long(p.max_nodes) * (p.H / p.HK)) > 0) {
        whole = never_cut(D == 256 ? 64 : 128, kFewWhole, 1);
        e = go(D == 256 ? 64 : 128, [&](int box) { return launch_attend_few(p, D, maps, plan, box, grid, st); });
    } else if (D == 256 || rows_cap > 128) {
        using C = Cfg<D, true>;
        whole = never_cut(C::N, C::kWhole, C::MT == 256 ? 2 : 1);
        e = go(C::N, [&](int box) {
            launch(attend_kernel<D, true>, grid, C::THREADS, C::Bytes, st, maps, p, plan, int32_t(box));
            return int(cudaGetLastError());
        });
    } else {
        using C = Cfg<D == 256 ? 128 : D, false>;            // (D = 256 went above)
        whole = never_cut(C::N, C::kWhole, 1);
        e = go(C::N, [&](int box) {
            launch(attend_kernel<C::D, false>, grid, C::THREADS, C::Bytes, st, maps, p, plan, int32_t(box));
            return int(cudaGetLastError());
        });
    }
    if (e != 0 || whole) return e;                           // 2.5 us for a join that finds nothing to do
    const int needed = (rows_cap + kJoinWarps - 1) / kJoinWarps, blocks = needed < kJoinBlocks ? needed : kJoinBlocks;
    if (rows_cap <= 16) launch(join_kernel<D, true>, unsigned(grid * blocks), kJoinWarps * 32, 0, st, p, plan, int32_t(blocks));
    else launch(join_kernel<D, false>, unsigned(grid * blocks), kJoinWarps * 32, 0, st, p, plan, int32_t(blocks));
    return int(cudaGetLastError());
}

}  // namespace

size_t attend_workspace_bytes(const speca_attn_dims *d)
{
    return align256(sizeof(Join) * kMaxCtas) + 2 * kMaxCtas * slot_bytes(unit_rows(d->max_nodes, d->heads / d->kv_heads, d->d_head), d->d_head);
}

static int g_withhold_first_load = 0, g_misplaced = 0;
void attend_set_withhold(int on) { g_withhold_first_load = on; }
void attend_set_misplaced(int on) { g_misplaced = on; }

int launch_attend(const AttnParams &call, int d_head, cudaStream_t st)
{
    AttnParams p = call;
    p.withhold_first_load = g_withhold_first_load;
    p.misplaced = g_misplaced;
    if (d_head == 64) return launch_width<64>(p, st);
    if (d_head == 128) return launch_width<128>(p, st);
    return launch_width<256>(p, st);
}

}  // namespace speca
