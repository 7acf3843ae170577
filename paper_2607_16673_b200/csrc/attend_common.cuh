// What the attention kernels share: the list of work and its equal pieces, the warp that schedules a CTA's piece, the warp that
// brings keys and values in.
#pragma once

#include "attn.cuh"
#include "tc_ptx.cuh"

namespace speca {
namespace attend {

using namespace tc;

constexpr int kMaxCtas = 160;            // pieces of the list at most (148 SMs)
constexpr int kRecords = 4;              // ring of segment records
constexpr int kFlagRing = 8;
constexpr int kFewWhole = 4;             // tiles of a unit of few rows that is never cut (6 chains behind 10..300 tokens 17.9 -> 15.4 us)

// A piece of one unit: key tiles t0 .. t1-1, of which the first `ct` of the unit are the cache's.
struct Rec {
    int l, b, hk, base;
    int n, len, row0, rows;
    int t0, t1, ct, nodes;                                   // nodes: draft nodes the unit's rows can see (0 .. nodes-1)
    int slot, pad0, pad1, pad2;                              // slot: -1 the whole unit, 0 / 1 where its sums go
};
static_assert(sizeof(Rec) == 64, "record");

// Joining: what a CTA's unit that goes on in the next CTAs needs.
struct Join {
    int parts, l, hk, base;
    int row0, rows, pad0, pad1;
};

struct Plan {
    int rows_cap;                                            // rows of a slot
    size_t slot_bytes;
    Join *join;
    char *slots;
};

__host__ __device__ inline size_t slot_bytes(int rows, int d) { return align256(size_t(rows) * d * 4 + size_t(rows) * 8 + 16); }

__device__ __forceinline__ float *slot_sums(const Plan &pl, int cta, int slot)
{
    return reinterpret_cast<float *>(pl.slots + (size_t(cta) * 2 + slot) * pl.slot_bytes);
}

// A tile of keys or values in shared memory: groups of eight rows, in a group one 64-wide block of columns behind the other,
// in a block eight rows of 128 bytes with the 128-byte swizzle.  So one copy brings a page whatever its width (with the blocks
// outermost it takes one a block, and 32 copies a tile of 16-row pages and 128 columns took longer than the tile's bytes).
template <int D> __device__ __forceinline__ uint32_t tile_offset(int row, int chunk)       // of 16 bytes
{
    return uint32_t((row >> 3) * (D / 64) + (chunk >> 3)) * 1024u + (row & 7) * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}
// as tma_load_3d, by the lane that has `lead` set
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar, uint32_t lead)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %7, 0;\n\t"
        "@q cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, int v, uint32_t bar, uint32_t lead)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %8, 0;\n\t"
        "@q cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];\n\t}"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "r"(bar), "r"(lead)
        : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 16 bytes from global to shared memory, none of a thread's copies waits for another
__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ bool not_finite(uint32_t pair)
{
    return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u;
}

// ---------------------------------------------------------------------------------------------------------------
// The list of tiles
// ---------------------------------------------------------------------------------------------------------------
// Query heads to a key head, and quotients of numbers >= 0 by them without a division (some forty instructions, and a prompt's
// list takes hundreds): the inverse is rounded up, so the product's high half is the quotient or one more.
struct Group {
    int n;
    uint32_t inverse;
    __device__ __forceinline__ explicit Group(int heads) : n(heads), inverse(heads > 1 ? 0xffffffffu / uint32_t(heads) + 1u : 0u) {}
    __device__ __forceinline__ int over(int y) const
    {
        if (n == 1) return y;
        const int q = int(__umulhi(uint32_t(y), inverse));
        return q - (q * n > y);
    }
};

struct Seq {
    int base, n, len, ct, fault;
};

template <class C> __device__ __forceinline__ Seq sequence(const AttnParams &p, int b)
{
    Seq s;
    s.fault = sequence_nodes(p, b, s.base, s.n);
    s.len = p.kv_len[b];
    if (s.len < 0 || (s.len >> p.page_shift) > p.max_pages || s.len > p.max_pages << p.page_shift) s.fault |= SPECA_STATUS_BAD_PAGE;
    if (s.fault) s.n = 0;
    s.ct = s.fault ? 0 : int((uint32_t(s.len) + C::N - 1) / C::N);           // (lengths go up to 2^31 - 1)
    return s;
}
// draft nodes that the rows of row tile m can see
template <int MT> __device__ __forceinline__ int nodes_seen(int n, const Group &group, int m)
{
    return min(n, group.over((m + 1) * MT - 1) + 1);
}
template <class C> __device__ __forceinline__ long unit_tiles(const Seq &s, const Group &group, int m)
{
    return s.ct + (nodes_seen<C::MT>(s.n, group, m) + C::N - 1) / C::N;
}
// Cost of a unit, in tiles: its own (twice as many where two row tiles share the keys) and what begins and ends it, queries in,
// sums out, the pipeline filled and drained.  Pieces are equal in this measure: with tiles alone counted, CTAs that got many
// short sequences took up to twice as long as the others.
template <class C> __device__ __forceinline__ int tile_cost(const Seq &s, const Group &group, int m)
{
    return C::MT == 256 && s.n * group.n - m * C::MT > 128 ? 2 : 1;
}
template <class C> __device__ __forceinline__ long unit_cost(const Seq &s, const Group &group, int m)
{
    return unit_tiles<C>(s, group, m) * tile_cost<C>(s, group, m) + C::kEnds;
}
template <class C> __device__ __forceinline__ int row_tiles(const Seq &s, const Group &group)
{
    return (s.n * group.n + C::MT - 1) / C::MT;             // (at most 8192 nodes and 4096 heads)
}
template <class C> __device__ __forceinline__ int longest_unit(const Seq &s, const Group &group)
{
    // (the last full row tile sees most)
    const int tiles = s.ct + (s.n + C::N - 1) / C::N;
    return tiles * (C::MT == 256 && s.n * group.n > 128 ? 2 : 1);
}
// cost of one layer and key head
template <class C> __device__ __forceinline__ long head_cost(const Seq &s, const Group &group)
{
    long sum = 0;
    const int tiles = row_tiles<C>(s, group);
    for (int m = 0; m < tiles; ++m) sum += unit_cost<C>(s, group, m);
    return sum;
}

// a / b of positive numbers: a division of 64 bits is a call of some hundred instructions, in front of the first tile
__device__ __forceinline__ long quotient(long a, long b)
{
    return ((a | b) >> 31) == 0 ? long(uint32_t(a) / uint32_t(b)) : a / b;
}

struct Maps {
    CUtensorMap k, v, k_draft, v_draft;
};

// A CTA's view of the work.  C: N keys a tile, D columns, MT rows of a unit, kEnds, kPiece and kWhole of the schedule, KS and VS
// slots of TILE bytes at OffRing (keys, then values), barriers from OffBars.
// (A barrier has two parities: whoever waits on one waits for all its phases in turn.  So keys and values have rings of their
// own, and where C::kMend, values that are looked over before they are used land on barriers of their own.)
template <class C> struct Cta {
    static constexpr int N = C::N, D = C::D, KS = C::KS, VS = C::VS;
    const AttnParams &p;
    const Plan &plan;
    uint8_t *smem;
    uint32_t sbase;
    int warp, lane;
    Group group;
    volatile int *abort_flag, *topo_bad, *page_bad, *value_bad;      // topo_bad [2], the others [kFlagRing]: 1 + segment number
    uint32_t lead;
    bool ok;

    __device__ __forceinline__ Cta(const AttnParams &p_, const Plan &plan_, uint8_t *smem_)
        : p(p_), plan(plan_), smem(smem_), sbase(smem_u32(smem_)), warp(threadIdx.x >> 5), lane(threadIdx.x & 31), group(p_.H / p_.HK),
          abort_flag(reinterpret_cast<volatile int *>(smem_ + C::OffMisc)), topo_bad(abort_flag + 2),
          page_bad(reinterpret_cast<volatile int *>(smem_ + C::OffFlags)), value_bad(page_bad + kFlagRing), ok(true)
    {
    }
    __device__ __forceinline__ uint32_t bar(int i) const { return sbase + C::OffBars + 8u * uint32_t(i); }
    // This CTA gives up: said in the status, and nothing of it is joined (what stands in the workspace is not a record of this call).
    __device__ __forceinline__ void refuse() const
    {
        if (threadIdx.x != 0) return;
        atomicOr(p.status, SPECA_STATUS_TIMEOUT);
        plan.join[blockIdx.x].parts = 0;
    }
    // by the first warp, before the barriers' fence
    __device__ __forceinline__ void init(int consumers, int empties)
    {
        if (lane == 0) *abort_flag = topo_bad[0] = topo_bad[1] = 0;
        if (lane < 2 * kFlagRing) page_bad[lane] = 0;
        if (lane < KS) { mbar_init(bar(C::kKFull + lane), 1); mbar_init(bar(C::kKEmpty + lane), empties); }
        if (lane < VS) { mbar_init(bar(C::kVFull + lane), 1); mbar_init(bar(C::kVEmpty + lane), empties); }
        if (lane < kRecords) { mbar_init(bar(C::kRecFull + lane), 1); mbar_init(bar(C::kRecEmpty + lane), consumers); }
    }

    // record of segment `s`; false: the list has ended, or (ok == false) the CTA is aborting
    __device__ __forceinline__ bool record(uint32_t s, Rec &r)
    {
        if (!(ok = wait_fast(bar(C::kRecFull + (s % kRecords)), (s / kRecords) & 1, abort_flag))) return false;
        const int4 *src = reinterpret_cast<const int4 *>(smem + C::OffRec) + 4 * (s % kRecords);
        const int4 a = src[0], b = src[1], c = src[2], d = src[3];
        r = Rec{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, c.y, c.z, c.w, d.x, 0, 0, 0};
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::kRecEmpty + (s % kRecords)));
        return r.rows > 0;
    }
    // rows of tile t that hold keys
    __device__ __forceinline__ int valid_of(const Rec &r, int t) const
    {
        const int left = t < r.ct ? r.len - t * N : r.nodes - (t - r.ct) * N;
        return left < N ? left : N;
    }
    // whether every row of the unit attends all keys of tile t (of a chain's draft those below its first node)
    __device__ __forceinline__ bool all_seen(const Rec &r, int t) const
    {
        return t < r.ct || (p.parent == nullptr && (t - r.ct + 1) * N <= group.over(r.row0) + 1);
    }
    __device__ __forceinline__ bool to_mend(const Rec &r, int t) const
    {
        return C::kMend && ((valid_of(r, t) & 15) != 0 || !all_seen(r, t));
    }

    // barriers and flags are set up; whole CTA
    __device__ __forceinline__ void begin()
    {
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        lead = elect_one();
    }

    // Keys (KV = 0) or values (KV = 1) into their ring, one warp each: a copy of a page of 16 rows is 220 cycles of its warp, so
    // that one warp for both took longer over a tile of such pages than its bytes do.
    template <int KV> __device__ __forceinline__ void load(const Maps &maps, int box_rows)
    {
        constexpr int SLOTS = KV ? VS : KS;
        const CUtensorMap *const map = KV ? &maps.v : &maps.k, *const draft = KV ? &maps.v_draft : &maps.k_draft;
        Rec r;
        uint32_t n = 0;
        for (uint32_t seg = 0; ok && record(seg, r); ++seg) {
            const int32_t *table = p.page_table + size_t(r.b) * p.max_pages;
            const int pages = int((uint32_t(r.len) + (1u << p.page_shift) - 1u) >> p.page_shift);
            int window = r.t0 < r.ct ? (r.t0 * N) >> p.page_shift : 0;        // 32 entries of the table, one a lane, and the 32 behind them
            auto entries = [&](int first) { return r.t0 < r.ct && first + lane < pages ? table[first + lane] : 0; };
            int ids = entries(window), next = entries(window + 32);
#pragma unroll 1
            for (int t = r.t0; t < r.t1; ++t, ++n) {
                int at = 0;                                  // this lane's page of the tile, as a row of the map
                if (t < r.ct) {
                    const int page = int((uint32_t(t * N) + uint32_t(lane * box_rows)) >> p.page_shift), first = (t * N) >> p.page_shift;
                    if (first >= window + 32) {
                        window = first;
                        ids = next;
                        next = entries(window + 32);
                    }
                    int id = __shfl_sync(0xffffffffu, ids, (page - window) & 31);
                    if (lane * box_rows < valid_of(r, t) && (id < 0 || id >= p.n_pages)) {
                        id = 0;                              // read what is there, and leave the unit's outputs alone
                        page_bad[seg % kFlagRing] = int(seg) + 1;
                        atomicOr(p.status, SPECA_STATUS_BAD_PAGE);
                    }
                    at = (r.l * p.n_pages + id) * p.HK + r.hk;
                }
                const int s = n % SLOTS;
                if (!(ok = wait_fast(bar((KV ? C::kVEmpty : C::kKEmpty) + s), ((n / SLOTS) & 1) ^ 1, abort_flag))) break;
                if (KV == 0 && n == 0 && p.withhold_first_load && blockIdx.x == 0) continue;
                const int valid = valid_of(r, t);
                const uint32_t full = bar((KV == 0 ? C::kKFull : to_mend(r, t) ? C::kVRaw : C::kVFull) + s);
                const uint32_t dst = sbase + C::OffRing + (KV ? KS + s : s) * C::TILE;
                if (t >= r.ct) {
                    const int boxes = (valid + 7) / 8, row = r.l * p.T + r.base + (t - r.ct) * N;
                    if (lead) mbar_arrive_expect_tx(full, uint32_t(boxes) * (8 * D * 2));
                    __syncwarp();
#pragma unroll 1
                    for (int j = 0; j < boxes; ++j) tma_load_4d(dst + j * (8 * D * 2), draft, 0, row + 8 * j, 0, r.hk, full, lead);
                } else {
                    const int boxes = (valid + box_rows - 1) / box_rows, rows = ((t * N) & ((1 << p.page_shift) - 1)) >> 3;
                    if (lead) mbar_arrive_expect_tx(full, uint32_t(boxes) * box_rows * (D * 2));
                    __syncwarp();
#pragma unroll 1
                    for (int j = 0; j < boxes; ++j)
                        tma_load_5d(dst + j * box_rows * (D * 2), map, 0, 0, 0, rows, __shfl_sync(0xffffffffu, at, j), full, lead);
                }
            }
        }
    }

    // Cost of the whole list, this CTA's piece of it, its records and what the join needs of it; one warp, the others only wait for
    // its first record (with all of them adding up sequences and two barriers it came 1.5 us later, most of it instructions
    // fetched for the first time).
    __device__ __forceinline__ void schedule()
    {
        const int grid = gridDim.x, cta = blockIdx.x;
        const int heads = p.L * p.HK;
        Join join{0, 0, 0, 0, 0, 0, 0, 0};
        uint32_t seg = 0;
        auto put = [&](const Rec &x) {
            // the unit's queries are asked into L2 while the segments before it are worked on
            for (int node = group.over(x.row0) + lane; node * group.n < x.row0 + x.rows; node += 32)
                prefetch_l2(p.q + ((size_t(x.l) * p.T + x.base + node) * p.H + x.hk * group.n) * D, uint32_t(group.n) * D * 2);
            ok = seg < kRecords || wait_fast(bar(C::kRecEmpty + (seg % kRecords)), ((seg / kRecords) & 1) ^ 1, abort_flag);
            if (!ok) return;
            if (lane == 0) {
                *reinterpret_cast<Rec *>(smem + C::OffRec + 64 * (seg % kRecords)) = x;
                mbar_arrive(bar(C::kRecFull + (seg % kRecords)));
            }
            __syncwarp();
            ++seg;
        };
        // 32 sequences at a time, one a lane: the cost of one layer and key head of each
        Seq s{};
        auto fetch = [&](int b0) {
            s = Seq{0, 0, 0, 0, 0};
            if (b0 + lane >= p.B) return 0L;
            s = sequence<C>(p, b0 + lane);
            return head_cost<C>(s, group);
        };
        long total = 0, first = 0;
        int longest = 0;                                     // unit, its ends aside
#pragma unroll 1
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const long c = fetch(b0);
            if (b0 == 0) first = c;
            if (s.fault && cta == 0) atomicOr(p.status, s.fault);
            total += c;
            if (c > 0) longest = max(longest, longest_unit<C>(s, group));
        }
        longest = int(__reduce_max_sync(0xffffffffu, unsigned(longest)));
#pragma unroll
        for (int i = 16; i > 0; i /= 2) total += __shfl_xor_sync(0xffffffffu, total, i);
        total *= heads;
        // A piece is at least kPiece long: at least one tile, so that every CTA between a unit's first and last has some of it, and
        // more where rows make their joining dear.  Units of up to kWhole are not cut at all, but go to the CTA in whose piece they
        // begin.
        const bool whole = longest <= C::kWhole;
        const int pieces = int(min(long(grid), max(1L, total / C::kPiece)));
        const long per = quotient(total, pieces), extra = total - per * pieces;
        const long begin = cta * per + min(long(cta), extra), end = cta < pieces ? begin + per + (cta < extra ? 1 : 0) : begin;
        long at = 0;                                         // place in the list of the sequence looked at
#pragma unroll 1
        for (int b0 = 0; b0 < p.B && at < end && ok; b0 += 32) {
            const long mine = p.B <= 32 ? first : fetch(b0);
            long upto = mine * heads;                        // to the end of this lane's sequence, from the first of the 32
#pragma unroll
            for (int i = 1; i < 32; i *= 2) {
                const long y = __shfl_up_sync(0xffffffffu, upto, i);
                if (lane >= i) upto += y;
            }
            const uint32_t later = __ballot_sync(0xffffffffu, at + upto > begin);
            const int from = later != 0u ? __ffs(int(later)) - 1 : 32;           // the first that reaches into the piece
            at += __shfl_sync(0xffffffffu, from > 0 ? upto : 0L, from > 0 ? from - 1 : 0);
#pragma unroll 1
            for (int i = from; i < 32 && b0 + i < p.B && at < end && ok; ++i) {
                const long hc = __shfl_sync(0xffffffffu, mine, i);
                if (hc == 0) continue;
                Seq q;
                q.base = __shfl_sync(0xffffffffu, s.base, i);
                q.n = __shfl_sync(0xffffffffu, s.n, i);
                q.len = __shfl_sync(0xffffffffu, s.len, i);
                q.ct = __shfl_sync(0xffffffffu, s.ct, i);
                const int mts = row_tiles<C>(q, group);
                int hd = 0;
                if (at < begin) {
                    hd = int(quotient(begin - at, hc));
                    at += hd * hc;
                }
#pragma unroll 1
                for (; hd < heads && at < end && ok; ++hd)
#pragma unroll 1
                    for (int m = 0; m < mts && at < end && ok; ++m) {
                        const int ut = int(unit_tiles<C>(q, group, m)), w = tile_cost<C>(q, group, m);
                        const long tiles_at = at + C::kEnds;                     // the unit's ends stand before its tiles
                        at = tiles_at + long(ut) * w;
                        if (at <= begin) continue;
                        // a tile is whose piece its beginning is in
                        auto tile_from = [&](long x) { return x <= tiles_at ? 0 : int(min(long(ut), (x - tiles_at + w - 1) >> (w - 1))); };
                        Rec x{};
                        const bool own = tiles_at - C::kEnds >= begin;           // (it is before the end)
                        x.t0 = whole ? 0 : tile_from(begin);
                        x.t1 = whole ? (own ? ut : 0) : tile_from(end);
                        if (x.t1 <= x.t0) continue;
                        x.l = hd / p.HK; x.b = b0 + i; x.hk = hd - x.l * p.HK; x.base = q.base; x.n = q.n; x.len = q.len;
                        x.row0 = m * C::MT;
                        x.rows = min(C::MT, q.n * group.n - x.row0);
                        x.ct = q.ct;
                        x.nodes = nodes_seen<C::MT>(q.n, group, m);
                        x.slot = x.t0 == 0 && x.t1 == ut ? -1 : x.t0 == 0 ? 1 : 0;
                        put(x);
                        if (x.slot == 1) {
                            // the unit ends in a later CTA's piece: where its last tile begins
                            const long last = tiles_at + long(ut - 1) * w, wide = extra * (per + 1);
                            const int owner = int(last < wide ? quotient(last, per + 1) : extra + quotient(last - wide, per));
                            join = Join{owner - cta + 1, x.l, x.hk, x.base, x.row0, x.rows, 0, 0};
                        }
                    }
                if (hd < heads) break;
            }
        }
        if (ok) put(Rec{});
        if (lane == 0) {
            if (!ok) join.parts = 0;
            plan.join[cta] = join;
        }
    }
};

// Barrier of `THREADS` threads' worth of warps, and whether all of them are well: a warp whose wait gave up comes to the next one
// once more, and all leave there together.  (An mbarrier that all arrive and wait on did the same in 250 ns; a segment has
// three to six.)
template <int THREADS> __device__ __forceinline__ bool all_well(bool ok)
{
    uint32_t r;
    __syncwarp();
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 q, %1, 0;\n\t"
        "bar.red.and.pred p, 1, %2, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(uint32_t(ok)), "n"(THREADS)
        : "memory");
    return r != 0u;
}

// the four maps of a call (a box of the cache is a page, or a tile's rows of one); 0 or an error
template <int D> inline int encode_maps(const AttnParams &p, int box_rows, Maps &maps)
{
    EncodeTiledFn encode = encode_tiled_fn();
    if (encode == nullptr) return int(cudaErrorNotSupported);
    const int page = 1 << p.page_shift;
    CUtensorMap *to[4] = {&maps.k, &maps.v, &maps.k_draft, &maps.v_draft};
    const cuuint32_t es[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < 4; ++i) {
        const bool cache = i < 2;
        const void *base = i == 0 ? p.k_cache : i == 1 ? p.v_cache : i == 2 ? p.k : p.v;
        // 64 columns, eight rows, blocks of columns; of the cache groups of eight rows and (layer, page, head) besides, of the
        // draft rows of all layers in place of the eight, and the head
        const cuuint64_t row = cuuint64_t(D) * 2 * (cache ? 1 : p.HK);
        const cuuint64_t dim[5] = {64, cache ? 8u : cuuint64_t(p.L) * p.T, D / 64, cuuint64_t(cache ? page / 8 : p.HK), cuuint64_t(p.L) * p.n_pages * p.HK};
        const cuuint64_t stride[4] = {row, 128, cache ? 8 * row : cuuint64_t(D) * 2, cuuint64_t(page) * D * 2};
        const cuuint32_t box[5] = {64, 8, D / 64, cuuint32_t(cache ? box_rows / 8 : 1), 1};
        if (encode(to[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, cache ? 5 : 4, const_cast<void *>(base), dim, stride, box, es,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return int(cudaErrorInvalidValue);
    }
    return 0;
}

inline Plan make_plan(const AttnParams &p, int rows_cap, int d)
{
    Plan plan;
    plan.rows_cap = rows_cap;
    plan.slot_bytes = slot_bytes(rows_cap, d);
    plan.join = static_cast<Join *>(p.workspace);
    plan.slots = static_cast<char *>(p.workspace) + align256(sizeof(Join) * kMaxCtas);
    return plan;
}

}  // namespace attend

// few rows a unit (max_nodes * heads / kv_heads of them at most): rows of its tile, or 0
int attend_few_rows(long rows);
int launch_attend_few(const AttnParams &p, int d_head, const attend::Maps &maps, const attend::Plan &plan, int box_rows, int grid,
                      cudaStream_t st);

}  // namespace speca
