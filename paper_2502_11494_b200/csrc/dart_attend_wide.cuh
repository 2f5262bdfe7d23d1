// Attention over the paged cache for many rows: tiles of 128 rows on the tensor cores (see dart_attend.cuh for the work's division
// and for how pieces are joined).
//
// A CTA has two ENGINES of a 128-row tile each: four softmax warps with a thread per row, 256 columns of tensor memory.  For each KV
// tile of 128 tokens an engine does
//   S = Q K^T   (Q and K in shared memory, 128-byte swizzle, S in tensor memory),
//   P = 2^(S scale - m), in the cache's type, written over S,
//   O += P V    (P from tensor memory, V as it lies in the cache: tokens along the product's inner dimension),
// so that one engine's products run while the other one takes exponentials: 1024 cycles of the tensor pipe and 1024 of the
// exponential unit a tile, the two that bound it.  O stays in tensor memory over a whole piece; it is only scaled when a
// row's maximum has grown by more than 2^8 since it was last (fp32 sums and 16-bit weights lose nothing by a common factor).
//   kPair false: the engines are two workers with a ring of tiles each (a place: keys or values of 128 tokens).
//   kPair true:  they are one worker, two row tiles, whose products one warp issues in turn: both multiply with the same KV tiles.  Half the
//                traffic from L2.
// Rows behind a sequence's end come from its last page as they are; their scores are left out by selection, and the values among
// the last 16 tokens of a product are set to zero in shared memory (0 * NaN would be NaN).
// What bounds it (128 columns, 256 rows, cycles of one KV tile): 2048 of the tensor pipe for both engines, 3800 measured: an engine's softmax takes
// 2000 from its scores to its weights (load 100, maximum 440, exponentials 1500), and what hands over between the warps 1300 more; the
// engines overlap, but not fully.  A piece's end takes some 10000 (its rows by way of shared memory, the next piece's queries and first scores).
// Tried and taken back: three of eight exponentials as polynomials on the FMA pipe (2600 instead of 1390), two threads a row (eight warps an
// engine: their meeting costs 1000), a warp per engine for the products (both engines fall into step, at the exponentials together and at the
// products together: 4600), the same with a turn for the exponentials (4150).
// Every wait is bounded in time; a kernel that gives up says so in the status word, waits for its own copies and products, frees
// the tensor memory and returns.
#pragma once
#include "dart_attend.cuh"
#include "dart_ptx.cuh"

namespace dart {
namespace attend {

using sweep::mbar_arrive;
using sweep::mbar_arrive_expect_tx;
using sweep::mbar_init;
using sweep::smem_u32;
using sweep::umma_commit;
using sweep::umma_desc;

constexpr int kWideRows = 128, kWideTile = 128, kWideThreads = 384, kWideCost = 3;
constexpr int kPieces = 4;                      // that may wait for the softmax threads
constexpr int kHalf = 16384;                    // bytes: 128 tokens (or rows) x 64 columns
constexpr int kWideSmem = 14 * kHalf + 1024;    // queries, the rings, 4 KB a softmax warp; the base is aligned to 1 KB
constexpr int kMaxPlaces = 10;
constexpr int kTmemCols = 512;
// which wait gave up (status[1])
enum { kWaitPlace = 110, kWaitKeys, kWaitValues, kWaitQueries, kWaitWeights, kWaitScores, kWaitSums, kWaitLastValues, kWaitPieces };

// A place's note: whether engine e has work with the tile (bit e), whether it is the piece's first (8) and engine e's last of the piece
// (bit 4 + e), how many 16-token steps its second product has (from bit 8); or that nothing follows.
constexpr uint32_t kNoteFirst = 8, kNoteLast = 16, kNoteEnd = 1u << 31;

// A piece as the softmax threads need it, written by the copying warp, which is ahead of them.
struct PieceNote {
    int a, b, vis, place;                  // tiles (b < 0: nothing follows); tokens that its last row sees; where its sums go: kToRows, or a
                                           // place among the workers'
    int hk, len, prefix;                   // KV head; tokens of the segment
    int n0[2], rows[2], tiles[2], sees[2]; // per engine: first packed row, rows, tiles, how many tokens its first row would see if len had no end
};
constexpr int kToRows = -1;

struct WideShared {
    PieceNote piece[2][kPieces];
    unsigned long long piece_full[2][kPieces], piece_empty[2][kPieces];
    unsigned long long full[2][kMaxPlaces], empty[2][kMaxPlaces];
    unsigned long long s_full[2], p_half[2], p_full[2], o_full[2], q_full[2], drain[2];
    uint32_t note[2][kMaxPlaces]; // what a place holds (kNote*), for the thread that issues the products
    uint32_t asked[2];            // query copies that an engine has begun so far
    uint32_t tmem;
    int abort;
    PlanShared<2> plan;
};

// The queries of whole tokens and one KV head: 64 columns of all its query heads and of as many tokens as a tile holds.
__device__ __forceinline__ void tma_queries(uint32_t dst, const CUtensorMap *tm, int x, int hk, int n, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(tm), "r"(x),
                 "r"(0), "r"(hk), "r"(n), "r"(bar)
                 : "memory");
}
// Bounded waits that sleep: the hardware wakes a waiting warp when the phase ends, or after the hint (in ns), when it looks whether the
// CTA has given up or its time is over.  (A warp that asks again and again takes issue slots from those that compute.)
constexpr uint32_t kSleepNs = 20000;
__device__ __forceinline__ bool asleep_until(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity), "r"(kSleepNs)
                 : "memory");
    return ok != 0;
}
struct Waits {
    sweep::Ctl ctl;
    // Rows that are not valid say more than a page that read as zeros: the status becomes TIMEOUT over CHECK too.
    __device__ void give_up(int where, long long task) const
    {
        *ctl.abort_flag = 1;
        int was = atomicCAS(ctl.status, 0, sweep::kStatusTimeout);
        if (was == kErrCheck && atomicCAS(ctl.status, kErrCheck, sweep::kStatusTimeout) == kErrCheck) was = 0;
        if (was == 0) ctl.status[1] = where, ctl.status[2] = (int)task, ctl.status[3] = (int)blockIdx.x;
    }
    __device__ bool wait_bar(uint32_t bar, uint32_t parity, int where, long long task) const
    {
        if (asleep_until(bar, parity)) return true;
        const long long t0 = clock64();
        while (!asleep_until(bar, parity)) {
            if (ctl.aborted()) return false;
            if ((unsigned long long)(clock64() - t0) > ctl.limit_cycles) {
                give_up(where, task);
                return false;
            }
        }
        return true;
    }
    __device__ void wait_landed(uint32_t bar, uint32_t parity) const { ctl.wait_landed(bar, parity); }
};
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap *tm, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(tm), "r"(x),
                 "r"(y), "r"(bar)
                 : "memory");
}
// D[128 x n] (+)= A[128 x 16] B[16 x n]; A and B of type T, D fp32.  b_mn: B's tokens run along the inner dimension (rows of 64 columns).
template <typename T>
constexpr uint32_t kFormat = 0; // fp16
template <>
constexpr uint32_t kFormat<__nv_bfloat16> = 1;
template <typename T>
__device__ __forceinline__ uint32_t wide_idesc(int n, bool b_mn)
{
    constexpr uint32_t fmt = kFormat<T>;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kWideRows >> 4) << 24);
}
__device__ __forceinline__ void umma_ss(uint32_t d, unsigned long long a, unsigned long long b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                 "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, unsigned long long b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b),
                 "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t at, float *v)
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
                 "%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
                   "=r"(r[31])
                 : "r"(at));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
                 "r"(r[15]), "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}

// An engine's part of a piece: its rows, and how many of the piece's tiles its last row sees anything of.
template <typename W>
__device__ __forceinline__ PieceNote piece_note(const Params &p, const W &w, int engines, int rows)
{
    PieceNote g;
    g.a = w.a, g.b = w.b, g.vis = w.vis, g.place = w.is_whole() ? kToRows : (int)w.place();
    g.hk = w.hk, g.len = w.g.len, g.prefix = w.g.prefix;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r0 = w.mb * p.pieces.M + e * rows, t0 = p.by_R.of(r0);
        g.n0[e] = w.g.row0 + t0;
        g.rows[e] = e < engines ? clamp(w.g.n_q * p.R - r0, 0, rows) : 0;
        const int vis = g.rows[e] == 0 ? 0 : sees(w.g, p.by_R.of(r0 + g.rows[e] - 1));
        g.tiles[e] = max(0, min(w.b, (vis + kWideTile - 1) / kWideTile) - w.a);
        g.sees[e] = w.g.prefix ? w.g.len : w.g.len - w.g.n_q + t0 + 1;
    }
    return g;
}

template <typename T, int D, bool kPair>
__global__ void __launch_bounds__(kWideThreads, 1)
    attend_wide_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                       const Params p, int *status,
                       unsigned long long limit_cycles, int withhold)
{
    constexpr int kHalves = D / 64, kWorkers = kPair ? 1 : 2;
    constexpr int kPlace = kHalves * kHalf;                              // bytes: the keys, or the values, of a tile
    constexpr int kPlaces = (12 - 2 * kHalves) / kHalves / kWorkers; // of a ring
    extern __shared__ unsigned char raw[];
    __shared__ WideShared sh;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rows = kPair ? p.pieces.M >> 1 : p.pieces.M; // of an engine: whole tokens, all of a KV head's query heads
    const auto q_at = [&](int e) { return base + (uint32_t)e * kPlace; };
    const auto place_at = [&](int ring, int i) { return base + (uint32_t)(2 + ring * kPlaces + i) * kPlace; };

    if (threadIdx.x == 0) {
        for (int r = 0; r < kWorkers; ++r)
            for (int i = 0; i < kPieces; ++i) {
                mbar_init(smem_u32(&sh.piece_full[r][i]), 1);
                mbar_init(smem_u32(&sh.piece_empty[r][i]), kPair ? 8 : 4);
            }
        for (int r = 0; r < kWorkers; ++r)
            for (int i = 0; i < kPlaces; ++i) {
                mbar_init(smem_u32(&sh.full[r][i]), 1);
                mbar_init(smem_u32(&sh.empty[r][i]), 1);
            }
        for (int e = 0; e < 2; ++e) {
            mbar_init(smem_u32(&sh.s_full[e]), 1);
            mbar_init(smem_u32(&sh.p_half[e]), 4);
            mbar_init(smem_u32(&sh.p_full[e]), 4);
            mbar_init(smem_u32(&sh.o_full[e]), 1);
            mbar_init(smem_u32(&sh.drain[e]), 1);
            mbar_init(smem_u32(&sh.q_full[e]), 1);
            sh.asked[e] = 0;
        }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh.tmem;
    wait_for_previous();
    plan<kWideTile, kWideCost, kWorkers>(p, *reinterpret_cast<PlanShared<kWorkers> *>(&sh.plan));
    const PlanShared<kWorkers> &pl = *reinterpret_cast<const PlanShared<kWorkers> *>(&sh.plan);
    const Waits ctl{{&sh.abort, status, limit_cycles}};

    // The softmax threads hold a row of 128 scores: 216 registers; the others give theirs (256 x 216 + 128 x 72 = 384 x 168).
    if (warp >= 8)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    else
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");

    if (warp >= 10) {
        // ------------------------------------------------------------------ copies: a lane per page
        // Two rings: a warp each.  One ring: a warp for the keys and one for the values (pages of 16 tokens are 16 copies a place, and a
        // warp takes 1300 cycles for them).
        {
            const int ring = kPair ? 0 : warp - 10, k0 = kPair ? warp - 10 : 0, k1 = kPair ? warp - 9 : 2;
            const bool first = k0 == 0;
            Walk<kWideTile, kWideCost> w{};
            w.begin(p, pl, ring);
            const int box = min(1 << p.page_shift, kWideTile), nowhere = (p.n_pages * p.Hk) << p.page_shift;
            uint32_t tiles = 0, pieces = 0, last = 0; // of the ring so far; the warp's newest copy + 1
            if (first && lane == 0) no_open_item(p, blockIdx.x * kWorkers + ring);
            bool ok = true;
            const auto announce = [&](const PieceNote &note) { // to the softmax threads
                const int at = (int)(pieces % kPieces);
                if (lane == 0) {
                    ok = ctl.wait_bar(smem_u32(&sh.piece_empty[ring][at]), ((pieces / kPieces) & 1u) ^ 1u, kWaitPieces, pieces);
                    if (ok) {
                        sh.piece[ring][at] = note;
                        mbar_arrive(smem_u32(&sh.piece_full[ring][at]));
                    }
                }
                ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                ++pieces;
            };
            for (; ok && !w.done; w.next(p)) {
                const PieceNote piece = piece_note(p, w, kPair ? 2 : 1, rows);
                if (first) {
                    if (lane == 0) {
                        w.note(p);
                        if (w.a == 0 && w.b < w.nt) open_item(p, w);
                    }
                    announce(piece);
                }
                if (!ok) break;
                const auto page_row = [&](int tile) { // where the lane's page of a tile begins among all rows of the cache
                    const int tok = tile * kWideTile + lane * box;
                    if (tile >= w.b || lane * box >= kWideTile || tok >= w.vis) return nowhere;
                    const int pg = w.g.table[tok >> p.page_shift];
                    if (pg < 0 || pg >= p.n_pages) {
                        report_check(p.status);
                        return nowhere; // reads as zeros
                    }
                    return ((pg * p.Hk + w.hk) << p.page_shift) + (tok & ((1 << p.page_shift) - 1));
                };
                int next_row = page_row(w.a);
                for (int tile = w.a; ok && tile < w.b; ++tile) {
                    const int row = next_row;
                    next_row = page_row(tile + 1);
                    const int tokens = clamp(w.vis - tile * kWideTile, 0, kWideTile), n = (tokens + box - 1) / box, i_tile = tile - w.a;
                    const uint32_t note = (i_tile < piece.tiles[0] ? 1u : 0u) | (i_tile < piece.tiles[1] ? 2u : 0u) | (i_tile == 0 ? kNoteFirst : 0u) |
                                          (i_tile == piece.tiles[0] - 1 ? kNoteLast : 0u) | (i_tile == piece.tiles[1] - 1 ? 2 * kNoteLast : 0u) | (uint32_t)((tokens + 15) >> 4) << 8;
#pragma unroll 1
                    for (int i = k0; ok && i < k1; ++i) {
                        const uint32_t fill = 2 * tiles + i;
                        const int at = (int)(fill % kPlaces);
                        const uint32_t bar = smem_u32(&sh.full[ring][at]);
                        if (lane == 0) {
                            ok = ctl.wait_bar(smem_u32(&sh.empty[ring][at]), ((fill / kPlaces) & 1u) ^ 1u, kWaitPlace, fill);
                            if (ok) {
                                sh.note[ring][at] = note;
                                mbar_arrive_expect_tx(bar, (uint32_t)(n * box * 128 * kHalves));
                            }
                        }
                        ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                        if (!ok) break;
                        last = fill + 1;
                        if (lane < n)
#pragma unroll
                            for (int h = 0; h < kHalves; ++h) tma_page(place_at(ring, at) + h * kHalf + lane * box * 128, i ? &tm_v : &tm_k, h * 64, row, bar);
                    }
                    ++tiles;
                }
            }
            if (first && ok) {
                PieceNote none = {};
                none.b = -1;
                announce(none);
            }
            if (first && ok && lane == 0) { // nothing follows
                const uint32_t fill = 2 * tiles;
                const int at = (int)(fill % kPlaces);
                ok = ctl.wait_bar(smem_u32(&sh.empty[ring][at]), ((fill / kPlaces) & 1u) ^ 1u, kWaitPlace, fill);
                if (ok) {
                    sh.note[ring][at] = kNoteEnd;
                    mbar_arrive(smem_u32(&sh.full[ring][at]));
                }
            }
            if (!ok && lane == 0) // a CTA does not end before its copies have landed
                for (uint32_t f = last > (uint32_t)kPlaces ? last - kPlaces : 0; f < last; ++f)
                    if (!kPair || (int)(f & 1u) == k0) ctl.wait_landed(smem_u32(&sh.full[ring][f % kPlaces]), (f / kPlaces) & 1u);
            __syncwarp();
        }
    } else if (warp >= 8) {
        // ------------------------------------------------------------------ products
        // The whole warp goes the same way, so that addresses stay in uniform registers; one lane issues.  (A lone thread that looks
        // for the next product that is ready took 500 cycles from one batch to the next, a tile 7700.)
        if (warp - 8 < kWorkers) {
            const int ring = warp - 8;
            const uint32_t id_s = wide_idesc<T>(kWideTile, false), id_o = wide_idesc<T>(D, true);
            const uint32_t full = smem_u32(&sh.full[ring][0]), empty = smem_u32(&sh.empty[ring][0]);
            const unsigned long long desc = umma_desc(place_at(ring, 0)); // of the ring's first place; a place on: kPlace / 16 more
            // values as they lie: tokens along the inner dimension, a second half of columns 16 KB on
            const unsigned long long desc_v = (desc & ~(0x3fffull << 16)) | (unsigned long long)(kHalf >> 4) << 16;
            const bool issues = elect_one();
            const auto wait = [&](uint32_t bar, uint32_t phase, int where) {
                if (__all_sync(0xffffffffu, sweep::mbar_try_wait(bar, phase))) return true;
                return __all_sync(0xffffffffu, ctl.wait_bar(bar, phase, where, -1)) != 0;
            };
            uint32_t n_p[2] = {0, 0}, n_q[2] = {0, 0};
            const auto queries = [&](int e) { // a piece's queries are there
                if (withhold == 2) {
                    if (issues) ctl.give_up(kWaitQueries, -1);
                    __syncwarp();
                    return false;
                }
                return wait(smem_u32(&sh.q_full[e]), n_q[e]++ & 1u, kWaitQueries);
            };
            const auto scores = [&](int e, int at) {
                const unsigned long long da = umma_desc(q_at(e)), db = desc + (unsigned)(at * (kPlace >> 4));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (issues) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) { // (32 bytes on; a half further on after 64 columns)
                        const int off = (kk >> 2) * (kHalf >> 4) + (kk & 3) * 2;
                        umma_ss(tmem + e * 256, da + off, db + off, id_s, kk != 0);
                    }
                    umma_commit(smem_u32(&sh.s_full[e]));
                }
                __syncwarp();
            };
            // the sums of a tile, in halves of 64 tokens, as their weights come, and with the second one the scores of the next tile
            // where its keys are there: twelve products on end
            const auto sums = [&](int e, int at, uint32_t note, int at_next, bool more) {
                const unsigned long long dv = desc_v + (unsigned)(at * (kPlace >> 4)), da = umma_desc(q_at(e)), db = desc + (unsigned)(at_next * (kPlace >> 4));
                const int steps = (int)(note >> 8) & 15;
                const uint32_t phase = n_p[e]++ & 1u, s_at = tmem + e * 256;
                if (!wait(smem_u32(&sh.p_half[e]), phase, kWaitWeights)) return false;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (issues) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) // (16 tokens on: 2048 bytes; 8 columns of weights)
                        if (kk < steps) umma_ts(s_at + 128, s_at + kk * 8, dv + kk * 128, id_o, kk > 0 || !(note & kNoteFirst));
                }
                __syncwarp();
                if (!wait(smem_u32(&sh.p_full[e]), phase, kWaitWeights)) return false;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (issues) {
#pragma unroll
                    for (int kk = 4; kk < 8; ++kk)
                        if (kk < steps) umma_ts(s_at + 128, s_at + kk * 8, dv + kk * 128, id_o, 1u);
                    if (note & (kPair ? kNoteLast << e : kNoteLast)) umma_commit(smem_u32(&sh.o_full[e]));
                    if (more) {
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const int off = (kk >> 2) * (kHalf >> 4) + (kk & 3) * 2;
                            umma_ss(s_at, da + off, db + off, id_s, kk != 0);
                        }
                        umma_commit(smem_u32(&sh.s_full[e]));
                    }
                }
                __syncwarp();
                return true;
            };
            const auto release = [&](int at) { // when all products so far have ended
                if (issues) umma_commit(empty + at * 8);
                __syncwarp();
            };
            int at = 0;
            uint32_t round = 0;
            bool ok = true;
            uint32_t note = 0;
            const auto next_place = [&]() {
                const int here = at;
                if (++at == kPlaces) at = 0, round ^= 1u;
                return here;
            };
            // keys of the first tile
            ok = wait(full + at * 8, round, kWaitKeys);
            if (ok) {
                note = sh.note[ring][at];
                if (!(note & kNoteEnd)) {
                    for (int e = 0; ok && e < (kPair ? 2 : 1); ++e)
                        if (note >> e & 1u) {
                            ok = queries(ring + e);
                            if (ok) scores(ring + e, at);
                        }
                    release(next_place());
                }
            }
            while (ok && !(note & kNoteEnd)) {
                // a tile's values, and the next one's keys if they are there: per engine the sums of the one, then the scores of the
                // other, so that one engine's softmax runs beside the other one's products
                ok = wait(full + at * 8, round, kWaitValues);
                if (!ok) break;
                const int at_v = next_place();
                const bool ready = __all_sync(0xffffffffu, sweep::mbar_try_wait(full + at * 8, round)) != 0;
                uint32_t next = ready ? sh.note[ring][at] : kNoteFirst;
                const bool along = !(next & (kNoteFirst | kNoteEnd)); // (where a piece ends the engines do not wait for each other's end)
                if (note & 1u) ok = sums(ring, at_v, note, at, along && (next & 1u));
                if (kPair && ok && (note & 2u)) ok = sums(1, at_v, note, at, along && (next & 2u));
                if (!ok) break;
                release(at_v);
                if (!ready) {
                    ok = wait(full + at * 8, round, kWaitKeys);
                    if (!ok) break;
                    next = sh.note[ring][at];
                }
                note = next;
                if (note & kNoteEnd) break;
                if (!along)
                    for (int e = 0; ok && e < (kPair ? 2 : 1); ++e)
                        if (note >> e & 1u) {
                            if (note & kNoteFirst) ok = queries(ring + e);
                            if (ok) scores(ring + e, at);
                        }
                if (!ok) break;
                release(next_place());
            }
            if (!ok && issues) {
                umma_commit(smem_u32(&sh.drain[ring]));
                ctl.wait_landed(smem_u32(&sh.drain[ring]), 0);
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------------ softmax: a thread per row
        const int e = warp >> 2, ring = kPair ? 0 : e, row = (warp & 3) * 32 + lane;
        const uint32_t s_at = tmem + e * 256 + ((uint32_t)((warp & 3) * 32) << 16), o_at = s_at + 128;
        const uint32_t stage = base + (uint32_t)(2 + kWorkers * kPlaces) * kPlace + warp * 4096;
        const int en = kPair ? e : 0, off = kPair ? e * rows : 0;  // the engine's part of a note; its first row
        const uint32_t inv_R = (65536u + p.R - 1) / (uint32_t)p.R; // row / R for rows below 128: (row * inv_R) >> 16
        uint32_t seen = 0, n_s = 0, n_o = 0, pieces = 0; // tiles of the ring passed so far; phases
        bool ok = true;
        const PieceNote *w = &sh.piece[ring][0]; // (read where it is wanted: registers are for scores)
        int my_rows = 0, my_tiles = 0, n0 = 0, lim = 0, begin = 0, end = -1; // the engine's rows, tiles and first packed row; tokens that the
                                                                             // thread's row sees; the piece's tiles
        // The next piece, and its queries: the scores of the piece before are all there, so that nobody reads its queries any more.
        const auto next_piece = [&]() {
            const int at = (int)(pieces % kPieces);
            ok = __all_sync(0xffffffffu, ctl.wait_bar(smem_u32(&sh.piece_full[ring][at]), (pieces / kPieces) & 1u, kWaitPieces, pieces));
            if (!ok) return;
            w = &sh.piece[ring][at];
            ++pieces;
            begin = w->a, end = w->b;
            if (end < 0) return;
            my_rows = w->rows[en], my_tiles = w->tiles[en], n0 = w->n0[en];
            lim = row >= my_rows ? w->vis : w->prefix ? w->len : clamp(w->sees[en] + (int)(row * inv_R >> 16), 0, w->len);
            if (my_tiles > 0 && (warp & 3) == 0 && lane == 0) {
                // rows behind the segment's last are whatever comes next: nobody reads what comes of them
                const uint32_t bar = smem_u32(&sh.q_full[e]);
                mbar_arrive_expect_tx(bar, (uint32_t)(rows * D * 2));
                ++sh.asked[e];
#pragma unroll
                for (int hh = 0; hh < kHalves; ++hh) tma_queries(q_at(e) + hh * kHalf, &tm_q, hh * 64, w->hk, n0, bar);
            }
        };
        next_piece();
        while (ok && end >= 0) {
            float m = -INFINITY, l = 0.0f;
            for (int tile = begin; ok && tile < begin + my_tiles; ++tile) {
                ok = __all_sync(0xffffffffu, ctl.wait_bar(smem_u32(&sh.s_full[e]), n_s & 1u, kWaitScores, pieces));
                if (!ok) break;
                ++n_s;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                float s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(s_at + c * 32, s + c * 32);
                tmem_wait_ld();
                const int n_see = lim - tile * kWideTile;
                if (__any_sync(0xffffffffu, n_see < kWideTile))
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i] = i < n_see ? s[i] : -INFINITY;
                const int n_here = w->vis - tile * kWideTile; // tokens behind the last one: their values must be zeros up to the product's end
                if (n_here < kWideTile && (n_here & 15)) {
                    const uint32_t fill = (seen + (tile - begin)) * 2 + 1;
                    const int at = (int)(fill % kPlaces), n_zero = 16 - (n_here & 15);
                    ok = __all_sync(0xffffffffu, ctl.wait_bar(smem_u32(&sh.full[ring][at]), (fill / kPlaces) & 1u, kWaitLastValues, pieces));
#pragma unroll
                    for (int hh = 0; hh < kHalves; ++hh)
                        if (ok && row < n_zero * 8)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(place_at(ring, at) + hh * kHalf + n_here * 128 + row * 16), "r"(0) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    if (!ok) break;
                }
                float t0 = s[0], t1 = s[1], t2 = s[2], t3 = s[3];
#pragma unroll
                for (int i = 4; i < 128; i += 4) t0 = fmaxf(t0, s[i]), t1 = fmaxf(t1, s[i + 1]), t2 = fmaxf(t2, s[i + 2]), t3 = fmaxf(t3, s[i + 3]);
                const float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * p.scale_log2;
                if (__any_sync(0xffffffffu, row < my_rows && top > m + 8.0f)) { // (from -inf: any; rows of nobody hold whatever was there)
                    const float now = fmaxf(m, top), fix = m == now ? 1.0f : exp2_approx(m - now);
                    if (tile > begin) { // (this tile's scores being there, the products before them have ended)
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_at + c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fix);
                            tmem_st16(o_at + c, o);
                        }
                    }
                    l *= fix, m = now;
                }
                // Weights, in halves of 64 tokens so that the second product starts on the first while the other is made.
                const float ref = m == -INFINITY ? 0.0f : m;
                float l0 = 0.0f, l1 = 0.0f, l2 = 0.0f, l3 = 0.0f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w16[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float a0 = exp2_approx(fmaf(s[c * 32 + 2 * i], p.scale_log2, -ref)), a1 = exp2_approx(fmaf(s[c * 32 + 2 * i + 1], p.scale_log2, -ref));
                        const float a2 = exp2_approx(fmaf(s[c * 32 + 2 * i + 2], p.scale_log2, -ref)), a3 = exp2_approx(fmaf(s[c * 32 + 2 * i + 3], p.scale_log2, -ref));
                        l0 += a0, l1 += a1, l2 += a2, l3 += a3;
                        // (weights enter the second product in the cache's type: half a step of it, relative, per token; fp16 weights below
                        // 2^-14 by 2^-25, where the row's largest is 1 to 2^8, while the sum counts them whole)
                        w16[i] = pack2<T>(a0, a1), w16[i + 1] = pack2<T>(a2, a3);
                    }
                    tmem_st16(s_at + c * 16, w16);
                    if (c & 1) {
                        tmem_wait_st();
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0 && !(withhold == 1 && warp == 0)) mbar_arrive(smem_u32(c == 1 ? &sh.p_half[e] : &sh.p_full[e]));
                    }
                }
                l += (l0 + l1) + (l2 + l3);
            }
            if (!ok) break;
            seen += end - begin;
            // what the piece leaves, and where; then, while its last products run, the next one's queries are asked for
            const int had_rows = my_rows, had_tiles = my_tiles, my_t = (int)(row * inv_R >> 16), my_h = row - my_t * p.R;
            const bool by_row = w->place == kToRows, at_once = by_row && p.n_groups == 0;
            const int h0 = w->hk * p.R;
            if (at_once) l = settled(l, lim > 0);
            char *dst;             // of the engine's first row; the next token's and the next head's are so far on
            long long per_t, per_h;
            if (at_once) {
                per_t = p.out_stride, per_h = D * 2;
                dst = p.out + (long long)n0 * p.out_stride + (long long)h0 * (D * 2);
            } else {
                per_t = (long long)(by_row ? p.Hq : p.R) * (D * 4), per_h = D * 4;
                dst = (char *)(by_row ? p.whole[w->prefix ? 0 : 1].o : p.pieces.o) + (by_row ? (long long)n0 * p.Hq + h0 : (long long)w->place * p.pieces.M + off) * (D * 4);
            }
            if (row < had_rows) {
                const long long at = by_row ? (long long)(n0 + my_t) * p.Hq + h0 + my_h : (long long)w->place * p.pieces.M + off + row;
                if (!at_once)
                    (by_row ? p.whole[w->prefix ? 0 : 1].ml : p.pieces.ml)[at] = make_float2(m, l);
                else if (p.lse)
                    p.lse[at] = lse_of(m, l);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.piece_empty[ring][(pieces - 1) % kPieces]));
            next_piece();
            if (!ok) break;
            if (had_tiles > 0) {
                ok = __all_sync(0xffffffffu, ctl.wait_bar(smem_u32(&sh.o_full[e]), n_o & 1u, kWaitSums, pieces));
                if (!ok) break;
                ++n_o;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            if (had_tiles == 0 && !at_once) continue; // (where l is 0 nobody reads the sums)
            // Rows go out by way of shared memory, 128 bytes of 32 rows at a time, so that a store fills whole lines (a thread that
            // writes its own row keeps the load-store unit for 32 lines an instruction: a piece took 17000 cycles beside its tiles).
            const float inv = inverse(l);
            const auto out_128 = [&](const uint32_t *v, int c) { // the thread's 128 bytes, c bytes into the rows
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(stage + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(v[4 * i]), "r"(v[4 * i + 1]),
                                 "r"(v[4 * i + 2]), "r"(v[4 * i + 3])
                                 : "memory");
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int in_warp = i * 4 + (lane >> 3), r = (warp & 3) * 32 + in_warp, piece = lane & 7;
                    const int t = (int)(r * inv_R >> 16), hh = r - t * p.R;
                    const uint4 x = sweep::lds128(stage + in_warp * 128 + ((piece ^ (in_warp & 7)) << 4));
                    if (r < had_rows) *reinterpret_cast<uint4 *>(dst + t * per_t + hh * per_h + c + piece * 16) = x;
                }
                __syncwarp();
            };
            if (at_once) {
#pragma unroll 1
                for (int c = 0; c < D; c += 64) {
                    float o[64];
                    uint32_t v[32];
                    if (had_tiles > 0) {
                        tmem_ld32(o_at + c, o), tmem_ld32(o_at + c + 32, o + 32);
                        tmem_wait_ld();
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = l == 0.0f ? 0u : pack2<T>(o[2 * i] * inv, o[2 * i + 1] * inv);
                    out_128(v, c * 2);
                }
            } else {
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    tmem_ld32(o_at + c, o);
                    tmem_wait_ld();
                    out_128(reinterpret_cast<const uint32_t *>(o), c * 4);
                }
            }
        }
        // a CTA that gives up does not end before the engine's query copy has landed either: the products need not have come to wait for it
        if (!ok && (warp & 3) == 0 && lane == 0 && sh.asked[e] > 0) ctl.wait_landed(smem_u32(&sh.q_full[e]), (sh.asked[e] - 1u) & 1u);
        __syncwarp();
    }
    // ---------------------------------------------------------------------- end
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

} // namespace attend
} // namespace dart
