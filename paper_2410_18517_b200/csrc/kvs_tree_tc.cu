// Attention of a tree of drafted tokens on the 5th-generation tensor cores (bf16 storage, head size 64 or 128).
// The mathematics and the masks are those of kvs_tree.cu.
//
// One thread block per SM with two softmax *slots*, each with its own scores and output in tensor memory:
//   warps 0..3 / 4..7  softmax of slot 0 / 1: one thread per query row (= tensor-memory lane), the 128 keys of a key
//                      tile; warps whose lanes hold no query row stay out of it
//   warp 8 (one lane)  TMA producer: query tiles per piece, K and V tiles through one ring (K0 V0 K1 V1 ...)
//   warp 9 (one lane)  MMA issuer: S(0) S(1), then PV(k) S(k+2) ..., step k belonging to slot k & 1, so that the
//                      tensor pipe works for one slot while the other slot's softmax runs
// Two query tiles (more than 128 rows per kv-head): the slots take one each and every K/V tile serves both, which
// halves the shared-memory traffic of the copies.  One query tile: the slots take alternate key tiles and their two
// results are merged at the end (a slot's threads can read the other's output: same tensor-memory lanes).
// 128-key tiles, because an S product of N = 64 keys reads 6 KiB of shared memory per 32 tensor cycles, more than
// the 128 bytes a cycle there are; N = 128 reads just that.
// P goes into the second contraction as one bf16 term (each weight off by at most 2^-8 of itself, the sum of the weights
// kept in fp32 from the unrounded ones): the result is rounded to bf16 anyway, and a second term would add half again to the
// tensor work of wide trees, which the tensor pipe bounds.
//
// The last tiles of a unit hold drafts and rows past its end.  There the softmax warps also clean the V tile in
// shared memory before the MMA may read it: rows past the end become zero, and so do non-finite elements of draft
// rows (0 * NaN would reach rows that do not see them); the rows that do see such an element get it back at the end
// from global memory, a path nothing but broken drafts takes.
#include <algorithm>

#include "kvs_umma.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

constexpr int kTcSlotWarps = 4;
constexpr int kTcThreads = (2 * kTcSlotWarps + 4) * 32;   // three warpgroups: two of softmax, one of producer and issuer
// A softmax thread holds a tile's 128 scores, more than the 168 registers a thread of twelve warps is launched with allow
// beside the rest: the third warpgroup hands its share over.  2 * 128 * 224 + 128 * 56 = 384 * 168 registers.
constexpr int kTcSoftmaxRegs = 224, kTcOtherRegs = 56;
constexpr int kTcKeys = 128;
constexpr int kTcQBlock = kTreeTileRows * 128;   // one swizzled block of Q: 128 rows x 64 bf16 columns
constexpr int kTcKvBlock = kTcKeys * 128;        // one swizzled block of K or V: 128 rows x 64 bf16 columns
constexpr int kTcBoxRows = 64, kTcTailRows = 16; // rows per copy: whole boxes, and the partly filled end of a unit
constexpr uint32_t kTcTmemCols = 512;            // slot s: scores [256 s, 256 s + 128), output [256 s + 128, 256 s + 128 + D)

template <int D>
struct TcShape {
    static constexpr int HALVES = D / 64;
    static constexpr int Q_BYTES = HALVES * kTcQBlock;           // one query tile
    static constexpr int KV_BYTES = HALVES * kTcKvBlock;
    static constexpr int RING = 10 / HALVES;                     // K and V buffers: 160 KiB
    static constexpr int SMEM_BYTES = 2 * Q_BYTES + RING * KV_BYTES + 512 + 4 * kTreeTileRows * 4;
};

struct TreeTcArgs {
    TreeArgs a;
    TreePlan p;
    long long krow0, vrow0;      // first row of the slot's planes in the pool-wide row numbering
    long long plane_rows;
};

// The pieces of one team, in order; every role of the block walks the same ones.  (A pool's rows, and so its tiles, are
// numbered in 32 bits.)
struct Pieces {
    const TreeTcArgs& x;
    int gt, t1;        // next tile of the line, end of the team's run
    int u, ti0, nt, n; // unit, first key tile, key tiles, rows of the unit
    bool whole;
    __device__ Pieces(const TreeTcArgs& args, int team) : x(args) {
        gt = (int)((long long)team * x.p.T / x.p.teams);
        t1 = (int)((long long)(team + 1) * x.p.T / x.p.teams);
    }
    __device__ bool next() {
        while (gt < t1) {
            u = gt / x.p.tpu;
            ti0 = gt - u * x.p.tpu;
            const int piece = min(x.p.tpu - ti0, t1 - gt);
            gt += piece;
            n = x.a.unit_len ? min(x.a.unit_len[u], x.a.capacity) : x.a.n;
            const int tiles = (n + kTcKeys - 1) / kTcKeys;       // key tiles the unit really has
            const int te = min(ti0 + piece, tiles);
            if (ti0 >= te) continue;                             // past a ragged unit's end
            nt = te - ti0;
            whole = ti0 == 0 && te == tiles;
            return true;
        }
        return false;
    }
};

// The steps of a block: step k is one key tile of one slot (k & 1).
struct Steps {
    Pieces pi;
    bool two;          // two query tiles: two steps per key tile
    int pc = -1;       // piece
    int i = 0, n = 0;  // step within the piece, steps of the piece
    int k = -1;        // step of the block
    int t0 = 0;        // key tiles of earlier pieces
    __device__ Steps(const TreeTcArgs& args, int team, bool two_) : pi(args, team), two(two_) {}
    __device__ bool next() {
        if (++i >= n) {
            if (pc >= 0) t0 += pi.nt;
            if (!pi.next()) return false;
            ++pc;
            i = 0;
            n = two ? 2 * pi.nt : pi.nt;
        }
        ++k;
        return true;
    }
    __device__ int tile() const { return two ? i >> 1 : i; }                 // key tile within the piece
    __device__ bool first() const { return i < 2; }                          // the slot's first step of the piece
    __device__ bool last_use() const { return !two || (i & 1); }             // of the key tile
    __device__ bool last() const { return i == n - 1; }
};

// The weights p = 2^(x * scale - m_ref) of 32 scores, 0 where the key's bit in `vis` is not set (MASK), as they go to
// tensor memory (two bf16 per column from `taddr` on); returns their sum.
template <bool MASK>
__device__ __forceinline__ float weights32(const float (&x)[32], float scale_log2, float m_ref, uint32_t vis, uint32_t taddr) {
    const float2 sc = make_float2(scale_log2, scale_log2), nm = make_float2(-m_ref, -m_ref);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        const float2 t = __ffma2_rn(make_float2(x[i], x[i + 1]), sc, nm);
        float2 p = make_float2(fast_exp2(t.x), fast_exp2(t.y));
        if (MASK) {
            p.x = (vis >> i) & 1u ? p.x : 0.f;
            p.y = (vis >> (i + 1)) & 1u ? p.y : 0.f;
        }
        sum[(i >> 1) & 1] = __fadd2_rn(sum[(i >> 1) & 1], p);
        w[i >> 1] = pack2_bf16(p.x, p.y);
    }
    tmem_st16(taddr, w);
    return (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
}

// Maximum of 32 scores, of those a query sees (MASK).
template <bool MASK>
__device__ __forceinline__ float max32(const float (&x)[32], uint32_t vis) {
    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < 32; i += 8)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float u = x[i + c], v = x[i + 4 + c];
            if (MASK) {
                u = (vis >> (i + c)) & 1u ? u : -INFINITY;
                v = (vis >> (i + 4 + c)) & 1u ? v : -INFINITY;
            }
            m4[c] = fmax3(m4[c], u, v);
        }
    return fmax3(fmaxf(m4[0], m4[1]), m4[2], m4[3]);
}

__device__ __forceinline__ uint32_t nonfinite16(uint32_t w) {      // mask of the halves of w that are Inf or NaN
    return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Which of the 64 keys from `off` rows behind the context's end on a query sees (off < 0: context rows first).
__device__ __forceinline__ unsigned long long visible64(unsigned long long sees, int off) {
    if (off >= 64) return 0ull;
    if (off >= 0) return sees >> off;
    if (off <= -64) return ~0ull;
    return sees << -off | ((1ull << -off) - 1ull);
}

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1)
    tree_attention_tc(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_kv,
                      const __grid_constant__ CUtensorMap tmap_tail, const __grid_constant__ TreeTcArgs x) {
    using S = TcShape<D>;
    constexpr int NB = S::RING, kKv = S::KV_BYTES;
    static_assert(2 * 128 * kTcSoftmaxRegs + 128 * kTcOtherRegs <= kTcThreads * 168, "registers at launch");
    const TreeArgs& a = x.a;
    const TreePlan& p = x.p;
    extern __shared__ __align__(1024) unsigned char sQ[];       // the 128-byte swizzle counts from 1024-byte boundaries
    if ((smem_u32(sQ) & 1023u) != 0u) {
        if (threadIdx.x == 0) atomicExch(a.status, kDevBounds);
        return;
    }
    unsigned char* ring = sQ + 2 * S::Q_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + NB * kKv);
    uint64_t* q_full = bars;           // [2]
    uint64_t* q_free = bars + 2;       // [2] every S of a piece is done
    uint64_t* o_full = bars + 4;       // [2] per slot: the step's PV is in the slot's output
    uint64_t* s_full = bars + 6;       // [2] per slot
    uint64_t* p_full = bars + 8;       // [2] per slot: one arrival per active softmax thread
    uint64_t* epi = bars + 10;         // all active softmax threads (one query tile only)
    uint64_t* drain = bars + 11;
    uint64_t* full = bars + 12;        // [NB]
    uint64_t* empty = full + NB;       // [NB]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(empty + NB);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);    // [2]; the second bounds the drains
    volatile int* broken = abort_flag + 2;                                        // [2] by piece parity
    float2* exch = reinterpret_cast<float2*>(bars + 64);                          // [2 slots][128 rows] maximum, sum

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int pairs = (p.m_tiles + 1) / 2;
    const int team = blockIdx.x / pairs, mt0 = 2 * (blockIdx.x - team * pairs);
    const bool two = mt0 + 1 < p.m_tiles;
    const int quarters = (p.tokens * a.G + 31) / 32;        // tensor-memory lane quarters that hold query rows
    const uint32_t active = quarters * 32;                  // softmax threads at work per slot

    if (tid == 0) {
        for (int i = 0; i < 12 + 2 * NB; ++i) mbar_init(&bars[i], 1);
        mbar_init(&p_full[0], active);
        mbar_init(&p_full[1], active);
        mbar_init(epi, 2 * active);
        abort_flag[0] = abort_flag[1] = broken[0] = broken[1] = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(kTcTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    // Key tile t of the block has K in ring entry 2 t and V in 2 t + 1; entry e lies in buffer e % NB, and its
    // barriers are then in phase (e / NB) & 1.  A piece's queries: buffer and barrier qi, phase qp.
    auto wait = [&](uint64_t* bar, uint32_t ph) { return mbar_wait_bounded(bar, ph & 1u, abort_flag, a.status, a.wait_ns); };
    if (warp >= 2 * kTcSlotWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcOtherRegs));
    if (warp == 2 * kTcSlotWarps) {
        // ------------------------------ TMA producer ------------------------------
        if (lane == 0) {
            const uint32_t q_bytes = (uint32_t)(S::HALVES * p.tokens * a.G * 128);
            int e = 0, pc = 0;               // ring entries issued, pieces
            int q_done = 0;                  // pieces whose queries were issued
            bool ok = true;
            for (Pieces pi(x, team); ok && pi.next(); ++pc) {
                const int b = pi.u / a.Hkv, hk = pi.u - b * a.Hkv;
                const int qi = two ? 0 : pc & 1, qn = two ? pc : pc >> 1;
                for (int j = 0; j < pi.nt && ok; ++j) {
                    const int row0 = (pi.ti0 + j) * kTcKeys;
                    const int rows = min(kTcKeys, pi.n - row0);
                    const int boxes = rows / kTcBoxRows, tails = (rows - boxes * kTcBoxRows + kTcTailRows - 1) / kTcTailRows;
                    const uint32_t bytes = (uint32_t)(boxes * kTcBoxRows + tails * kTcTailRows) * S::HALVES * 128;
                    long long row = (long long)pi.u * a.row_stride + row0;
                    if (!KVS_BOUNDS_OK(row, boxes * kTcBoxRows + tails * kTcTailRows, x.plane_rows, a.status)) row = 0;
                    for (int kv = 0; kv < 2; ++kv) {
                        const int st = e % NB;
                        if (e >= NB) ok = wait(&empty[st], e / NB - 1);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&full[st], bytes);
                        const int y = (int)((kv == 0 ? x.krow0 : x.vrow0) + row);
#pragma unroll
                        for (int h = 0; h < S::HALVES; ++h) {
                            unsigned char* dst = ring + st * kKv + h * kTcKvBlock;
                            for (int i = 0; i < boxes; ++i)
                                tma_load_2d_pf(dst + i * kTcBoxRows * 128, &tmap_kv, h * 64, y + i * kTcBoxRows, &full[st]);
                            for (int i = 0; i < tails; ++i)
                                tma_load_2d_pf(dst + (boxes * kTcBoxRows + i * kTcTailRows) * 128, &tmap_tail, h * 64,
                                               y + boxes * kTcBoxRows + i * kTcTailRows, &full[st]);
                        }
                        ++e;
                        if (kv == 0 && j == 0) {      // the queries, behind the piece's first K tile
                            if (qn >= 1) ok = wait(&q_free[qi], qn - 1);
                            if (!ok) break;
                            mbar_arrive_expect_tx(&q_full[qi], two ? 2 * q_bytes : q_bytes);
                            for (int m = 0; m < (two ? 2 : 1); ++m)
#pragma unroll
                                for (int h = 0; h < S::HALVES; ++h)
                                    tma_load_4d(sQ + (two ? m : qi) * S::Q_BYTES + h * kTcQBlock, &tmap_q, h * 64, hk * a.G,
                                                (mt0 + m) * p.tokens, b, &q_full[qi]);
                            ++q_done;
                        }
                    }
                }
            }
            if (!ok || abort_flag[0] != 0) {
                // Gave up: wait (bounded) for the copies already issued, so that none is in flight into this
                // block's shared memory when it exits.
                for (int j = max(0, e - NB); j < e; ++j)
                    mbar_wait_bounded(&full[j % NB], (uint32_t)(j / NB) & 1u, abort_flag + 1, a.status, a.wait_ns);
                for (int j = max(0, q_done - 2); j < q_done; ++j) {
                    const int qi = two ? 0 : j & 1, qn = two ? j : j >> 1;
                    if (!two || j == q_done - 1)
                        mbar_wait_bounded(&q_full[qi], (uint32_t)qn & 1u, abort_flag + 1, a.status, a.wait_ns);
                }
            }
        }
    } else if (warp == 2 * kTcSlotWarps + 1) {
        // ------------------------------ MMA issuer ------------------------------
        // The pipe runs one thread's MMAs in issue order: S(k+2) overwrites its slot's scores only after PV(k) has
        // read the weights that lie over them.  The whole warp walks the steps, one elected lane issues.
        const uint32_t idesc_s = instr_desc_bf16(0, kTcKeys);
        const uint32_t idesc_o = instr_desc_bf16(1, D);
        const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
        const bool leader = elect_one();
        auto all_wait = [&](uint64_t* bar, uint32_t ph) { return __all_sync(0xffffffffu, wait(bar, ph)) != 0; };   // one answer for the warp
        // descriptors of the buffers' starts; steps inside a buffer are added in units of 16 bytes
        const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ), 16, 1024);
        const uint64_t k_desc = smem_desc_sw128(smem_u32(ring), 16, 1024);
        // V is MN-major: 64 head-dim columns contiguous per key row, the other 64 (D = 128) one column block (LBO)
        // away; 8-key groups 1024 bytes (SBO) apart
        const uint64_t v_desc = smem_desc_sw128(smem_u32(ring), kTcKvBlock, 1024);
        auto issue_s = [&](const Steps& s) {
            const int qi = two ? 0 : s.pc & 1, qn = two ? s.pc : s.pc >> 1;
            const int e = 2 * (s.t0 + s.tile()), st = e % NB;
            if (s.i == 0 && !all_wait(&q_full[qi], qn)) return false;
            if (!all_wait(&full[st], e / NB)) return false;
            tc_fence_after();
            const uint64_t q = q_desc + (uint32_t)(two ? s.k & 1 : qi) * (S::Q_BYTES / 16);
            const uint64_t k = k_desc + (uint32_t)st * (kKv / 16);
            const uint32_t d = tmem + (s.k & 1) * 256;
            if (leader) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_bf16(d, q + ((ks >> 2) * kTcQBlock + (ks & 3) * 32) / 16, k + ((ks >> 2) * kTcKvBlock + (ks & 3) * 32) / 16,
                              idesc_s, ks > 0);
                umma_commit(&s_full[s.k & 1]);
                if (s.last_use()) umma_commit(&empty[st]);
                if (s.last()) umma_commit(&q_free[qi]);
            }
            __syncwarp();
            return true;
        };
        Steps sa(x, team, two), sp(x, team, two);     // next S, next PV
        bool more = sa.next(), ok = true;
        for (int i = 0; i < 2 && ok && more; ++i) {
            ok = issue_s(sa);
            more = sa.next();
        }
        while (ok && sp.next()) {
            const int e = 2 * (sp.t0 + sp.tile()) + 1, st = e % NB, slot = sp.k & 1;
            ok = all_wait(&p_full[slot], sp.k >> 1) && all_wait(&full[st], e / NB);
            if (!ok) break;
            tc_fence_after();
            const uint64_t v = v_desc + (uint32_t)st * (kKv / 16);
            const uint32_t o = tmem + slot * 256 + 128, w = tmem + slot * 256, add = !sp.first();
            if (leader) {
#pragma unroll
                for (int ks = 0; ks < kTcKeys / 16; ++ks) umma_bf16_ts(o, w + ks * 8, v + ks * 16 * 128 / 16, idesc_o, ks > 0 ? 1 : add);
                umma_commit(&o_full[slot]);
                if (sp.last_use()) umma_commit(&empty[st]);
            }
            __syncwarp();
            if (more) {
                ok = issue_s(sa);
                more = sa.next();
            }
        }
        if (!ok && leader) {     // the MMAs already issued must be done before the block gives its memory back
            umma_commit(drain);
            mbar_wait_bounded(drain, 0, abort_flag + 1, a.status, a.wait_ns);
        }
    }
    } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTcSoftmaxRegs));
    if ((warp & 3) < quarters) {
        // ------------------------------ softmax / output rows ------------------------------
        const int slot = warp >> 2;
        const int r = tid & 127;                             // query row in the tile = tensor-memory lane
        const int mt = mt0 + (two ? slot : 0), tok0 = mt * p.tokens;
        const int rows = min(p.tokens, a.n_t - tok0) * a.G;
        const uint32_t lanes = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t ts = lanes + slot * 256, to = ts + 128;
        const bool real = r < rows;                          // lanes past the last row hold no query: their scores are junk
        const int tok = tok0 + min(r, rows - 1) / a.G, g = min(r, rows - 1) % a.G;
        const unsigned long long all = a.n_t >= 64 ? ~0ull : (1ull << a.n_t) - 1;
        int k0 = 0, t0 = 0, pc = 0;                          // steps, key tiles, pieces before this one
        uint32_t ep = 0;                                     // phases used of epi
        bool ok = true;
        for (Pieces pi(x, team); ok && pi.next(); ++pc) {
            const int b = pi.u / a.Hkv, hk = pi.u - b * a.Hkv;
            const int ctx = pi.n - a.n_t;                    // rows every query sees
            const unsigned long long sees =
                a.mask ? a.mask[(long long)b * a.n_t + tok] & all : (tok >= 63 ? ~0ull : (2ull << tok) - 1);
            const int steps = two ? 2 * pi.nt : pi.nt;
            float m_ref = -1.0e30f, l = 0.f;                 // p is taken relative to m_ref (log2 domain)
            const int i0 = (k0 ^ slot) & 1;                  // the slot's first step of the piece
            for (int i = i0; i < steps; i += 2) {
                const int c = (k0 + i) >> 1;                 // the slot's count of steps
                const int tile = two ? i >> 1 : i;
                const int key0 = (pi.ti0 + tile) * kTcKeys;
                const bool mask = key0 + kTcKeys > ctx;      // the tile holds drafts or rows past the end
                ok = wait(&s_full[slot], c);
                if (!ok) break;
                tc_fence_after();
                unsigned long long vx = ~0ull, vy = ~0ull;
                if (mask) {
                    vx = visible64(sees, key0 - ctx);
                    vy = visible64(sees, key0 + 64 - ctx);
                    // Clean the V tile (see the head of this file).  Only behind the wait above: S of this tile is
                    // done, so the ring entry that had this V buffer before was released and filled again in
                    // order, and its barrier cannot be a phase behind the one waited for.  (With two query tiles
                    // both slots clean the same tile: they write the same values.)
                    const int e = 2 * (t0 + tile) + 1, st = e % NB;
                    ok = wait(&full[st], e / NB);
                    if (!ok) break;
                    for (int v16 = r; v16 < kKv / 16; v16 += active) {
                        const int key = key0 + (v16 * 16 % kTcKvBlock) / 128;
                        if (key < ctx) continue;
                        uint4* q4 = reinterpret_cast<uint4*>(ring + st * kKv + v16 * 16);
                        uint4 v = make_uint4(0u, 0u, 0u, 0u);
                        if (key < pi.n) {
                            v = *q4;
                            const uint32_t bx = nonfinite16(v.x), by = nonfinite16(v.y), bz = nonfinite16(v.z), bw = nonfinite16(v.w);
                            if ((bx | by | bz | bw) == 0u) continue;
                            broken[pc & 1] = pc + 1;
                            v = make_uint4(v.x & ~bx, v.y & ~by, v.z & ~bz, v.w & ~bw);
                        }
                        *q4 = v;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                // All of the scores are asked for at once: beside running MMAs, which read and write tensor memory
                // through the same ports, a load takes 250 to 400 cycles.
                float x0[32], x1[32], x2[32], x3[32];
                __syncwarp();                                // the warp's tensor-memory accesses are made together
                tmem_ld32_issue(ts, x0);
                tmem_ld32_issue(ts + 32, x1);
                tmem_ld32_issue(ts + 64, x2);
                tmem_ld32_issue(ts + 96, x3);
                tmem_ld_wait(x0);
                tmem_ld_wait(x1);
                tmem_ld_wait(x2);
                tmem_ld_wait(x3);
                float mx;
                if (mask)
                    mx = fmaxf(fmaxf(max32<true>(x0, (uint32_t)vx), max32<true>(x1, (uint32_t)(vx >> 32))),
                               fmaxf(max32<true>(x2, (uint32_t)vy), max32<true>(x3, (uint32_t)(vy >> 32))));
                else
                    mx = fmaxf(fmaxf(max32<false>(x0, 0u), max32<false>(x1, 0u)), fmaxf(max32<false>(x2, 0u), max32<false>(x3, 0u)));
                mx *= a.scale_log2;
                // The reference maximum only moves when the new one is more than 8 (a factor 256) above it; then
                // the output row and the sum so far are rescaled.  (S of this step is done, so PV of the slot's
                // step before it is too: nothing is being added to the output.)
                const bool grow = real && mx > m_ref + 8.0f;
                if (__any_sync(0xffffffffu, grow)) {
                    const float m_new = grow ? mx : m_ref;
                    const float alpha = fast_exp2(m_ref - m_new);
                    if (i > i0) {
#pragma unroll 1
                        for (int cc = 0; cc < D; cc += 8) tmem_scale8(to + cc, alpha);
                    }
                    l *= alpha;
                    m_ref = m_new;
                }
                if (mask) {
                    l += weights32<true>(x0, a.scale_log2, m_ref, (uint32_t)vx, ts);
                    l += weights32<true>(x1, a.scale_log2, m_ref, (uint32_t)(vx >> 32), ts + 16);
                    l += weights32<true>(x2, a.scale_log2, m_ref, (uint32_t)vy, ts + 32);
                    l += weights32<true>(x3, a.scale_log2, m_ref, (uint32_t)(vy >> 32), ts + 48);
                } else {
                    l += weights32<false>(x0, a.scale_log2, m_ref, 0u, ts);
                    l += weights32<false>(x1, a.scale_log2, m_ref, 0u, ts + 16);
                    l += weights32<false>(x2, a.scale_log2, m_ref, 0u, ts + 32);
                    l += weights32<false>(x3, a.scale_log2, m_ref, 0u, ts + 48);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                mbar_arrive(&p_full[slot]);
            }
            if (!ok) break;
            const bool has = i0 < steps;
            if (has) {
                const int last = i0 + (steps - 1 - i0) / 2 * 2;
                ok = wait(&o_full[slot], (uint32_t)(k0 + last) >> 1);
                if (!ok) break;
                tc_fence_after();
            }
            float w0 = 1.f, w1 = 0.f;          // weights of the own and the other slot's output
            bool other = false;
            if (!two) {
                exch[slot * kTreeTileRows + r] = make_float2(m_ref, l);
                tc_fence_before();
                mbar_arrive(epi);
                ok = wait(epi, ep);
                ++ep;
                if (!ok) break;
                tc_fence_after();
                const float2 ml = exch[(slot ^ 1) * kTreeTileRows + r];
                const float m_new = fmaxf(m_ref, ml.x);
                w0 = fast_exp2(m_ref - m_new);
                w1 = fast_exp2(ml.x - m_new);
                other = steps >= 2 || !has;
                l = has ? (other ? fmaf(w0, l, w1 * ml.y) : l) : ml.y;
                m_ref = m_new;
            }
            const bool patch = broken[pc & 1] == pc + 1;
            const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;        // nothing visible: 0
            const long long orow = ((long long)b * a.n_t + tok) * a.Hq + hk * a.G + g;
            const long long prow = ((2ll * team + (pi.ti0 == 0 ? 1 : 0)) * p.m_tiles + mt) * p.tile_rows + r;
            // one query tile: each slot's threads write half of the columns
            const int c0 = two ? 0 : slot * (D / 2), c1 = two ? D : c0 + D / 2;
#pragma unroll 1
            for (int cc = c0; cc < c1; cc += 32) {
                float o[32];
                __syncwarp();
                if (has) tmem_ld32(to + cc, o);
                if (other) {
                    float o2[32];
                    tmem_ld32(lanes + (slot ^ 1) * 256 + 128 + cc, o2);
#pragma unroll
                    for (int j = 0; j < 32; ++j) o[j] = has ? fmaf(w1, o2[j], w0 * o[j]) : o2[j];
                }
                if (patch) {
                    // a draft row this query sees holds Inf or NaN: its elements go into the sum as they are
                    for (int d = 0; d < a.n_t; ++d) {
                        const int key = ctx + d;
                        if (!(sees >> d & 1ull) || key < pi.ti0 * kTcKeys || key >= (pi.ti0 + pi.nt) * kTcKeys) continue;
                        const __nv_bfloat16* vr = reinterpret_cast<const __nv_bfloat16*>(a.vplane) + ((long long)pi.u * a.row_stride + key) * D + cc;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float v = __bfloat162float(vr[j]);
                            if (!isfinite(v)) o[j] += v;
                        }
                    }
                }
                if (real && pi.whole) {
                    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + orow * D + cc);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        dst[j] = make_uint4(pack2_bf16(o[8 * j] * inv, o[8 * j + 1] * inv), pack2_bf16(o[8 * j + 2] * inv, o[8 * j + 3] * inv),
                                            pack2_bf16(o[8 * j + 4] * inv, o[8 * j + 5] * inv), pack2_bf16(o[8 * j + 6] * inv, o[8 * j + 7] * inv));
                } else if (real) {
                    float4* dst = reinterpret_cast<float4*>(a.part_o + prow * D + cc);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dst[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                }
            }
            if (!pi.whole && real && (two || slot == 0)) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(m_ref, l);
            tc_fence_before();      // the slot's first PV of the next piece waits for this thread's arrival on p_full
            if (!two) {             // ... and, as both slots' threads read both outputs, for the other slot's too
                mbar_arrive(epi);
                ok = wait(epi, ep);
                ++ep;
                tc_fence_after();
            }
            k0 += steps;
            t0 += pi.nt;
        }
    }
    }
    // every thread of every role ends here; tensor memory is released by the warp that took it
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTcTmemCols) : "memory");
    }
}

}  // namespace

cudaError_t init_tree_tc_kernels() {
    const cudaError_t e = cudaFuncSetAttribute(tree_attention_tc<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<128>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(tree_attention_tc<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<64>::SMEM_BYTES);
}

void plan_tree_tc(const TreeArgs& a, int blocks, TreePlan* p) {
    // as many query tiles as 128 rows ask for, of equal size
    const int most = kTreeTileRows / a.G;
    p->m_tiles = (a.n_t + most - 1) / most;
    p->tokens = (a.n_t + p->m_tiles - 1) / p->m_tiles;
    p->tile_rows = tree_partial_rows(a.G);
    p->key_rows = kTcKeys;
    p->tpu = (a.n + kTcKeys - 1) / kTcKeys;
    p->T = (long long)a.units * p->tpu;
    p->teams = (int)std::min<long long>(p->T, std::max(1, blocks / ((p->m_tiles + 1) / 2)));
}

cudaError_t launch_tree_tc(const TreeArgs& a, const TreePlan& plan, cudaStream_t stream) {
    EncodeFn encode = nullptr;
    cudaError_t e = get_encode(&encode);
    if (e != cudaSuccess) return e;
    alignas(64) CUtensorMap tq;
    const cuuint64_t d = (cuuint64_t)a.D;
    cuuint64_t dims[4] = {d, (cuuint64_t)a.Hq, (cuuint64_t)a.n_t, (cuuint64_t)a.B};
    cuuint64_t strides[3] = {d * 2, (cuuint64_t)a.Hq * d * 2, (cuuint64_t)a.n_t * a.Hq * d * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)a.G, (cuuint32_t)plan.tokens, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    if (encode(&tq, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    TreeTcArgs x;
    x.a = a;
    x.p = plan;
    x.plane_rows = a.plane_bytes / (a.D * 2);
    x.krow0 = a.krow0;
    x.vrow0 = a.vrow0;
    const CUtensorMap& tkv = *reinterpret_cast<const CUtensorMap*>(a.pool_map);
    const CUtensorMap& tail = *reinterpret_cast<const CUtensorMap*>(a.pool_map_tail);
    const unsigned blocks = (unsigned)(plan.teams * ((plan.m_tiles + 1) / 2));
    if (a.D == 128) tree_attention_tc<128><<<blocks, kTcThreads, TcShape<128>::SMEM_BYTES, stream>>>(tq, tkv, tail, x);
    else tree_attention_tc<64><<<blocks, kTcThreads, TcShape<64>::SMEM_BYTES, stream>>>(tq, tkv, tail, x);
    return cudaGetLastError();
}

}  // namespace kvs
