// Attention of a tree of drafted tokens on the 5th-generation tensor cores (bf16 storage, head size 64 or 128).
// The mathematics and the masks are those of kvs_tree.cu.
//
// One thread block = one query tile (up to 128 rows: the G heads of as many drafts as fit) walking over key tiles
// of 64; two blocks share an SM, so that one block's softmax runs beside the other's products.
//   warps 0..3         softmax: one thread per query row (= tensor-memory lane), the 64 keys of a tile; warps whose
//                      lanes hold no query row stay out of it
//   warp 4 (one lane)  TMA producer: the query tile per piece; K and V tiles through one ring (K0 V0 K1 V1 ...)
//   warp 5             MMA issuer: S = Q K^T into one of two score buffers (S of tile t+1 runs during the softmax of
//                      tile t), O += P V with P = hi + lo (two bf16 terms) read from tensor memory.  The whole warp walks
//                      the tiles and an elected lane issues: operands are then in uniform registers (issued from a one-lane
//                      branch the sixteen MMAs of a 128-key tile took 1700 cycles instead of 1200)
// Bound: up to 128 query rows per kv-head HBM (32 heads, B = 8, n = 4096, 16 drafts: 537 MB in 87 us, 6.2 TB/s, tensor pipe
// busy 64 % of the time).  Above that the tensor pipe more than anything: at 256 rows (32q/8kv, B = 4, n = 32768, 64
// drafts: 160 us, 0.86 PFLOP/s and half again as much issued for the second term of P) it is busy 74 % of the time at the
// 1.54 GHz the power cap leaves, issue slots 48, the special-function unit 50; an S product of 64 keys reads 6 KiB of shared
// memory per 32 tensor cycles, more than the 128 bytes a cycle there are (Q is read again for every tile).
// Measured against this layout at 256 rows while P had one term (147 us with the combine step, now 174): one block per SM whose
// two softmax groups take a query tile each and share K/V tiles of 128 keys, 156 us (a score buffer is free only after the
// product that reads its weights, and S then waits for softmax, PV and S in a row); one block per SM with 128-key tiles, two
// score buffers and two threads per row, 177; a quarter of the exp2 by a polynomial on the FMA pipe, 151; two stages per
// operand instead of the ring of five, 147; K/V fetched before the wait for the previous kernel, 150.
// P goes into the second contraction as two bf16 terms, like the prefill kernel's: a weight is then off by 2^-16 of itself at
// most.  With one term (2^-8) an element with large cancelling shares is off by several of its own rounding steps, which
// shows at any length (70 keys: nine times the bound).  Per call, one term / two: 32 heads, B = 8, n = 4096, 16 drafts
// 102 / 111 us; 32q/8kv, B = 4, n = 32768, 64 drafts 182 / 211; B = 4, n = 8192, 32 drafts 52.3 / 52.6.
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

constexpr int kTcSoftmaxWarps = 4;
constexpr int kTcThreads = (kTcSoftmaxWarps + 2) * 32;
constexpr int kTcKeys = 64;
constexpr int kTcQBlock = kTreeTileRows * 128;   // one swizzled block of Q: 128 rows x 64 bf16 columns
constexpr int kTcKvBlock = kTcKeys * 128;        // one swizzled block of K or V: 64 rows x 64 bf16 columns
constexpr int kTcTailRows = 16;                  // rows per copy at the partly filled end of a unit
constexpr uint32_t kTcTmemCols = 256;            // two score buffers [0,64), [64,128); O: [128,128+D)

template <int D>
struct TcShape {
    static constexpr int HALVES = D / 64;
    static constexpr int Q_BYTES = HALVES * kTcQBlock;
    static constexpr int KV_BYTES = HALVES * kTcKvBlock;
    // K and V buffers: as many as leave room for two blocks (and the 1 KiB the system keeps of each) on an SM's 228 KiB
    static constexpr int RING = HALVES == 2 ? 5 : 12;
    static constexpr int SMEM_BYTES = Q_BYTES + RING * KV_BYTES + 512;
    static_assert(2 * (SMEM_BYTES + 1024) <= 228 * 1024, "two blocks per SM");
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

// The weights p = 2^(x * scale - m_ref) of 32 scores, 0 where the key's bit in `vis` is not set (MASK), as they go to
// tensor memory: p = hi + lo in bf16, two keys per column, hi from `taddr` and lo from `taddr + kTcKeys / 2` on.  Returns
// their sum.
template <bool MASK>
__device__ __forceinline__ float weights32(const float (&x)[32], float scale_log2, float m_ref, uint32_t vis, uint32_t taddr) {
    const float2 sc = make_float2(scale_log2, scale_log2), nm = make_float2(-m_ref, -m_ref), minus1 = make_float2(-1.f, -1.f);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t hi[16], lo[16];
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        const float2 t = __ffma2_rn(make_float2(x[i], x[i + 1]), sc, nm);
        float2 p = make_float2(fast_exp2(t.x), fast_exp2(t.y));
        if (MASK) {
            p.x = (vis >> i) & 1u ? p.x : 0.f;
            p.y = (vis >> (i + 1)) & 1u ? p.y : 0.f;
        }
        sum[(i >> 1) & 1] = __fadd2_rn(sum[(i >> 1) & 1], p);
        const uint32_t h = pack2_bf16(p.x, p.y);
        hi[i >> 1] = h;
        const float2 r = __ffma2_rn(make_float2(__uint_as_float(h << 16), __uint_as_float(h & 0xffff0000u)), minus1, p);
        lo[i >> 1] = pack2_bf16(r.x, r.y);
    }
    tmem_st16(taddr, hi);
    tmem_st16(taddr + kTcKeys / 2, lo);
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
__global__ void __launch_bounds__(kTcThreads, 2)
    tree_attention_tc(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_kv,
                      const __grid_constant__ CUtensorMap tmap_tail, const __grid_constant__ TreeTcArgs x) {
    using S = TcShape<D>;
    constexpr int NB = S::RING, kKv = S::KV_BYTES;
    const TreeArgs& a = x.a;
    const TreePlan& p = x.p;
    extern __shared__ __align__(1024) unsigned char sQ[];       // the 128-byte swizzle counts from 1024-byte boundaries
    if ((smem_u32(sQ) & 1023u) != 0u) {
        if (threadIdx.x == 0) atomicExch(a.status, kDevBounds);
        return;
    }
    unsigned char* ring = sQ + S::Q_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + NB * kKv);
    uint64_t* q_full = bars;
    uint64_t* q_free = bars + 1;       // every S of a piece is done
    uint64_t* o_full = bars + 2;       // [2] by tile parity: the tile's PV is in O
    uint64_t* s_full = bars + 4;       // [2] per score buffer
    uint64_t* p_full = bars + 6;       // [2] one arrival per active softmax thread
    uint64_t* drain = bars + 8;
    uint64_t* full = bars + 9;         // [NB]
    uint64_t* empty = full + NB;       // [NB]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(empty + NB);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);    // [2]; the second bounds the drains
    volatile int* broken = abort_flag + 2;                                        // [2] by piece parity

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int team = blockIdx.x / p.m_tiles, mt = blockIdx.x - team * p.m_tiles;
    const int tok0 = mt * p.tokens, rows = min(p.tokens, a.n_t - tok0) * a.G;
    const int quarters = (p.tokens * a.G + 31) / 32;        // tensor-memory lane quarters that hold query rows
    const uint32_t active = quarters * 32;                  // softmax threads at work

    if (tid == 0) {
        for (int i = 0; i < 9 + 2 * NB; ++i) mbar_init(&bars[i], 1);
        mbar_init(&p_full[0], active);
        mbar_init(&p_full[1], active);
        abort_flag[0] = abort_flag[1] = broken[0] = broken[1] = 0;
        fence_mbar_init();
        prefetch_map(&tmap_q);
        prefetch_map(&tmap_kv);
        prefetch_map(&tmap_tail);
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
    const uint32_t tmem_s = tmem_base, tmem_o = tmem_base + 128;
    pdl_wait();                  // everything above runs beside the end of the previous kernel
    pdl_launch_dependents();

    // Every role keeps its own count t of key tiles done in earlier pieces.  Tile t has K in ring entry 2 t and V in
    // 2 t + 1 and uses score buffer t & 1; entry e lies in buffer e % NB, whose barriers are then in phase (e / NB) & 1.
    auto wait = [&](uint64_t* bar, uint32_t ph) { return mbar_wait_bounded(bar, ph & 1u, abort_flag, a.status, a.wait_ns); };
    if (warp == kTcSoftmaxWarps) {
        // ------------------------------ TMA producer ------------------------------
        if (lane == 0) {
            const uint32_t q_bytes = (uint32_t)(S::HALVES * p.tokens * a.G * 128);
            int e = 0, pc = 0, q_done = 0;   // ring entries, pieces, pieces whose queries were issued
            bool ok = true;
            for (Pieces pi(x, team); ok && pi.next(); ++pc) {
                const int b = pi.u / a.Hkv, hk = pi.u - b * a.Hkv;
                for (int j = 0; j < pi.nt && ok; ++j) {
                    const int row0 = (pi.ti0 + j) * kTcKeys;
                    const int rows_t = min(kTcKeys, pi.n - row0);
                    // a whole tile in one box per half, a partly filled one in 16-row boxes, only those that hold rows
                    const int tails = rows_t < kTcKeys ? (rows_t + kTcTailRows - 1) / kTcTailRows : 0;
                    const uint32_t bytes = (uint32_t)(tails ? tails * kTcTailRows : kTcKeys) * S::HALVES * 128;
                    long long row = (long long)pi.u * a.row_stride + row0;
                    if (!KVS_BOUNDS_OK(row, tails ? tails * kTcTailRows : kTcKeys, x.plane_rows, a.status)) row = 0;
                    for (int kv = 0; kv < 2; ++kv) {
                        const int st = e % NB;
                        if (e >= NB) ok = wait(&empty[st], e / NB - 1);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&full[st], bytes);
                        const int y = (int)((kv == 0 ? x.krow0 : x.vrow0) + row);
#pragma unroll
                        for (int h = 0; h < S::HALVES; ++h) {
                            unsigned char* dst = ring + st * kKv + h * kTcKvBlock;
                            if (!tails) tma_load_2d_pf(dst, &tmap_kv, h * 64, y, &full[st]);
                            for (int i = 0; i < tails; ++i)
                                tma_load_2d_pf(dst + i * kTcTailRows * 128, &tmap_tail, h * 64, y + i * kTcTailRows, &full[st]);
                        }
                        ++e;
                        if (kv == 0 && j == 0) {      // the queries, behind the piece's first K tile
                            if (pc >= 1) ok = wait(q_free, pc - 1);
                            if (!ok) break;
                            mbar_arrive_expect_tx(q_full, q_bytes);
#pragma unroll
                            for (int h = 0; h < S::HALVES; ++h) tma_load_4d(sQ + h * kTcQBlock, &tmap_q, h * 64, hk * a.G, tok0, b, q_full);
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
                if (q_done > 0) mbar_wait_bounded(q_full, (uint32_t)(q_done - 1) & 1u, abort_flag + 1, a.status, a.wait_ns);
            }
        }
    } else if (warp == kTcSoftmaxWarps + 1) {
        // ------------------------------ MMA issuer ------------------------------
        // Order on the tensor pipe: S_0, then per tile t: S_{t+1}, PV_t.  The pipe runs one thread's MMAs in issue
        // order, so S_{t+1} overwrites its buffer only after PV_{t-1} has read P_{t-1} from it.
        const uint32_t idesc_s = instr_desc_bf16(0, kTcKeys);
        const uint32_t idesc_o = instr_desc_bf16(1, D);
        const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
        const bool leader = elect_one();
        // descriptors of the buffers' starts; steps inside a buffer are added in units of 16 bytes
        const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ), 16, 1024);
        const uint64_t k_desc = smem_desc_sw128(smem_u32(ring), 16, 1024);
        // V is MN-major: 64 head-dim columns contiguous per key row, the other 64 (D = 128) one column block (LBO)
        // away; 8-key groups 1024 bytes (SBO) apart
        const uint64_t v_desc = smem_desc_sw128(smem_u32(ring), kTcKvBlock, 1024);
        auto all_wait = [&](uint64_t* bar, uint32_t ph) { return __all_sync(0xffffffffu, wait(bar, ph)) != 0; };   // one answer for the warp
        auto issue_s = [&](int t, bool last) {
            const int st = 2 * t % NB;
            const uint64_t k = k_desc + (uint32_t)st * (kKv / 16);
            const uint32_t d = tmem + (t & 1) * kTcKeys;
            if (leader) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_bf16(d, q_desc + ((ks >> 2) * kTcQBlock + (ks & 3) * 32) / 16, k + ((ks >> 2) * kTcKvBlock + (ks & 3) * 32) / 16,
                              idesc_s, ks > 0);
                umma_commit(&s_full[t & 1]);
                umma_commit(&empty[st]);
                if (last) umma_commit(q_free);
            }
            __syncwarp();
        };
        int t = 0, pc = 0;
        bool ok = true;
        for (Pieces pi(x, team); ok && pi.next(); ++pc) {
            ok = all_wait(q_full, pc) && all_wait(&full[2 * t % NB], 2 * t / NB);
            if (!ok) break;
            tc_fence_after();
            issue_s(t, pi.nt == 1);
            for (int j = 0; j < pi.nt; ++j, ++t) {
                if (j + 1 < pi.nt) {
                    ok = all_wait(&full[(2 * t + 2) % NB], (2 * t + 2) / NB);
                    if (!ok) break;
                    tc_fence_after();
                    issue_s(t + 1, j + 2 == pi.nt);
                }
                const int st = (2 * t + 1) % NB;
                ok = all_wait(&full[st], (2 * t + 1) / NB) && all_wait(&p_full[t & 1], t >> 1);
                if (!ok) break;
                tc_fence_after();
                const uint64_t v = v_desc + (uint32_t)st * (kKv / 16);
                const uint32_t o = tmem + 128, w = tmem + (t & 1) * kTcKeys;
                if (leader) {
#pragma unroll
                    for (int ks = 0; ks < kTcKeys / 16; ++ks) {
                        umma_bf16_ts(o, w + ks * 8, v + ks * 16 * 128 / 16, idesc_o, ks > 0 ? 1 : j > 0);             // hi
                        umma_bf16_ts(o, w + kTcKeys / 2 + ks * 8, v + ks * 16 * 128 / 16, idesc_o, 1);                // lo
                    }
                    umma_commit(&o_full[t & 1]);
                    umma_commit(&empty[st]);
                }
                __syncwarp();
            }
        }
        if (!ok && leader) {     // the MMAs already issued must be done before the block gives its memory back
            umma_commit(drain);
            mbar_wait_bounded(drain, 0, abort_flag + 1, a.status, a.wait_ns);
        }
    } else if (warp < quarters) {
        // ------------------------------ softmax / output rows ------------------------------
        const int r = tid;                                   // query row in the tile = tensor-memory lane
        const uint32_t lane_addr = (uint32_t)(warp * 32) << 16;
        const uint32_t to = tmem_o + lane_addr;
        const bool real = r < rows;                          // lanes past the last row hold no query: their scores are junk
        const int tok = tok0 + min(r, rows - 1) / a.G, g = min(r, rows - 1) % a.G;
        const unsigned long long all = a.n_t >= 64 ? ~0ull : (1ull << a.n_t) - 1;
        int t = 0, pc = 0;
        bool ok = true;
        for (Pieces pi(x, team); ok && pi.next(); ++pc) {
            const int b = pi.u / a.Hkv, hk = pi.u - b * a.Hkv;
            const int ctx = pi.n - a.n_t;                    // rows every query sees
            const unsigned long long sees =
                a.mask ? a.mask[(long long)b * a.n_t + tok] & all : (tok >= 63 ? ~0ull : (2ull << tok) - 1);
            float m_ref = -1.0e30f, l = 0.f;                 // p is taken relative to m_ref (log2 domain)
            for (int j = 0; j < pi.nt; ++j, ++t) {
                const int sbuf = t & 1;
                const int key0 = (pi.ti0 + j) * kTcKeys;
                const bool mask = key0 + kTcKeys > ctx;      // the tile holds drafts or rows past the end
                ok = wait(&s_full[sbuf], t >> 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t sb = tmem_s + lane_addr + sbuf * kTcKeys;
                // Both halves of the scores are asked for at once: beside running MMAs, which read and write tensor
                // memory through the same ports, a load takes 250 to 400 cycles.
                float x0[32], x1[32];
                __syncwarp();                                // the warp's tensor-memory accesses are made together
                tmem_ld32_issue(sb, x0);
                tmem_ld32_issue(sb + 32, x1);
                tmem_ld_wait(x0);
                tmem_ld_wait(x1);
                unsigned long long vis = ~0ull;
                float mx;
                if (mask) {
                    vis = visible64(sees, key0 - ctx);
                    // Clean the V tile (see the head of this file).  Only behind the wait above: S of this tile is
                    // done, so whatever had this buffer before has been used, and its barrier cannot be a phase
                    // behind the one waited for.
                    const int st = (2 * t + 1) % NB;
                    ok = wait(&full[st], (2 * t + 1) / NB);
                    if (!ok) break;
                    for (int i = tid; i < kKv / 16; i += active) {
                        const int key = key0 + (i * 16 % kTcKvBlock) / 128;
                        if (key < ctx) continue;
                        uint4* q4 = reinterpret_cast<uint4*>(ring + st * kKv + i * 16);
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
                    __syncwarp();
                    mx = fmaxf(max32<true>(x0, (uint32_t)vis), max32<true>(x1, (uint32_t)(vis >> 32)));
                } else {
                    mx = fmaxf(max32<false>(x0, 0u), max32<false>(x1, 0u));
                }
                mx *= a.scale_log2;
                // The reference maximum only moves when the new one is more than 8 (a factor 256) above it; then
                // the output row and the sum so far are rescaled, once every PV issued so far has landed in O.
                const bool grow = real && mx > m_ref + 8.0f;
                if (__any_sync(0xffffffffu, grow)) {
                    const float m_new = grow ? mx : m_ref;
                    const float alpha = fast_exp2(m_ref - m_new);
                    if (j > 0) {
                        ok = wait(&o_full[(t - 1) & 1], (uint32_t)(t - 1) >> 1);
                        if (!ok) break;
                        tc_fence_after();
                        __syncwarp();
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) tmem_scale32(to + c, alpha);
                    }
                    l *= alpha;
                    m_ref = m_new;
                }
                if (mask) {
                    l += weights32<true>(x0, a.scale_log2, m_ref, (uint32_t)vis, sb);
                    l += weights32<true>(x1, a.scale_log2, m_ref, (uint32_t)(vis >> 32), sb + 16);
                } else {
                    l += weights32<false>(x0, a.scale_log2, m_ref, 0u, sb);
                    l += weights32<false>(x1, a.scale_log2, m_ref, 0u, sb + 16);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                mbar_arrive(&p_full[sbuf]);
            }
            if (!ok) break;
            // the last tile's PV group is behind every other MMA of the piece on the pipe
            ok = wait(&o_full[(t - 1) & 1], (uint32_t)(t - 1) >> 1);
            if (!ok) break;
            tc_fence_after();
            const bool patch = broken[pc & 1] == pc + 1;
            const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;        // nothing visible: 0
            const long long orow = ((long long)b * a.n_t + tok) * a.Hq + hk * a.G + g;
            const bool inside = KVS_BOUNDS_OK(orow, 1, (long long)a.B * a.n_t * a.Hq, a.status);
            const long long prow = ((2ll * team + (pi.ti0 == 0 ? 1 : 0)) * p.m_tiles + mt) * p.tile_rows + r;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                float o[32];
                __syncwarp();
                tmem_ld32(to + c, o);
                if (patch) {
                    // a draft row this query sees holds Inf or NaN: its elements go into the sum as they are
                    for (int d = 0; d < a.n_t; ++d) {
                        const int key = ctx + d;
                        if (!(sees >> d & 1ull) || key < pi.ti0 * kTcKeys || key >= (pi.ti0 + pi.nt) * kTcKeys) continue;
                        const __nv_bfloat16* vr = reinterpret_cast<const __nv_bfloat16*>(a.vplane) + ((long long)pi.u * a.row_stride + key) * D + c;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float v = __bfloat162float(vr[i]);
                            if (!isfinite(v)) o[i] += v;
                        }
                    }
                }
                if (real && pi.whole && inside) {
                    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + orow * D + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[i] = make_uint4(pack2_bf16(o[8 * i] * inv, o[8 * i + 1] * inv), pack2_bf16(o[8 * i + 2] * inv, o[8 * i + 3] * inv),
                                            pack2_bf16(o[8 * i + 4] * inv, o[8 * i + 5] * inv), pack2_bf16(o[8 * i + 6] * inv, o[8 * i + 7] * inv));
                } else if (real && KVS_BOUNDS_OK(prow, 1, tree_piece_rows(a.G), a.status)) {
                    float4* dst = reinterpret_cast<float4*>(a.part_o + prow * D + c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
            }
            if (!pi.whole && real && KVS_BOUNDS_OK(prow, 1, tree_piece_rows(a.G), a.status)) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(m_ref, l);
            tc_fence_before();      // the next piece's first PV waits for this thread's arrival on p_full
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
    p->teams = (int)std::min<long long>(p->T, std::max(1, blocks / p->m_tiles));
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
    const dim3 blocks((unsigned)(plan.teams * plan.m_tiles)), threads(kTcThreads);
    return a.D == 128 ? launch_kernel(tree_attention_tc<128>, blocks, threads, TcShape<128>::SMEM_BYTES, stream, a.programmatic, tq, tkv, tail, x)
                      : launch_kernel(tree_attention_tc<64>, blocks, threads, TcShape<64>::SMEM_BYTES, stream, a.programmatic, tq, tkv, tail, x);
}

}  // namespace kvs
