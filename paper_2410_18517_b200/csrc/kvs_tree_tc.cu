// Attention of a tree of drafted tokens on the 5th-generation tensor cores (bf16 storage, head size 64 or 128).
// The mathematics and the masks are those of kvs_tree.cu.
//
// One thread block = one query tile (up to 128 rows: the G heads of as many drafts as fit) walking over key tiles
// of 64; two blocks share an SM.
//   warp 4 (one lane)  TMA producer: the query tile per piece, K and V tiles, kTcStages stages each
//   warp 5 (one lane)  MMA issuer:   S = Q K^T into one of two score buffers (S of tile j+1 runs during the softmax of
//                                    tile j), O += P V with P as bf16 read from tensor memory
//   warps 0..3         softmax: one thread per query row (= tensor-memory lane), all 64 keys of the tile; warps whose
//                      lanes hold no query row stay out of it
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

constexpr int kTcSoftmaxWarps = 4;
constexpr int kTcThreads = (kTcSoftmaxWarps + 2) * 32;
constexpr int kTcKeys = 64;
constexpr int kTcStages = 2;
constexpr int kTcQBlock = kTreeTileRows * 128;   // one swizzled block of Q: 128 rows x 64 bf16 columns
constexpr int kTcKvBlock = kTcKeys * 128;        // one swizzled block of K or V: 64 rows x 64 bf16 columns
constexpr uint32_t kTcTmemCols = 256;            // two score buffers [0,64), [64,128); O: [128,128+D)

template <int D>
struct TcShape {
    static constexpr int HALVES = D / 64;
    static constexpr int Q_BYTES = HALVES * kTcQBlock;
    static constexpr int KV_BYTES = HALVES * kTcKvBlock;
    static constexpr int SMEM_BYTES = 1024 + Q_BYTES + 2 * kTcStages * KV_BYTES + 512;
};

struct TreeTcArgs {
    TreeArgs a;
    TreePlan p;
    long long krow0, vrow0;      // first row of the slot's planes in the pool-wide row numbering
    long long plane_rows;
};

// The pieces of one team, in order; every role of the block walks the same ones.
struct Pieces {
    const TreeTcArgs& x;
    long long gt, t1;
    long long u;
    int ti0, nt, n;
    bool whole;
    __device__ Pieces(const TreeTcArgs& args, int team) : x(args) {
        gt = (long long)team * x.p.T / x.p.teams;
        t1 = (long long)(team + 1) * x.p.T / x.p.teams;
    }
    __device__ bool next() {
        while (gt < t1) {
            u = gt / x.p.tpu;
            ti0 = (int)(gt - u * x.p.tpu);
            const int piece = (int)min((long long)(x.p.tpu - ti0), t1 - gt);
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

// p = 2^(x * scale - m_ref) of 16 scores as bf16 pairs, 0 where the key's bit in `vis` is not set (MASK).
template <bool MASK, int OFF>
__device__ __forceinline__ float weights_chunk(const float (&x)[64], float scale_log2, float m_ref, unsigned long long vis,
                                               uint32_t (&w)[8]) {
    const float2 sc = make_float2(scale_log2, scale_log2), nm = make_float2(-m_ref, -m_ref);
    const uint32_t bits = (uint32_t)(vis >> OFF);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const float2 t = __ffma2_rn(make_float2(x[OFF + i], x[OFF + i + 1]), sc, nm);
        float2 p = make_float2(fast_exp2(t.x), fast_exp2(t.y));
        if (MASK) {
            p.x = (bits >> i) & 1u ? p.x : 0.f;
            p.y = (bits >> (i + 1)) & 1u ? p.y : 0.f;
        }
        sum = __fadd2_rn(sum, p);
        w[i >> 1] = pack2_bf16(p.x, p.y);
    }
    return sum.x + sum.y;
}

// The weights of a tile's 64 keys, as they go to tensor memory (key k -> column k / 2 at `taddr`); returns their sum.
template <bool MASK>
__device__ __forceinline__ float weights_tile(const float (&x)[64], float scale_log2, float m_ref, unsigned long long vis, uint32_t taddr) {
    uint32_t w[8];
    float l = weights_chunk<MASK, 0>(x, scale_log2, m_ref, vis, w);
    tmem_st8(taddr, w);
    l += weights_chunk<MASK, 16>(x, scale_log2, m_ref, vis, w);
    tmem_st8(taddr + 8, w);
    l += weights_chunk<MASK, 32>(x, scale_log2, m_ref, vis, w);
    tmem_st8(taddr + 16, w);
    l += weights_chunk<MASK, 48>(x, scale_log2, m_ref, vis, w);
    tmem_st8(taddr + 24, w);
    return l;
}

__device__ __forceinline__ uint32_t nonfinite16(uint32_t w) {      // mask of the halves of w that are Inf or NaN
    return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

template <int D>
__global__ void __launch_bounds__(kTcThreads, 2)
    tree_attention_tc(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_kv,
                      const __grid_constant__ TreeTcArgs x) {
    using S = TcShape<D>;
    constexpr int NS = kTcStages, kKv = S::KV_BYTES;
    const TreeArgs& a = x.a;
    const TreePlan& p = x.p;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* sQ = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char* sK = sQ + S::Q_BYTES;
    unsigned char* sV = sK + NS * kKv;
    uint64_t* bars = reinterpret_cast<uint64_t*>(sV + NS * kKv);
    uint64_t* q_full = bars;
    uint64_t* q_free = bars + 1;       // every S of a piece is done
    uint64_t* o_full = bars + 2;       // [2] by tile parity: the tile's PV is in O
    uint64_t* s_full = bars + 4;       // [2] per score buffer
    uint64_t* p_full = bars + 6;       // [2] one arrival per active softmax thread
    uint64_t* drain = bars + 12;
    uint64_t* k_full = bars + 16;      // [NS] each
    uint64_t* k_empty = k_full + NS;
    uint64_t* v_full = k_empty + NS;
    uint64_t* v_empty = v_full + NS;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(v_empty + NS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);    // [2]; the second bounds the drains
    volatile int* broken = abort_flag + 2;                                        // [2] by piece parity

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int team = blockIdx.x / p.m_tiles, mt = blockIdx.x - team * p.m_tiles;
    const int tok0 = mt * p.tokens, rows = min(p.tokens, a.n_t - tok0) * a.G;
    const int quarters = (p.tokens * a.G + 31) / 32;        // tensor-memory lane quarters that hold query rows
    const uint32_t active = quarters * 32;                  // softmax threads at work

    if (tid == 0) {
        for (int i = 0; i < 16 + 4 * NS; ++i) mbar_init(&bars[i], 1);
        mbar_init(&p_full[0], active);
        mbar_init(&p_full[1], active);
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
    const uint32_t tmem_s = tmem_base, tmem_o = tmem_base + 128;

    // Every role keeps its own count t of key tiles done in earlier pieces: tile t uses K/V stage t % NS and score
    // buffer t & 1.
    if (warp == kTcSoftmaxWarps) {
        // ------------------------------ TMA producer ------------------------------
        if (lane == 0) {
            const uint32_t q_bytes = (uint32_t)(S::HALVES * p.tokens * a.G * 128);
            int t = 0, pc = 0;
            bool ok = true;
            for (Pieces pi(x, team); ok && pi.next(); ++pc) {
                const int b = (int)(pi.u / a.Hkv), hk = (int)(pi.u - (long long)b * a.Hkv);
                for (int j = 0; j < pi.nt; ++j, ++t) {
                    const int st = t % NS;
                    const uint32_t prev = (uint32_t)(t / NS - 1) & 1u;
                    long long row = pi.u * a.row_stride + (long long)(pi.ti0 + j) * kTcKeys;
                    if (!KVS_BOUNDS_OK(row, kTcKeys, x.plane_rows, a.status)) row = 0;
                    if (t >= NS && !mbar_wait_bounded(&k_empty[st], prev, abort_flag, a.status, a.wait_ns)) { ok = false; break; }
                    mbar_arrive_expect_tx(&k_full[st], kKv);
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h)
                        tma_load_2d_pf(sK + st * kKv + h * kTcKvBlock, &tmap_kv, h * 64, (int)(x.krow0 + row), &k_full[st]);
                    if (j == 0) {
                        if (pc >= 1 && !mbar_wait_bounded(q_free, (uint32_t)(pc - 1) & 1u, abort_flag, a.status, a.wait_ns)) {
                            ok = false;
                            ++t;       // this tile's K copy is in flight, its V copy is not
                            break;
                        }
                        mbar_arrive_expect_tx(q_full, q_bytes);
#pragma unroll
                        for (int h = 0; h < S::HALVES; ++h) tma_load_4d(sQ + h * kTcQBlock, &tmap_q, h * 64, hk * a.G, tok0, b, q_full);
                    }
                    if (t >= NS && !mbar_wait_bounded(&v_empty[st], prev, abort_flag, a.status, a.wait_ns)) {
                        ok = false;
                        ++t;
                        break;
                    }
                    mbar_arrive_expect_tx(&v_full[st], kKv);
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h)
                        tma_load_2d_pf(sV + st * kKv + h * kTcKvBlock, &tmap_kv, h * 64, (int)(x.vrow0 + row), &v_full[st]);
                }
            }
            if (!ok || abort_flag[0] != 0) {
                // Gave up: wait (bounded) for the copies already issued, so that none is in flight into this block's
                // shared memory when it exits.  (The last tile may lack its V copy: that wait then sees the
                // stage's previous phase, or runs into its limit.)
                for (int j = max(0, t - NS); j < t; ++j) {
                    mbar_wait_bounded(&k_full[j % NS], (uint32_t)(j / NS) & 1u, abort_flag + 1, a.status, a.wait_ns);
                    mbar_wait_bounded(&v_full[j % NS], (uint32_t)(j / NS) & 1u, abort_flag + 1, a.status, a.wait_ns);
                }
                if (pc > 0 || t > 0) mbar_wait_bounded(q_full, (uint32_t)max(pc - (ok ? 1 : 0), 0) & 1u, abort_flag + 1, a.status, a.wait_ns);
            }
        }
    } else if (warp == kTcSoftmaxWarps + 1) {
        // ------------------------------ MMA issuer ------------------------------
        // Order on the tensor pipe: S_0, then per tile j: S_{j+1}, PV_j.  The pipe runs one thread's MMAs in issue
        // order, so S_{j+1} overwrites its buffer only after PV_{j-1} has read P_{j-1} from it.
        if (lane == 0) {
            const uint32_t idesc_s = instr_desc_bf16(0, kTcKeys);
            const uint32_t idesc_o = instr_desc_bf16(1, D);
            const uint32_t q_addr = smem_u32(sQ), k_addr = smem_u32(sK), v_addr = smem_u32(sV);
            auto issue_s = [&](int t, bool last) {
                const int st = t % NS;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t qoff = (ks >> 2) * kTcQBlock + (ks & 3) * 32;
                    const uint32_t koff = st * kKv + (ks >> 2) * kTcKvBlock + (ks & 3) * 32;
                    umma_bf16(tmem_s + (t & 1) * kTcKeys, smem_desc_sw128(q_addr + qoff, 16, 1024),
                              smem_desc_sw128(k_addr + koff, 16, 1024), idesc_s, ks > 0);
                }
                umma_commit(&s_full[t & 1]);
                umma_commit(&k_empty[st]);
                if (last) umma_commit(q_free);
            };
            auto wait = [&](uint64_t* bar, uint32_t ph) { return mbar_wait_bounded(bar, ph & 1u, abort_flag, a.status, a.wait_ns); };
            int t = 0, pc = 0;
            bool ok = true;
            for (Pieces pi(x, team); ok && pi.next(); ++pc) {
                ok = wait(q_full, pc) && wait(&k_full[t % NS], t / NS);
                if (!ok) break;
                tc_fence_after();
                issue_s(t, pi.nt == 1);
                for (int j = 0; j < pi.nt; ++j, ++t) {
                    if (j + 1 < pi.nt) {
                        ok = wait(&k_full[(t + 1) % NS], (t + 1) / NS);
                        if (!ok) break;
                        tc_fence_after();
                        issue_s(t + 1, j + 2 == pi.nt);
                    }
                    const int st = t % NS;
                    ok = wait(&p_full[t & 1], t >> 1) && wait(&v_full[st], t / NS);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int ks = 0; ks < kTcKeys / 16; ++ks) {
                        const uint64_t vdesc = smem_desc_sw128(v_addr + st * kKv + ks * 16 * 128, kTcKvBlock, 1024);
                        umma_bf16_ts(tmem_o, tmem_s + (t & 1) * kTcKeys + ks * 8, vdesc, idesc_o, (j > 0) || (ks > 0));
                    }
                    umma_commit(&o_full[t & 1]);
                    umma_commit(&v_empty[st]);
                }
            }
            if (!ok) {     // the MMAs already issued must be done before the block gives its memory back
                umma_commit(drain);
                mbar_wait_bounded(drain, 0, abort_flag + 1, a.status, a.wait_ns);
            }
        }
    } else if (warp < quarters) {
        // ------------------------------ softmax / output rows ------------------------------
        const int r = tid;                                   // query row in the tile = tensor-memory lane
        const uint32_t lane_addr = (uint32_t)(warp * 32) << 16;
        const uint32_t to = tmem_o + lane_addr;
        const bool real = r < rows;                          // lanes past the last row hold no query: their scores are junk
        const int tok = tok0 + min(r, rows - 1) / a.G, g = min(r, rows - 1) % a.G;
        const unsigned long long all = a.n_t >= 64 ? ~0ull : (1ull << a.n_t) - 1;
        auto wait = [&](uint64_t* bar, uint32_t ph) { return mbar_wait_bounded(bar, ph & 1u, abort_flag, a.status, a.wait_ns); };
        int t = 0, pc = 0;
        bool ok = true;
        for (Pieces pi(x, team); ok && pi.next(); ++pc) {
            const int b = (int)(pi.u / a.Hkv), hk = (int)(pi.u - (long long)b * a.Hkv);
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
                float xs[64];
                __syncwarp();                                // the warp's tensor-memory accesses are made together
                tmem_ld64(sb, xs);
                unsigned long long vis = ~0ull;
                float mx = -INFINITY;
                if (mask) {
                    const int off = key0 - ctx;
                    if (off >= 0) vis = off < 64 ? sees >> off : 0ull;
                    else if (off > -64) vis = sees << -off | ((1ull << -off) - 1ull);
                    // Clean the V tile (see the head of this file).  Only behind the wait above: S of this tile is
                    // done, so PV of the tile that had this V stage before is too, and v_full cannot be a phase
                    // behind the one waited for.
                    const int st = t % NS;
                    ok = wait(&v_full[st], t / NS);
                    if (!ok) break;
                    for (int i = tid; i < kKv / 16; i += active) {
                        const int key = key0 + (i * 16 % kTcKvBlock) / 128;
                        if (key < ctx) continue;
                        uint4* q4 = reinterpret_cast<uint4*>(sV + st * kKv + i * 16);
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
#pragma unroll
                    for (int i = 0; i < 64; ++i) mx = fmaxf(mx, (vis >> i) & 1ull ? xs[i] : -INFINITY);
                } else {
                    float m4[4] = {xs[0], xs[1], xs[2], xs[3]};
#pragma unroll
                    for (int i = 4; i < 60; i += 8)
#pragma unroll
                        for (int c = 0; c < 4; ++c) m4[c] = fmax3(m4[c], xs[i + c], xs[i + 4 + c]);
                    mx = fmax3(fmax3(m4[0], m4[1], fmaxf(m4[2], m4[3])), fmaxf(xs[60], xs[61]), fmaxf(xs[62], xs[63]));
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
                l += mask ? weights_tile<true>(xs, a.scale_log2, m_ref, vis, sb) : weights_tile<false>(xs, a.scale_log2, m_ref, vis, sb);
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
                        const __nv_bfloat16* vr = reinterpret_cast<const __nv_bfloat16*>(a.vplane) + (pi.u * a.row_stride + key) * D + c;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float v = __bfloat162float(vr[i]);
                            if (!isfinite(v)) o[i] += v;
                        }
                    }
                }
                if (real && pi.whole) {
                    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + orow * D + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[i] = make_uint4(pack2_bf16(o[8 * i] * inv, o[8 * i + 1] * inv), pack2_bf16(o[8 * i + 2] * inv, o[8 * i + 3] * inv),
                                            pack2_bf16(o[8 * i + 4] * inv, o[8 * i + 5] * inv), pack2_bf16(o[8 * i + 6] * inv, o[8 * i + 7] * inv));
                } else if (real) {
                    float4* dst = reinterpret_cast<float4*>(a.part_o + prow * D + c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
            }
            if (!pi.whole && real) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(m_ref, l);
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
    const unsigned blocks = (unsigned)(plan.teams * plan.m_tiles);
    if (a.D == 128) tree_attention_tc<128><<<blocks, kTcThreads, TcShape<128>::SMEM_BYTES, stream>>>(tq, tkv, x);
    else tree_attention_tc<64><<<blocks, kTcThreads, TcShape<64>::SMEM_BYTES, stream>>>(tq, tkv, x);
    return cudaGetLastError();
}

}  // namespace kvs
