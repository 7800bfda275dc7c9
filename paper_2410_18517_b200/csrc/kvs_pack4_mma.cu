// Split-K decode attention over a 4-bit cache, bf16 storage: the codes become bf16 tensor-core operands in registers.
//
// Mathematics: S = K q^T, P = 2^(S - max), O = P^T V over the values of the rows (kvs_pack4.cuh), one pass with a running
// maximum and sum, by mma.sync.m16n8k16.  S has 16 keys as rows and the q-heads of a kv-head as columns (no row is padding, no
// operand register holds constant zeros: those cost a move each per product); P's 8 x 8 blocks are transposed on the way to
// the second product, which has the heads as rows.  A product of 16 rows costs what one of 8 does, so the rows the heads leave
// free carry the weights' further terms.  P = hi + mid + lo, three bf16 terms:
//   up to four heads:  rows 0..3 hi, 8..11 mid, 4..7 lo, in ONE product (column c of S is head c mod 4, so the lanes of
//                      columns 4..7 have the weights too);
//   five to eight:     rows 0..7 hi and 8..15 mid in one product, lo in a second.
// Two terms would leave 1.5e-6 of the result, three the fp32 rounding.  The products of a chunk start from zero and are added to
// the running state rounded to nearest: an MMA cuts its sum off, and over thousands of rows that would drift.
//
// Fragments: the contraction may take the elements in any order, so lane t of a quad takes group t of its key's row - D/8 bytes in
// a run and one (s, b) pair - and the queries' fragments follow that order.  For P V the columns may be numbered at will:
// column n stands for D/8 neighbouring elements of a row, again of one group; the codes of two keys are interleaved by byte
// permutes.  A code costs 1/2 (shift + and-or + multiply-add); everything else per row is small beside that.
//
// What bounds it: the conversion.  A row of K and V together is D + 32 bytes, 7 cycles of an SM at 6.5 TB/s; its codes take 11 warp
// instructions to become operands, 7 of them on the integer pipe and 4 on the heavy half of the FMA pipe, which take one every
// other cycle and hardly overlap; the MMAs (1.5 a row) and the rest take as long again.  And registers: ten warps put three on one SM
// partition, which leaves a thread 168, and heads of 128 spill (32 bytes stored and 116 loaded a thread, with five to eight heads 68
// and 240; what that costs is not measured).  13B shape, 16 x 40 heads x 8192 rows: 190 to 208 us over several GPUs, 8 x 8 kv-heads x
// 32768 rows 83 to 88; 16 x 8 x 8192 rows with four heads each 48, with eight 61.
//
// Work decomposition (see DecodePlan), pieces, the hand-over between blocks and the combine kernel are those of the other
// split-K kernels.  Rows of a tile are contiguous and come by two 1-D bulk copies, exactly as many as the unit holds.  A tile
// has up to 512 rows, 64 for each of 8 warps: a chunk.  How many it has the plan
// decides (plan_decode_pack4), and with it how many stages the ring has.
#include <algorithm>
#include <type_traits>

#include "kvs_kernels.h"
#include "kvs_pack4.cuh"

namespace kvs {

namespace {

constexpr int kPack4Warps = 8;           // consumer warps
constexpr int kPack4Blocks = 4;          // 16-row blocks a warp takes of a tile at most
constexpr int kPack4TileMax = kPack4Warps * kPack4Blocks * 16;
constexpr int kPack4Stages = 8;          // of the ring at most

template <int D>
struct Pack4Shape {
    static constexpr int WARPS = kPack4Warps;
    static constexpr int RB = Pack4Row<D>::RB;
    static constexpr int QBYTES = 8 * D * 2;               // room for the queries of eight heads
    static constexpr int RING = 2 * (2 * kPack4TileMax * RB + QBYTES);     // two of the largest tiles
    static constexpr int CONSUMERS = WARPS * 32;
    static constexpr int THREADS = CONSUMERS + 64;         // + the producer warp and the hand-over warp
    static constexpr int SCRATCH_FLOATS = WARPS * 8 * (D + 2);
    static constexpr int HANDOVER_FLOATS = 8 * (D + 2);
    static constexpr int SMEM_BYTES = 16 + RING + (SCRATCH_FLOATS + HANDOVER_FLOATS) * 4 + (2 * kPack4Stages + 2) * 8 + 16;
};

struct Pack4KernelArgs {
    const char* q;
    const char* kplane;
    const char* vplane;
    float* part_o;
    float* part_ml;
    float* out;             // [units][G][D], or nullptr: every piece goes to part_o / part_ml
    int* flags;             // [units], zero between launches: 1 = the unit's second piece is written
    int* status;
    int n, row_stride, tpu, G, units, cap, safe_rows;
    int tile_rows;          // a multiple of 16, at most kPack4TileMax
    long long T;
    float scale_log2;
    const int* unit_len;
    const int* n_extra;
    long long plane_bytes;
    unsigned long long wait_ns;
    long long stall_tile;
    unsigned long long* trace;
    const char* k_new;      // the step's new rows (bf16, [units][D]), appended by this kernel (n counts them), or nullptr
    const char* v_new;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_bf16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {      // of an 8 x 8 matrix of 16-bit elements
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

// the next bf16 term of a pair: its value, and what remains of the pair
__device__ __forceinline__ uint32_t take_term(float& x, float& y) {
    const uint32_t t = pack2(x, y);
    x -= bf16_lo(t);
    y -= bf16_hi(t);
    return t;
}

template <int D, bool WIDE>      // WIDE: five to eight q-heads per kv-head
__global__ void __launch_bounds__(Pack4Shape<D>::THREADS, 1) decode_pack4_mma(const Pack4KernelArgs a_in) {
    using S = Pack4Shape<D>;
    constexpr int RB = S::RB, WARPS = S::WARPS;
    const int TN = a_in.tile_rows, kTile = TN * RB, stage_bytes = 2 * kTile + S::QBYTES;
    const int stages = min(kPack4Stages, S::RING / stage_bytes);
    constexpr int KSTEPS = D / 16;        // products of a score block
    constexpr int NB = D / 8;             // column blocks of the output: D/8 elements per column
    constexpr int XW = D / 32;            // words of a row's group (K)
    constexpr int VW = D / 64;            // words of a column's elements (V)
    Pack4KernelArgs a = a_in;
    unsigned long long* tr = a.trace ? a.trace + (size_t)blockIdx.x * kTraceSlots : nullptr;
    if (threadIdx.x == 0) {
        KVS_TRACE_STAMP(tr, kTrEntry);
        KVS_TRACE_VALUE(tr, kTrSm, sm_id());
    }
    bool over = false;    // a replayed launch with an append that would pass the capacity
    if (a.n_extra != nullptr) {
        // a replayed launch: the counter is stable here without a wait (see decode_splitk_mma)
        over = a.n + *a.n_extra > a.cap;
        a.n = min(a.n + *a.n_extra, a.cap);
        a.tpu = (a.n + TN - 1) / TN;
        a.T = (long long)a.units * a.tpu;
    }
    const int G = a.G;
    const int qbytes = G * D * 2;

    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((16u - (smem_u32(smem_raw) & 15u)) & 15u);
    float* scratch = reinterpret_cast<float*>(smem + S::RING);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(scratch + S::SCRATCH_FLOATS);
    uint64_t* empty_bar = full_bar + kPack4Stages;
    uint64_t* tail_bar = empty_bar + kPack4Stages;
    uint64_t* head_bar = tail_bar + 1;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(head_bar + 1);
    float* handover = const_cast<float*>(reinterpret_cast<volatile float*>(abort_flag + 4));

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int NC = gridDim.x;
    const long long t0 = ((long long)blockIdx.x * a.T) / NC;
    const long long t1 = ((long long)(blockIdx.x + 1) * a.T) / NC;

    if (tid == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], WARPS);
        }
        mbar_init(tail_bar, S::CONSUMERS);
        mbar_init(head_bar, 1);
        abort_flag[0] = 0;
        abort_flag[1] = 0;
        fence_mbar_init();
    }
    __syncthreads();

    if (warp == WARPS) {
        // ------------------------------ producer ------------------------------
        // Lane 0 issues the copies; the whole warp packs the step's new rows when the launch carries an append.
        // The barrier of a stage is armed once with its full byte count; K/V and q may be issued apart.
        auto issue = [&](long long gt, int st, bool arm, bool kv, bool qpart) {
            const long long u = gt / a.tpu;
            const int ti = (int)(gt - u * a.tpu);
            const bool with_q = (gt == t0) || (ti == 0);
            const int n_u = a.unit_len ? min(a.unit_len[u], a.cap) : a.n;
            const int rows = min(TN, n_u - ti * TN);          // <= 0: a ragged unit ended before this tile
            const uint32_t bytes = rows > 0 ? (uint32_t)rows * RB : 0u;
            unsigned char* sb = smem + st * stage_bytes;
            if (arm) {
                const uint32_t total = 2 * bytes + (with_q ? qbytes : 0);
                if (total) mbar_arrive_expect_tx(&full_bar[st], total);
                else mbar_arrive(&full_bar[st]);
            }
            if (kv && bytes && gt != a.stall_tile) {
                long long off = (u * a.row_stride + (long long)ti * TN) * RB;
                if (!KVS_BOUNDS_OK(off, bytes, a.plane_bytes, a.status) || !KVS_BOUNDS_OK(u, 1, a.units, a.status)) off = 0;
                bulk_g2s(sb, a.kplane + off, bytes, &full_bar[st]);
                bulk_g2s(sb + kTile, a.vplane + off, bytes, &full_bar[st]);
            }
            if (qpart && with_q)
                bulk_g2s(sb + 2 * kTile, a.q + (KVS_BOUNDS_OK(u, 1, a.units, a.status) ? u : 0) * (long long)qbytes, qbytes, &full_bar[st]);
        };
        // until the preceding kernel is known to have finished: only tiles made of rows that nothing in flight writes
        int npre = 0;
        if (lane == 0)
            for (; npre < stages && t0 + npre < t1; ++npre) {
                const int ti = (int)((t0 + npre) % a.tpu);
                if ((long long)(ti + 1) * TN > a.safe_rows) break;
                issue(t0 + npre, npre, true, true, false);
            }
        if (lane == 0) KVS_TRACE_STAMP(tr, kTrProducerPre);
        pdl_wait();
        if (lane == 0) KVS_TRACE_STAMP(tr, kTrProducerGo);
        pdl_launch_dependents();
        if (lane == 0)
            for (int j = 0; j < npre; ++j) issue(t0 + j, j, false, false, true);
        if (a.k_new != nullptr && t0 < t1) {
            // Of every unit whose last tile lies in this block's share the new row, a group per lane, four units at a time.  Only
            // this block fetches that tile, after this: the fence orders the stores before the copies lane 0 issues next.
            if (over) {
                if (lane == 0 && blockIdx.x == 0) atomicExch(a.status, 4);
            } else {
                constexpr int PIECES = Pack4Row<D>::GROUP / 8;
                const bool isv = lane & 4;
                const uint32_t group = lane & 3;
                for (long long u = t0 / a.tpu + lane / 8; u <= (t1 - 1) / a.tpu; u += 4) {
                    const long long last = u * a.tpu + a.tpu - 1, to = (u * a.row_stride + a.n - 1) * RB;
                    if (last < t0 || last >= t1) continue;
                    if (!KVS_BOUNDS_OK(to, RB, a.plane_bytes, a.status) || !KVS_BOUNDS_OK(u, 1, a.units, a.status)) continue;
                    const uint4* p = reinterpret_cast<const uint4*>((isv ? a.v_new : a.k_new) + u * (D * 2)) + group * PIECES;
                    uint4 in[PIECES];
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) in[i] = p[i];
                    uint32_t pair, words[PIECES];
                    pack_group<__nv_bfloat16, D>(in, &pair, words);
                    store_group<D>(reinterpret_cast<uint32_t*>(const_cast<char*>(isv ? a.vplane : a.kplane) + to), group, pair, words);
                }
            }
            asm volatile("fence.proxy.async.global;" ::: "memory");
            __syncwarp();
        }
        if (lane != 0) return;
        // tile j of the block lies in stage j % stages; its phase there is j / stages
        int st = npre % stages, turn = npre / stages;
        int it = npre;
        bool ok = true;
        for (long long gt = t0 + npre; gt < t1; ++gt, ++it) {
            if (turn > 0) ok = mbar_wait_bounded(&empty_bar[st], (turn - 1) & 1, abort_flag, a.status, a.wait_ns);
            if (!ok) break;
            issue(gt, st, true, true, true);
            if (++st == stages) st = 0, ++turn;
        }
        if (!ok)
            for (int j = max(0, it - stages); j < it; ++j)
                mbar_wait_bounded(&full_bar[j % stages], (j / stages) & 1, abort_flag + 1, a.status, a.wait_ns);
        return;
    }

    if (warp == WARPS + 1) {
        // ------------------ hand-over of units that are cut between two blocks (see decode_splitk_mma) ------------------
        if (a.out == nullptr || t0 >= t1) return;
        const bool has_tail = (t0 % a.tpu) != 0, has_head = (t1 % a.tpu) != 0;
        if (!has_tail && !has_head) return;
        pdl_wait();   // the flags are back to zero only once the previous launch has completed
        if (has_tail) {
            if (!mbar_wait_bounded(tail_bar, 0, abort_flag, a.status, a.wait_ns)) return;
            if (lane == 0) st_release_gpu(a.flags + t0 / a.tpu, 1);
        }
        if (has_head) {
            const long long u = (t1 - 1) / a.tpu;
            int ok = 1;
            if (lane == 0) ok = flag_wait_bounded(a.flags + u, 1, abort_flag, a.status, a.wait_ns) ? 1 : 0;
            ok = __shfl_sync(0xffffffffu, ok, 0);
            __syncwarp();
            if (!ok) return;
            const long long pt = u + blockIdx.x + 1;
            for (int i = lane; i < G * D; i += 32) handover[(i / D) * (D + 2) + (i % D)] = __ldcg(a.part_o + pt * G * D + i);
            for (int i = lane; i < G * 2; i += 32) handover[(i >> 1) * (D + 2) + D + (i & 1)] = __ldcg(a.part_ml + pt * G * 2 + i);
            __syncwarp();
            if (lane == 0) {
                a.flags[u] = 0;          // this block is the flag's only reader
                mbar_arrive(head_bar);
            }
        }
        return;
    }

    // ---------------------------------- consumers ----------------------------------
    pdl_wait();               // partial results of the previous call may still be read until here
    if (tid == 0) KVS_TRACE_STAMP(tr, kTrConsumerGo);
    pdl_launch_dependents();
    int trace_piece = 0;
    // S: keys row and row + 8, heads 2 quad and 2 quad + 1; O: head row, columns 2 quad and 2 quad + 1
    const int row = lane >> 2, quad = lane & 3;
    const int head = WIDE ? row : (row & 3);       // whose queries this lane brings in
    const bool third = !WIDE && quad >= 2;         // this lane's columns of S carry the third term

    int st = 0, phase = 0;    // of the next tile
    long long gt = t0;
    while (gt < t1) {
        const long long u = gt / a.tpu;
        const int ti0 = (int)(gt - u * a.tpu);
        const int piece_tiles = (int)min((long long)(a.tpu - ti0), t1 - gt);
        const int n_u = a.unit_len ? min(a.unit_len[u], a.cap) : a.n;

        uint32_t qa[KSTEPS][2];
        uint64_t o[NB];                   // pairs: elements nb of the lane's two columns
        float m[2] = {-1.0e30f, -1.0e30f}, lsum[2] = {0.f, 0.f};   // maximum (log2 domain) of a head, sum over the lane's keys
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) o[nb] = 0;

        auto chunk = [&](const unsigned char* ks, unsigned char* vs, int rows, auto blocks) {
            constexpr int NBK = decltype(blocks)::value;
            // ---- scores ----
            // Two blocks side by side, even and odd steps of each apart: an MMA waits for the fourth before it.
            float s[NBK][4];                            // [block]: (key row, two heads), (key row + 8, two heads)
#pragma unroll
            for (int blk0 = 0; blk0 < NBK; blk0 += 2) {
                constexpr int AT_ONCE = 2;
                // rows past the end hold whatever the stage held before: their scores are replaced below
                uint32_t w[AT_ONCE][2][XW], s2[AT_ONCE][2], b2[AT_ONCE][2];
#pragma unroll
                for (int z = 0; z < AT_ONCE && blk0 + z < NBK; ++z)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const unsigned char* kr = ks + ((blk0 + z) * 16 + y * 8 + row) * RB;
                        const uint32_t pair = *reinterpret_cast<const uint32_t*>(kr + 4 * quad);
                        s2[z][y] = __byte_perm(pair, pair, 0x1010);
                        b2[z][y] = __byte_perm(pair, pair, 0x3232);
                        if constexpr (D == 128) {
                            const uint4 x = *reinterpret_cast<const uint4*>(kr + 16 + 16 * quad);
                            w[z][y][0] = x.x, w[z][y][1] = x.y, w[z][y][2] = x.z, w[z][y][3] = x.w;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2*>(kr + 16 + 8 * quad);
                            w[z][y][0] = x.x, w[z][y][1] = x.y;
                        }
                    }
                float c[AT_ONCE][2][4];
#pragma unroll
                for (int x = 0; x < XW; ++x) {
                    uint32_t v[AT_ONCE][2][4];          // [block][key row, row + 8][pair]
#pragma unroll
                    for (int z = 0; z < AT_ONCE && blk0 + z < NBK; ++z)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            v[z][y][0] = fma_bf16x2(pack4_pair<0>(w[z][y][x]), s2[z][y], b2[z][y]);
                            v[z][y][1] = fma_bf16x2(pack4_pair<1>(w[z][y][x]), s2[z][y], b2[z][y]);
                            v[z][y][2] = fma_bf16x2(pack4_pair<2>(w[z][y][x]), s2[z][y], b2[z][y]);
                            v[z][y][3] = fma_bf16x2(pack4_pair<3>(w[z][y][x]), s2[z][y], b2[z][y]);
                        }
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int z = 0; z < AT_ONCE && blk0 + z < NBK; ++z) {
                            const uint32_t* q = qa[2 * x + e];
                            if (x == 0) mma_bf16_first(c[z][e], v[z][0][2 * e], v[z][1][2 * e], v[z][0][2 * e + 1], v[z][1][2 * e + 1], q[0], q[1]);
                            else mma_bf16(c[z][e], v[z][0][2 * e], v[z][1][2 * e], v[z][0][2 * e + 1], v[z][1][2 * e + 1], q[0], q[1]);
                        }
                }
#pragma unroll
                for (int z = 0; z < AT_ONCE && blk0 + z < NBK; ++z)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[blk0 + z][i] = c[z][0][i] + c[z][1][i];
            }
            if (rows < NBK * 16) {            // the end of a unit, inside the last block
#pragma unroll
                for (int i = 0; i < NBK * 4; ++i)
                    if (i / 4 * 16 + i / 2 % 2 * 8 + row >= rows) s[i / 4][i % 4] = -INFINITY;
                // Value rows past the end may hold anything (0 * NaN is not 0).  With s = b = 0 their values are zero; the fence
                // orders the stores before the copy that refills the stage.
                for (int r = lane; r < NBK * 16; r += 32)
                    if (r >= rows) *reinterpret_cast<uint4*>(vs + r * RB) = make_uint4(0u, 0u, 0u, 0u);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            // ---- the heads' reference (the scale is positive) ----
            // The weights are taken relative to m, the maximum when it was last looked for: it is looked for again only when a score
            // exceeds it by 2^8, which fp32 sums and three bf16 terms bear as well as 1.  (With a new maximum every chunk its
            // way around the lanes and the rescaling of the state stand between the two products: 193 us instead of 190.)
            float top[2];
            bool grown = false;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[j] = fmaxf(s[0][j], s[0][2 + j]);
#pragma unroll
                for (int blk = 1; blk < NBK; ++blk) top[j] = fmaxf(top[j], fmaxf(s[blk][j], s[blk][2 + j]));
                grown |= top[j] * a.scale_log2 > m[j] + 8.f;
            }
            if (__any_sync(0xffffffffu, grown)) {
                float alpha[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], d));
                    const float m_new = fmaxf(m[j], top[j] * a.scale_log2);
                    alpha[j] = fast_exp2(m[j] - m_new);
                    m[j] = m_new;
                    lsum[j] *= alpha[j];
                }
                // the head of this lane's row of O: its alpha is with lane row / 2
                const float alpha0 = __shfl_sync(0xffffffffu, alpha[0], row >> 1), alpha1 = __shfl_sync(0xffffffffu, alpha[1], row >> 1);
                const uint64_t alpha2 = row & 1 ? pair_of(alpha1, alpha1) : pair_of(alpha0, alpha0);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) o[nb] = mul2(o[nb], alpha2);
            }
            // A fragments of P: [block][keys 0..7 or 8..15]: rows 0..7 / rows 8..15 (/ the second product's rows 0..7)
            uint32_t pa[NBK][2], pb[NBK][2];
            [[maybe_unused]] uint32_t pc[NBK][2];
#pragma unroll
            for (int blk = 0; blk < NBK; ++blk)
#pragma unroll
                for (int nb = 0; nb < 2; ++nb) {
                    float p0 = fast_exp2(fmaf(s[blk][2 * nb], a.scale_log2, -m[0])), p1 = fast_exp2(fmaf(s[blk][2 * nb + 1], a.scale_log2, -m[1]));
                    lsum[0] += p0;
                    lsum[1] += p1;
                    const uint32_t hi = take_term(p0, p1), mid = take_term(p0, p1), lo = pack2(p0, p1);
                    pa[blk][nb] = transposed(third ? lo : hi);
                    pb[blk][nb] = transposed(third ? 0u : mid);
                    if constexpr (WIDE) pc[blk][nb] = transposed(lo);
                }
            // ---- O += P V ----
            const unsigned char* vq = vs + quad * 2 * RB;       // the first of this lane's rows
            uint32_t s2[NBK][2], b2[NBK][2];       // (s, b) of the keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9
#pragma unroll
            for (int blk = 0; blk < NBK; ++blk)
#pragma unroll
                for (int nb = 0; nb < 2; ++nb) {
                    const unsigned char* vr = vq + (blk * 16 + nb * 8) * RB + 4 * (row >> 1);
                    const uint32_t h0 = *reinterpret_cast<const uint32_t*>(vr), h1 = *reinterpret_cast<const uint32_t*>(vr + RB);
                    s2[blk][nb] = __byte_perm(h0, h1, 0x5410);
                    b2[blk][nb] = __byte_perm(h0, h1, 0x7632);
                }
#pragma unroll
            for (int x = 0; x < VW; ++x) {
                uint32_t w[NBK][2][2];             // codes of the two keys, interleaved: [block][key pair][half of the word]
#pragma unroll
                for (int blk = 0; blk < NBK; ++blk)
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
                        const unsigned char* vr = vq + (blk * 16 + nb * 8) * RB + 16 + row * (D / 16) + 4 * x;
                        const uint32_t w0 = *reinterpret_cast<const uint32_t*>(vr), w1 = *reinterpret_cast<const uint32_t*>(vr + RB);
                        w[blk][nb][0] = __byte_perm(w0, w1, 0x5410);
                        w[blk][nb][1] = __byte_perm(w0, w1, 0x7632);
                    }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    // four column blocks side by side, for the same reason
                    float c[4][4];
#pragma unroll
                    for (int blk = 0; blk < NBK; ++blk) {
                        uint32_t v[4][2];
#pragma unroll
                        for (int nb = 0; nb < 2; ++nb) {
                            v[0][nb] = fma_bf16x2(pack4_pair<0>(w[blk][nb][half]), s2[blk][nb], b2[blk][nb]);
                            v[1][nb] = fma_bf16x2(pack4_pair<1>(w[blk][nb][half]), s2[blk][nb], b2[blk][nb]);
                            v[2][nb] = fma_bf16x2(pack4_pair<2>(w[blk][nb][half]), s2[blk][nb], b2[blk][nb]);
                            v[3][nb] = fma_bf16x2(pack4_pair<3>(w[blk][nb][half]), s2[blk][nb], b2[blk][nb]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (blk == 0) mma_bf16_first(c[i], pa[blk][0], pb[blk][0], pa[blk][1], pb[blk][1], v[i][0], v[i][1]);
                            else mma_bf16(c[i], pa[blk][0], pb[blk][0], pa[blk][1], pb[blk][1], v[i][0], v[i][1]);
                        if constexpr (WIDE)
#pragma unroll
                            for (int i = 0; i < 4; ++i) mma_bf16(c[i], pc[blk][0], 0u, pc[blk][1], 0u, v[i][0], v[i][1]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint64_t& acc = o[8 * x + 4 * half + i];
                        acc = add2(acc, add2(pair_of(c[i][0], c[i][1]), pair_of(c[i][2], c[i][3])));
                    }
                }
            }
        };
        for (int k = 0; k < piece_tiles; ++k) {
            if (!mbar_wait_bounded(&full_bar[st], phase, abort_flag, a.status, a.wait_ns)) return;
            if (tid == 0 && k == 0 && gt == t0) KVS_TRACE_STAMP(tr, kTrFirstTile);
            unsigned char* tile = smem + st * stage_bytes;
            if (k == 0) {
                // B fragments of Q.  Step j of lane t: elements e, e + 4 and e + 1, e + 5 of its group, e = 8 (j / 2) + 2 (j % 2)
                const uint32_t* qs = reinterpret_cast<const uint32_t*>(tile + 2 * kTile) + (head < G ? head : 0) * (D / 2) + quad * (D / 8);
#pragma unroll
                for (int j = 0; j < KSTEPS; ++j) {
                    const uint32_t lo = head < G ? qs[4 * (j / 2) + j % 2] : 0u, hi = head < G ? qs[4 * (j / 2) + j % 2 + 2] : 0u;
                    qa[j][0] = __byte_perm(lo, hi, 0x5410);
                    qa[j][1] = __byte_perm(lo, hi, 0x7632);
                }
            }
            // an even share of the tile's 16-row blocks for every warp
            const int have = min(TN, n_u - (ti0 + k) * TN), blocks = max(0, (have + 15) / 16);
            const int b0 = blocks * warp / WARPS, rows = min(have, blocks * (warp + 1) / WARPS * 16) - b0 * 16;
            if (rows > 0) {
                unsigned char *ks = tile + b0 * 16 * RB, *vs = ks + kTile;
                // (exactly as many blocks as there are: what lies behind them is another warp's, or another buffer's)
                if (rows > 48) chunk(ks, vs, rows, std::integral_constant<int, 4>());
                else if (rows > 32) chunk(ks, vs, rows, std::integral_constant<int, 3>());
                else if (rows > 16) chunk(ks, vs, rows, std::integral_constant<int, 2>());
                else chunk(ks, vs, rows, std::integral_constant<int, 1>());
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[st]);
            if (++st == stages) st = 0, phase ^= 1;
        }

        // ---- end of piece: merge the consumer warps (see decode_splitk_mma for the cases) ----
        const long long pid = u + blockIdx.x;
        if (tid == 0 && trace_piece < 8) KVS_TRACE_STAMP(tr, kTrPiece + 2 * trace_piece);
        const bool finish = a.out != nullptr;
        const bool whole = finish && ti0 == 0 && piece_tiles == a.tpu;
        const bool head_piece = finish && ti0 == 0 && piece_tiles < a.tpu;
        const bool tail = finish && ti0 > 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int d = 4; d < 32; d *= 2) lsum[j] += __shfl_xor_sync(0xffffffffu, lsum[j], d);
        const float m0 = __shfl_sync(0xffffffffu, m[0], row >> 1), m1 = __shfl_sync(0xffffffffu, m[1], row >> 1);
        const float l0 = __shfl_sync(0xffffffffu, lsum[0], row >> 1), l1 = __shfl_sync(0xffffffffu, lsum[1], row >> 1);
        if constexpr (!WIDE)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)         // the third term's share, from rows 4..7
                o[nb] = add2(o[nb], __shfl_down_sync(0xffffffffu, o[nb], 16));
        named_bar_sync(1, S::CONSUMERS);
        if (row < G) {
            float* dst = scratch + (warp * 8 + row) * (D + 2);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                dst[quad * 2 * NB + nb] = low_of(o[nb]);
                dst[(quad * 2 + 1) * NB + nb] = high_of(o[nb]);
            }
            if (quad == 0) {
                dst[D] = row & 1 ? m1 : m0;
                dst[D + 1] = row & 1 ? l1 : l0;
            }
        }
        if (head_piece && !mbar_wait_bounded(head_bar, 0, abort_flag, a.status, a.wait_ns)) return;
        named_bar_sync(1, S::CONSUMERS);
        for (int idx = tid; idx < G * D; idx += S::CONSUMERS) {
            const int g = idx / D, d = idx - g * D;
            const float* src = scratch + g * (D + 2);
            constexpr int WS = 8 * (D + 2);
            float M = -1.0e30f;
#pragma unroll
            for (int j = 0; j < WARPS; ++j) M = fmaxf(M, src[j * WS + D]);
            float acc = 0.f, den = 0.f;
#pragma unroll
            for (int j = 0; j < WARPS; ++j) {
                const float w = fast_exp2(src[j * WS + D] - M);
                acc = fmaf(w, src[j * WS + d], acc);
                den = fmaf(w, src[j * WS + D + 1], den);
            }
            if (whole) {
                a.out[(u * G + g) * D + d] = acc / den;
            } else if (head_piece) {
                const float* hv = handover + g * (D + 2);      // the unit's second piece
                const float Mx = fmaxf(M, hv[D]);
                const float w0 = fast_exp2(M - Mx), w1 = fast_exp2(hv[D] - Mx);
                a.out[(u * G + g) * D + d] = fmaf(w1, hv[d], w0 * acc) / fmaf(w1, hv[D + 1], w0 * den);
            } else if (KVS_BOUNDS_OK(pid, 1, a.units + (long long)gridDim.x, a.status)) {
                a.part_o[(pid * G + g) * D + d] = acc;
                if (d == 0) {
                    a.part_ml[(pid * G + g) * 2] = M;
                    a.part_ml[(pid * G + g) * 2 + 1] = den;
                }
            }
        }
        if (tail) mbar_arrive(tail_bar);   // this thread's part of the piece is written
        if (tid == 0 && trace_piece < 8) KVS_TRACE_STAMP(tr, kTrPiece + 2 * trace_piece + 1);
        ++trace_piece;
        gt += piece_tiles;
    }
    if (tid == 0) {
        KVS_TRACE_STAMP(tr, kTrEnd);
        KVS_TRACE_VALUE(tr, kTrPieces, trace_piece);
    }
}

template <int D, bool WIDE>
cudaError_t set_attr() {
    cudaError_t e = cudaFuncSetAttribute(decode_pack4_mma<D, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, Pack4Shape<D>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    // room for the combine kernel's blocks beside this kernel's (see decode_splitk_mma)
    return cudaFuncSetAttribute(decode_pack4_mma<D, WIDE>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
}

template <int D>
cudaError_t launch_one(const Pack4KernelArgs& ka, int NC, bool pdl, cudaStream_t stream) {
    using S = Pack4Shape<D>;
    return ka.G > 4 ? launch_kernel(decode_pack4_mma<D, true>, dim3(NC), dim3(S::THREADS), S::SMEM_BYTES, stream, pdl, ka)
                    : launch_kernel(decode_pack4_mma<D, false>, dim3(NC), dim3(S::THREADS), S::SMEM_BYTES, stream, pdl, ka);
}

}  // namespace

cudaError_t init_pack4_kernels() {
    cudaError_t e;
    if ((e = set_attr<128, false>()) != cudaSuccess || (e = set_attr<128, true>()) != cudaSuccess || (e = set_attr<64, false>()) != cudaSuccess) return e;
    return set_attr<64, true>();
}

// The tile: as many rows as make the longest block's share cheapest.  A warp takes its 16-row blocks of a tile one after the other,
// so a tile costs its rows rounded up to 128 and a constant - barriers and the latency of a chunk's chain of products, worth
// about kTileCost rows (13B shape, 16 x 40 heads x 8192 rows: tiles of 512 rows 193 us, 384 210, 256 227, 128 294).
void plan_decode_pack4(int units, int n, int sm_count, int max_ctas, DecodePlan* plan) {
    constexpr int kTileCost = 108, kGrain = kPack4Warps * 16;
    int cap = sm_count;
    if (max_ctas > 0) cap = std::min(cap, max_ctas);
    cap = std::min(cap, kMaxCtas);
    double best = 0;
    for (int rows = kPack4TileMax; rows >= kGrain; rows -= kGrain) {
        const int tpu = (n + rows - 1) / rows, last = (n - (tpu - 1) * rows + kGrain - 1) / kGrain * kGrain;
        const long long T = (long long)units * tpu;
        const double cost = (double)((T + cap - 1) / cap) * ((double)(tpu - 1) * (rows + kTileCost) + last + kTileCost) / tpu;
        if (rows == kPack4TileMax || cost < best) {
            best = cost;
            plan->tile_rows = rows;
            plan->tpu = tpu;
            plan->T = T;
        }
    }
    plan->NC = (int)std::min<long long>(plan->T, cap);
    plan->kernel = 3;
}

cudaError_t launch_decode_pack4(const DecodeArgs& a, const DecodePlan& plan, cudaStream_t stream) {
    if (a.G < 1 || a.G > 8 || (a.D != 64 && a.D != 128)) return cudaErrorInvalidValue;
    Pack4KernelArgs ka;
    ka.q = static_cast<const char*>(a.q);
    ka.kplane = static_cast<const char*>(a.kplane);
    ka.vplane = static_cast<const char*>(a.vplane);
    ka.part_o = a.part_o;
    ka.part_ml = a.part_ml;
    ka.out = a.finish_in_kernel ? a.out : nullptr;
    ka.flags = a.flags;
    ka.status = a.status;
    ka.n = a.n;
    ka.row_stride = a.row_stride;
    ka.tpu = plan.tpu;
    ka.tile_rows = plan.tile_rows;
    ka.G = a.G;
    ka.units = a.units;
    ka.cap = a.capacity;
    ka.safe_rows = (a.programmatic && !a.unit_len) ? a.safe_rows : 0;
    ka.T = plan.T;
    ka.scale_log2 = a.scale_log2;
    ka.unit_len = a.unit_len;
    ka.n_extra = a.n_extra;
    ka.plane_bytes = a.plane_bytes;
    ka.wait_ns = a.wait_ns;
    ka.stall_tile = a.stall_tile;
    ka.trace = a.trace;
    ka.k_new = static_cast<const char*>(a.k_new);
    ka.v_new = static_cast<const char*>(a.v_new);
    return a.D == 128 ? launch_one<128>(ka, plan.NC, a.programmatic, stream) : launch_one<64>(ka, plan.NC, a.programmatic, stream);
}

}  // namespace kvs
