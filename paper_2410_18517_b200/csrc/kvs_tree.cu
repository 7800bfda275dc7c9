// Attention of a tree of drafted tokens over a cache, its combine step, and the move that keeps the accepted drafts.
//
// The n_t queries of a sequence sit on the newest n_t rows of its units.  Query (token t, head g) of a kv-head sees
// every row before the drafts and those drafts whose bit is set in mask[t]:
//   out = sum_j p_j V_j / sum_j p_j,   p_j = 2^(s_j - m),  s_j = q . K_j * scale * log2(e),  m = max over visible j
// and 0 where nothing is visible.  The result has the storage type: as many as 64 rows per head go into the next
// matrix product in that type, and the rounding (one, at the end) is that type's half step.
//
// A masked draft contributes nothing whatever its row holds: its score is replaced, not added to, and its value row
// is left out of the sum (0 * infinity would be NaN).  Padding tokens of a batch may hold anything.
#include <algorithm>

#include "kvs_device.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

constexpr int kTreeThreads = 256;
constexpr int kTreeRows = 32;    // query rows per tile of the fp32 kernel
constexpr int kTreeKeys = 64;    // keys per tile

__host__ __device__ __forceinline__ long long first_tile(long long c, long long T, int teams) { return c * T / teams; }
__host__ __device__ __forceinline__ int team_of_tile(long long gt, long long T, int teams) {
    return (int)(((gt + 1) * teams + T - 1) / T - 1);
}

struct TreeKernelArgs {
    TreeArgs a;
    TreePlan p;
};

// --------------------------------------------------------------------------------------
// FMA kernel of fp32 storage.  32 query rows x 64 keys per step; thread (ty, tx) owns rows 2 ty, 2 ty + 1 and, of the
// scores, keys tx + 16 i, of the output, columns 4 tx + 64 c: every operand comes from shared memory as float4 and
// the 16 lanes of a row reduce its softmax with shuffles.  Bound: the FMA pipe and the shared-memory reads that feed it
// (32q/8kv, D = 128, B = 4, n = 4096, 16 drafts: 189 us, 22.8 TFLOP/s; its 134 MB would take 21).
// --------------------------------------------------------------------------------------
template <int D>
struct TreeShape {
    static constexpr int LD = D + 4;       // row stride of Q and K in shared memory: eight rows hit eight bank quads
    static constexpr int SMEM_BYTES = (kTreeRows * LD + kTreeKeys * LD + kTreeKeys * D + kTreeRows * kTreeKeys) * 4 + kTreeRows * 8;
};

template <int D>
__global__ void __launch_bounds__(kTreeThreads, 2) tree_attention_fma(const __grid_constant__ TreeKernelArgs ka) {
    using S = TreeShape<D>;
    constexpr int LPR = D / 4, CB = D / 64;       // 16-byte chunks of a row
    const TreeArgs& a = ka.a;
    const TreePlan& p = ka.p;
    extern __shared__ __align__(16) float smem_f[];
    float* Qs = smem_f;
    float* Ks = Qs + kTreeRows * S::LD;
    float* Vs = Ks + kTreeKeys * S::LD;
    float* Ps = Vs + kTreeKeys * D;
    unsigned long long* sees = reinterpret_cast<unsigned long long*>(Ps + kTreeRows * kTreeKeys);

    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int team = blockIdx.x / p.m_tiles, mt = blockIdx.x - team * p.m_tiles;
    const int tok0 = mt * p.tokens, rows = min(p.tokens, a.n_t - tok0) * a.G;
    const unsigned long long all = a.n_t >= 64 ? ~0ull : (1ull << a.n_t) - 1;
    const long long t1 = first_tile(team + 1, p.T, p.teams);
    pdl_wait();
    pdl_launch_dependents();

    for (long long gt = first_tile(team, p.T, p.teams); gt < t1;) {
        const long long u = gt / p.tpu;
        const int ti0 = (int)(gt - u * p.tpu);
        const int piece = (int)min((long long)(p.tpu - ti0), t1 - gt);
        gt += piece;
        const int n = a.unit_len ? min(a.unit_len[u], a.capacity) : a.n;
        const int nt = (n + kTreeKeys - 1) / kTreeKeys;          // key tiles the unit really has
        const int te = min(ti0 + piece, nt);
        if (ti0 >= te) continue;                                 // the piece lies past a ragged unit's end
        const int b = (int)(u / a.Hkv), hk = (int)(u - (long long)b * a.Hkv);
        const int ctx = n - a.n_t;                               // rows every query sees
        const float* K = static_cast<const float*>(a.kplane) + u * a.row_stride * (long long)D;
        const float* V = static_cast<const float*>(a.vplane) + u * a.row_stride * (long long)D;
        __syncthreads();                                         // the previous piece's readers are done
        for (int i = tid; i < kTreeRows * LPR; i += kTreeThreads) {
            const int r = i / LPR, c = i - r * LPR;
            float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < rows && KVS_BOUNDS_OK(tok0 + r / a.G, 1, a.n_t, a.status) && KVS_BOUNDS_OK(u, 1, a.units, a.status)) {
                const long long off = (((long long)b * a.n_t + tok0 + r / a.G) * a.Hq + hk * a.G + r % a.G) * D + c * 4;
                f = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + off);
            }
            *reinterpret_cast<float4*>(Qs + r * S::LD + c * 4) = f;
        }
        if (tid < kTreeRows) {
            const int t = tok0 + tid / a.G;
            unsigned long long w = 0;
            if (tid < rows) w = a.mask ? a.mask[(long long)b * a.n_t + t] & all : (t >= 63 ? ~0ull : (2ull << t) - 1);
            sees[tid] = w;
        }
        float m[2] = {-1.0e30f, -1.0e30f}, l[2] = {0.f, 0.f};
        float4 o[2][CB];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int c = 0; c < CB; ++c) o[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);

        for (int ti = ti0; ti < te; ++ti) {
            const int key0 = ti * kTreeKeys;
            __syncthreads();
            for (int i = tid; i < 2 * kTreeKeys * LPR; i += kTreeThreads) {
                const bool isv = i >= kTreeKeys * LPR;
                const int ii = isv ? i - kTreeKeys * LPR : i;
                const int r = ii / LPR, c = ii - r * LPR;
                float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
                if (key0 + r < n && KVS_BOUNDS_OK(((u * a.row_stride + key0 + r) * (long long)D + c * 4) * (int)sizeof(float), 16,
                                                  a.plane_bytes, a.status))
                    f = *reinterpret_cast<const float4*>((isv ? V : K) + (long long)(key0 + r) * D + c * 4);
                *reinterpret_cast<float4*>((isv ? Vs + r * D : Ks + r * S::LD) + c * 4) = f;
            }
            __syncthreads();
            float s[2][4];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][i] = 0.f;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 qv[2], kv[4];
#pragma unroll
                for (int r = 0; r < 2; ++r) qv[r] = *reinterpret_cast<const float4*>(Qs + (2 * ty + r) * S::LD + d);
#pragma unroll
                for (int i = 0; i < 4; ++i) kv[i] = *reinterpret_cast<const float4*>(Ks + (tx + 16 * i) * S::LD + d);
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[r][i] = fmaf(qv[r].x, kv[i].x, s[r][i]);
                        s[r][i] = fmaf(qv[r].y, kv[i].y, s[r][i]);
                        s[r][i] = fmaf(qv[r].z, kv[i].z, s[r][i]);
                        s[r][i] = fmaf(qv[r].w, kv[i].w, s[r][i]);
                    }
            }
            const bool masked = key0 + kTreeKeys > ctx;          // the tile holds drafts or ends past the unit
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                bool vis[4];
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = key0 + tx + 16 * i;
                    vis[i] = !masked || j < ctx || (j < n && (sees[2 * ty + r] >> (j - ctx) & 1ull));
                    s[r][i] = vis[i] ? s[r][i] * a.scale_log2 : -INFINITY;
                    mx = fmaxf(mx, s[r][i]);
                }
#pragma unroll
                for (int off = 8; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                const float m_new = fmaxf(m[r], mx);
                const float alpha = fast_exp2(m[r] - m_new);
                m[r] = m_new;
                l[r] *= alpha;
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    o[r][c].x *= alpha; o[r][c].y *= alpha; o[r][c].z *= alpha; o[r][c].w *= alpha;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = vis[i] ? fast_exp2(s[r][i] - m_new) : 0.f;
                    l[r] += w;
                    Ps[(2 * ty + r) * kTreeKeys + tx + 16 * i] = w;
                }
            }
            __syncwarp();                                        // a row's weights are written and read by one warp
#pragma unroll 4
            for (int j = 0; j < kTreeKeys; ++j) {
                const float w0 = Ps[(2 * ty) * kTreeKeys + j], w1 = Ps[(2 * ty + 1) * kTreeKeys + j];
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(Vs + j * D + 64 * c + 4 * tx);
                    if (!masked || w0 != 0.f) {
                        o[0][c].x = fmaf(w0, v.x, o[0][c].x); o[0][c].y = fmaf(w0, v.y, o[0][c].y);
                        o[0][c].z = fmaf(w0, v.z, o[0][c].z); o[0][c].w = fmaf(w0, v.w, o[0][c].w);
                    }
                    if (!masked || w1 != 0.f) {
                        o[1][c].x = fmaf(w1, v.x, o[1][c].x); o[1][c].y = fmaf(w1, v.y, o[1][c].y);
                        o[1][c].z = fmaf(w1, v.z, o[1][c].z); o[1][c].w = fmaf(w1, v.w, o[1][c].w);
                    }
                }
            }
        }
        const bool whole = ti0 == 0 && te == nt;
        const long long slot = 2ll * team + (ti0 == 0 ? 1 : 0);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int off = 8; off >= 1; off >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
            const int row = 2 * ty + r;
            if (row >= rows) continue;
            if (whole) {
                const float inv = l[r] > 0.f || l[r] != l[r] ? 1.0f / l[r] : 0.f;    // nothing visible: 0
                float* dst = static_cast<float*>(a.out) + (((long long)b * a.n_t + tok0 + row / a.G) * a.Hq + hk * a.G + row % a.G) * D;
#pragma unroll
                for (int c = 0; c < CB; ++c)
                    *reinterpret_cast<float4*>(dst + 64 * c + 4 * tx) = make_float4(o[r][c].x * inv, o[r][c].y * inv, o[r][c].z * inv, o[r][c].w * inv);
            } else {
                const long long pr = (slot * p.m_tiles + mt) * p.tile_rows + row;
                if (!KVS_BOUNDS_OK(pr, 1, tree_piece_rows(a.G), a.status)) continue;
#pragma unroll
                for (int c = 0; c < CB; ++c) *reinterpret_cast<float4*>(a.part_o + pr * D + 64 * c + 4 * tx) = o[r][c];
                if (tx == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = make_float2(m[r], l[r]);
            }
        }
    }
}

// --------------------------------------------------------------------------------------
// Combine of the units that were cut between teams, per (unit, token, head).  Lane c fetches the (max, sum) of piece c, so
// that all of them take one round trip to L2, and the output vectors follow eight at a time (one piece after the
// other, three dependent loads each: 13 us for 17 pieces, now 7).  One warp per item, or (LONG) a block of four warps, warp w with pieces w, w + 4, ..., added in warp order: a fixed order either way.
// --------------------------------------------------------------------------------------
constexpr int kTreeCombineWarps = 4;

template <typename T, int D, bool LONG>
__global__ void __launch_bounds__(kTreeCombineWarps * 32) tree_combine_kernel(const __grid_constant__ TreeKernelArgs ka) {
    constexpr int VEC = D / 32, STEP = LONG ? kTreeCombineWarps : 1;
    struct __align__(VEC * 4) Vec {
        float v[VEC];
    };
    __shared__ float s_max[kTreeCombineWarps], s_den[kTreeCombineWarps], s_acc[LONG ? kTreeCombineWarps : 1][D];
    const TreeArgs& a = ka.a;
    const TreePlan& p = ka.p;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per_unit = a.n_t * a.G;
    const long long item = LONG ? blockIdx.x : (long long)blockIdx.x * kTreeCombineWarps + warp;
    const bool there = item < (long long)a.units * per_unit;
    const int u = there ? (int)(item / per_unit) : 0;
    const int q = there ? (int)(item - (long long)u * per_unit) : 0, t = q / a.G, g = q - t * a.G;
    const int mt = t / p.tokens, row = (t - mt * p.tokens) * a.G + g;
    pdl_launch_dependents();
    pdl_wait();
    if (!there) return;
    const int n = a.unit_len ? min(a.unit_len[u], a.capacity) : a.n;
    const int nt = (n + p.key_rows - 1) / p.key_rows;
    const long long first = (long long)u * p.tpu;
    const int c0 = team_of_tile(first, p.T, p.teams), np = team_of_tile(first + nt - 1, p.T, p.teams) - c0 + 1;
    if (np == 1) return;                                         // finished by its one team
    if (!KVS_BOUNDS_OK(((2ll * (c0 + np) - 1) * p.m_tiles + mt) * p.tile_rows + row, 1, tree_piece_rows(a.G), a.status)) return;
    // this warp's pieces, c = 0 .. mine-1; piece i of the unit: slot 2 (c0 + i), the first one 2 c0 + 1
    const int w0 = LONG ? warp : 0, mine = (np - w0 + STEP - 1) / STEP;
    auto where = [&](int c) {
        const int i = w0 + c * STEP;
        return ((2ll * (c0 + i) + (i == 0 ? 1 : 0)) * p.m_tiles + mt) * p.tile_rows + row;
    };
    float M = -1.0e30f;
    for (int cb = 0; cb < mine; cb += 32)
        if (cb + lane < mine) M = fmaxf(M, a.part_ml[where(cb + lane) * 2]);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    if (LONG) {
        if (lane == 0) s_max[warp] = M;
        __syncthreads();
        M = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    }
    float den = 0.f, acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    for (int cb = 0; cb < mine; cb += 32) {
        const float2 ml = cb + lane < mine ? *reinterpret_cast<const float2*>(a.part_ml + where(cb + lane) * 2) : make_float2(-1.0e30f, 0.f);
        const float w = cb + lane < mine ? fast_exp2(ml.x - M) : 0.f;
        den = fmaf(w, ml.y, den);
        const int cnt = min(32, mine - cb);
        for (int j = 0; j < cnt; j += 8) {
            Vec x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (j + i < cnt) x[i] = reinterpret_cast<const Vec*>(a.part_o + where(cb + j + i) * D)[lane];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float wi = __shfl_sync(0xffffffffu, w, j + i);
                if (j + i < cnt)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] = fmaf(wi, x[i].v[e], acc[e]);
            }
        }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
    if (LONG) {
        if (lane == 0) s_den[warp] = den;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s_acc[warp][lane * VEC + e] = acc[e];
        __syncthreads();
        if (warp != 0) return;
#pragma unroll
        for (int w = 1; w < kTreeCombineWarps; ++w) {
            den += s_den[w];
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += s_acc[LONG ? w : 0][lane * VEC + e];
        }
    }
    const float inv = den > 0.f || den != den ? 1.0f / den : 0.f;
    const int b = u / a.Hkv, hk = u - b * a.Hkv;
    T* dst = reinterpret_cast<T*>(a.out) + (((long long)b * a.n_t + t) * a.Hq + hk * a.G + g) * D + lane * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        if constexpr (sizeof(T) == 2) dst[e] = __float2bfloat16_rn(acc[e] * inv);
        else dst[e] = acc[e] * inv;
    }
}

// --------------------------------------------------------------------------------------
// Accepted drafts: rows base + path[i] -> base + i of every unit, i < n_acc (path strictly ascending: path[i] >= i).
// One block per unit; all of a unit's rows go through shared memory, K and then V, so that no row is read after it was
// written.  The rows of the rejected drafts are cleared: what lies past a unit's end stays finite, whatever they held.  An
// entry that is not ascending or out of range sets the status word to 1 and keeps the row already there.
// --------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) accept_draft_kernel(char* kplane, char* vplane, const int* __restrict__ path, int path_stride,
                                                           const __grid_constant__ AcceptCounts counts, int seq0, int Hkv,
                                                           int n_draft, int len, int* unit_len, bool write_len, int row_vecs,
                                                           int row_stride, int* status, long long plane_vecs) {
    __shared__ uint4 buf[kTreeMaxTokens * 32];     // 64 rows of up to 512 bytes
    pdl_wait();
    const int b = seq0 + blockIdx.x / Hkv, cnt = counts.n[blockIdx.x / Hkv];
    const long long u = (long long)seq0 * Hkv + blockIdx.x;
    // (a slot that becomes ragged with this call has no lengths on the device yet)
    const int base = (unit_len && !(write_len && len >= 0) ? unit_len[u] : len) - n_draft;
    const int* list = path + (long long)b * path_stride;
    for (int kv = 0; kv < 2; ++kv) {
        uint4* rows = reinterpret_cast<uint4*>(kv == 0 ? kplane : vplane) + (u * row_stride + base) * row_vecs;
        __syncthreads();
        for (int i = threadIdx.x; i < cnt * row_vecs; i += blockDim.x) {
            const int j = i / row_vecs, v = i - j * row_vecs;
            int src = list[j];
            if (src < j || src >= n_draft || (j > 0 && list[j - 1] >= src)) {
                if (v == 0) atomicExch(status, 1);
                src = j;
            }
            if (!KVS_BOUNDS_OK((u * row_stride + base + src) * (long long)row_vecs, row_vecs, plane_vecs, status) ||
                !KVS_BOUNDS_OK(i, 1, kTreeMaxTokens * 32, status))
                continue;
            buf[i] = rows[(long long)src * row_vecs + v];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < cnt * row_vecs; i += blockDim.x)
            if (KVS_BOUNDS_OK((u * row_stride + base) * (long long)row_vecs + i, 1, plane_vecs, status)) rows[i] = buf[i];
        for (int i = cnt * row_vecs + threadIdx.x; i < n_draft * row_vecs; i += blockDim.x)
            if (KVS_BOUNDS_OK((u * row_stride + base) * (long long)row_vecs + i, 1, plane_vecs, status)) rows[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (write_len && threadIdx.x == 0) unit_len[u] = base + cnt;
}

template <typename T, int D>
cudaError_t launch_combine_one(const TreeKernelArgs& ka, int sm_count, cudaStream_t stream) {
    const long long items = (long long)ka.a.units * ka.a.n_t * ka.a.G;
    // four warps per item where a unit may have more than 16 pieces and the items are few enough that their latency
    // counts (one unit of 8192 rows, 64 items: 22.5 us with one warp, 14.5 with four; 2048 items of 20 pieces: 25 and 29)
    const bool many = ka.p.teams / ka.a.units + 2 > 16 && items <= 8 * sm_count;
    const dim3 block(kTreeCombineWarps * 32), grid((unsigned)(many ? items : (items + kTreeCombineWarps - 1) / kTreeCombineWarps));
    return many ? launch_kernel(tree_combine_kernel<T, D, true>, grid, block, 0, stream, ka.a.programmatic, ka)
                : launch_kernel(tree_combine_kernel<T, D, false>, grid, block, 0, stream, ka.a.programmatic, ka);
}

}  // namespace

cudaError_t init_tree_kernels() {
    cudaError_t e;
    if ((e = cudaFuncSetAttribute(tree_attention_fma<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, TreeShape<128>::SMEM_BYTES)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(tree_attention_fma<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, TreeShape<64>::SMEM_BYTES)) != cudaSuccess)
        return e;
    return init_tree_tc_kernels();
}

cudaError_t launch_tree(const TreeArgs& a, int sm_count, int max_ctas, int* launches, cudaStream_t stream) {
    TreeKernelArgs ka;
    ka.a = a;
    TreePlan& p = ka.p;
    int blocks = std::min(2 * sm_count, kTreeMaxBlocks);     // two per SM of either kernel
    if (max_ctas > 0) blocks = std::min(blocks, max_ctas);
    cudaError_t e;
    if (a.dtype == 0) {
        plan_tree_tc(a, blocks, &p);
        e = launch_tree_tc(a, p, stream);
    } else {
        p.tokens = std::min(a.n_t, kTreeRows / a.G);
        p.m_tiles = (a.n_t + p.tokens - 1) / p.tokens;
        p.tile_rows = kTreeRows;
        p.key_rows = kTreeKeys;
        p.tpu = (a.n + kTreeKeys - 1) / kTreeKeys;
        p.T = (long long)a.units * p.tpu;
        p.teams = (int)std::min<long long>(p.T, std::max(1, blocks / p.m_tiles));
        const unsigned grid = (unsigned)(p.teams * p.m_tiles);
        e = a.D == 128 ? launch_kernel(tree_attention_fma<128>, dim3(grid), dim3(kTreeThreads), TreeShape<128>::SMEM_BYTES, stream,
                                       a.programmatic, ka)
                       : launch_kernel(tree_attention_fma<64>, dim3(grid), dim3(kTreeThreads), TreeShape<64>::SMEM_BYTES, stream,
                                       a.programmatic, ka);
    }
    // some unit is cut unless every team boundary falls on a unit boundary
    const bool cut = a.units % p.teams != 0;
    *launches = cut ? 2 : 1;
    if (e != cudaSuccess || !cut) return e;
    if (a.dtype == 0)
        return a.D == 128 ? launch_combine_one<__nv_bfloat16, 128>(ka, sm_count, stream)
                          : launch_combine_one<__nv_bfloat16, 64>(ka, sm_count, stream);
    return a.D == 128 ? launch_combine_one<float, 128>(ka, sm_count, stream) : launch_combine_one<float, 64>(ka, sm_count, stream);
}

cudaError_t launch_accept(void* kplane, void* vplane, const int* path, int path_stride, const AcceptCounts& counts,
                          int seq0, int seqs, int Hkv, int n_draft, int len, int* unit_len, bool write_len, int row_bytes,
                          int row_stride, int* status, long long plane_bytes, bool programmatic, cudaStream_t stream) {
    return launch_kernel(accept_draft_kernel, dim3((unsigned)(seqs * Hkv)), dim3(256), 0, stream, programmatic, static_cast<char*>(kplane),
                         static_cast<char*>(vplane), path, path_stride, counts, seq0, Hkv, n_draft, len, unit_len, write_len,
                         row_bytes / 16, row_stride, status, plane_bytes / 16);
}

}  // namespace kvs
