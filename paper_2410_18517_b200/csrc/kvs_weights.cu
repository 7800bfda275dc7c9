// Cache reduction by attention weight: the running totals a decode step leaves behind, and the rows a budget keeps.
#include <algorithm>

#include "kvs_device.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

// --------------------------------------------------------------------------------------
// Finish of a decode step that stored its scores s_gj (log2 domain) beside the split-K pieces:
//   out[g]   = sum_c w_c o_c / L_g,   w_c = 2^(m_c - M_g),  M_g = max_c m_c,  L_g = sum_c w_c l_c
//   total[j] += sum_g 2^(s_gj - M_g) / L_g          (heads in order: no atomics, the same bits every time)
// Blocks 0 .. chunks-1 of a unit take a run of rows each, blocks chunks .. chunks+G-1 one head's output each; every
// block works M and L out for itself from the pieces' (max, sum) pairs, which are few and in L2, while its first scores
// are on their way.  A thread takes four neighbouring rows and asks for all heads' scores at once.
// Bound: HBM / L2 for the scores and totals, (4 G + 8) bytes per row beside the step's 4 D or 8 D bytes.
// --------------------------------------------------------------------------------------
constexpr int kFinishThreads = 256;
constexpr int kFinishRows = 4 * kFinishThreads;    // rows per turn of a block

struct FinishArgs {
    const float* part_o;
    const float* part_ml;
    const float* scores;
    const float* total_in;     // nullptr: totals start at zero
    float* total_out;
    float* out;
    long long T;
    int total_stride, score_stride, G, tpu, NC, n, tile_rows, units, cap, chunks;
    int turns;                 // turns of a block: it takes turns * kFinishRows rows
    bool vec;                  // totals can be read and written four at a time
    const int* n_extra;
    const int* unit_len;
    long long score_count;
    int* status;
};

__device__ __forceinline__ int block_of_tile(long long gt, long long T, int NC) { return (int)(((gt + 1) * NC + T - 1) / T - 1); }

template <int D>
__global__ void __launch_bounds__(kFinishThreads) weights_finish_kernel(const FinishArgs a_in) {
    FinishArgs a = a_in;
    __shared__ float s_max[8], s_inv[8];
    __shared__ float s_acc[kFinishThreads / (D / 4)][D];
    pdl_launch_dependents();
    pdl_wait();
    if (a.n_extra) {    // replayed launch: the lengths have grown on the device
        a.n = min(a.n + *a.n_extra, a.cap);
        a.tpu = (a.n + a.tile_rows - 1) / a.tile_rows;
        a.T = (long long)a.units * a.tpu;
    }
    const int per_unit = a.chunks + a.G;
    const long long u = blockIdx.x / per_unit;
    const int part = blockIdx.x - (int)u * per_unit;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c0 = block_of_tile(u * a.tpu, a.T, a.NC);
    int np = block_of_tile((u + 1) * a.tpu - 1, a.T, a.NC) - c0 + 1;
    if (!KVS_BOUNDS_OK(u, 1, a.units, a.status) || !KVS_BOUNDS_OK(u + c0, np, (long long)a.units + a.NC, a.status)) np = 0;
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + (u + c0) * a.G;    // piece c, head g: ml[c * G + g]
    const int n = a.unit_len ? min(a.unit_len[u], a.cap) : a.n;
    const float* sc = a.scores + u * a.G * a.score_stride;
    const long long tot = u * (long long)a.total_stride;
    // (a score array's rows are padded to a multiple of 128: reading four at a time is safe)
    float4 s[8];
    auto fetch = [&](int j) {
#pragma unroll
        for (int g = 0; g < 8; ++g)
            if (g < a.G && j < n && KVS_BOUNDS_OK((u * a.G + g) * a.score_stride + j, 4, a.score_count, a.status)) s[g] = *reinterpret_cast<const float4*>(sc + (long long)g * a.score_stride + j);
    };
    const int j_first = part * a.turns * kFinishRows + 4 * threadIdx.x;
    if (part < a.chunks) fetch(j_first);
    if (warp < a.G) {
        float M = -1.0e30f, L = 0.f;
        for (int c = lane; c < np; c += 32) M = fmaxf(M, ml[c * a.G + warp].x);
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        for (int c = lane; c < np; c += 32) {
            const float2 v = ml[c * a.G + warp];
            L = fmaf(fast_exp2(v.x - M), v.y, L);
        }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
        if (lane == 0) {
            s_max[warp] = M;
            s_inv[warp] = 1.0f / L;
        }
    }
    __syncthreads();
    if (part < a.chunks) {
        for (int turn = 0; turn < a.turns; ++turn) {
            const int j = j_first + turn * kFinishRows;
            if (j >= n || !KVS_BOUNDS_OK(j, min(4, n - j), a.total_stride, a.status)) break;
            if (turn > 0) fetch(j);
            float t[4] = {0.f, 0.f, 0.f, 0.f};
            const bool vec = a.vec && j + 4 <= n;
            if (a.total_in != nullptr) {
                if (vec) *reinterpret_cast<float4*>(t) = *reinterpret_cast<const float4*>(a.total_in + tot + j);
                else
                    for (int i = 0; i < 4 && j + i < n; ++i) t[i] = a.total_in[tot + j + i];
            }
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < 8; ++g)
                if (g < a.G) {
                    const float M = s_max[g], inv = s_inv[g];
                    sum[0] = fmaf(fast_exp2(s[g].x - M), inv, sum[0]);
                    sum[1] = fmaf(fast_exp2(s[g].y - M), inv, sum[1]);
                    sum[2] = fmaf(fast_exp2(s[g].z - M), inv, sum[2]);
                    sum[3] = fmaf(fast_exp2(s[g].w - M), inv, sum[3]);
                }
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] += sum[i];
            if (vec) *reinterpret_cast<float4*>(a.total_out + tot + j) = *reinterpret_cast<const float4*>(t);
            else
                for (int i = 0; i < 4 && j + i < n; ++i) a.total_out[tot + j + i] = t[i];
        }
        return;
    }
    // one head's output: D / 4 threads per piece, the groups take pieces in turn, then add up in group order
    constexpr int TPP = D / 4, GROUPS = kFinishThreads / TPP;
    const int g = part - a.chunks, grp = threadIdx.x / TPP, t = threadIdx.x - grp * TPP;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = grp; c < np; c += GROUPS) {
        const float w = fast_exp2(ml[c * a.G + g].x - s_max[g]);
        const float4 o = *reinterpret_cast<const float4*>(a.part_o + ((u + c0 + c) * a.G + g) * D + 4 * t);
        acc.x = fmaf(w, o.x, acc.x);
        acc.y = fmaf(w, o.y, acc.y);
        acc.z = fmaf(w, o.z, acc.z);
        acc.w = fmaf(w, o.w, acc.w);
    }
    *reinterpret_cast<float4*>(&s_acc[grp][4 * t]) = acc;
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += kFinishThreads) {
        float r = 0.f;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) r += s_acc[i][d];
        a.out[(u * a.G + g) * D + d] = r * s_inv[g];
    }
}

// --------------------------------------------------------------------------------------
// Selection: of a unit's n rows keep the newest n_recent and, of the others, the n_keep - n_recent with the largest
// totals; equal totals go to the older row, NaN counts below everything.  The list comes out ascending.
// Radix select on order-preserving 32-bit keys, 11 + 11 + 10 bits from the top, by histograms in shared memory: after three
// passes the key of the last row kept is known exactly, and how many rows with that very key stay.  One block per
// unit, or a cluster of blocks where units are few and long; a warp owns IPT * 32 neighbouring rows, lane l the rows 32 i + l, in registers: loads and stores are
// contiguous, and one vote orders 32 rows.  What pads a unit's end has the lowest key and the highest row numbers, so it
// is never reached.  Bound: the chain of a block (three passes of histogram, barriers and search, then the positions), and
// with many units how many blocks an SM holds: a block of 256 threads with 64 registers each, four of them, 592 in all.
// Units of 8192 rows, cold: 304 in 20.5 us, 592 in 24.6, 600 to 720 in 30.7 (a second wave on an almost empty GPU); issuing
// the 40 to 80 instructions for 32 rows would take 6 to 12.
// (Keys in shared memory and a list of the first bin's keys for the later passes: 100 for 32 rows, 53 us for 640 units
// of 8192 rows; neighbouring rows in one thread: the loads of a warp then touch 32 lines each, 47 us.)
// --------------------------------------------------------------------------------------
constexpr int kSelectThreads = 1024;
constexpr int kSelectBins = 2048;
constexpr int kSelectCluster = 8;

__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0u;                            // NaN: below minus infinity (whose key is 0x007fffff)
    const uint32_t b = __float_as_uint(x + 0.0f);     // -0 becomes +0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The total a key was made from; of zeros and NaN, which lose their sign and payload in the key, the total itself.  (Read
// again for every row kept, each store waited for its load: 35 us instead of 27 for 640 units of 8192 rows.)
__device__ __forceinline__ float total_of(uint32_t key, const float* from) {
    if (key == 0x80000000u || key == 0u) return *from;
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// The same place of another block's shared memory.
__device__ __forceinline__ uint32_t in_block(const void* p, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ int4 ld_cluster4(uint32_t at) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster4(uint32_t at, const int4& v) {
    asm volatile("st.shared::cluster.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ int2 ld_cluster2(uint32_t at) {
    int2 v;
    asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}

// IPT: rows per lane.  SPREAD: the blocks of a cluster share a unit, block r takes the r-th tile of blockDim.x * IPT rows.  Each sums
// its share of the digits over all blocks' histograms and hands all blocks the sums (every block summing every digit: 16.4
// us instead of 12.6 for eight blocks on 32768 rows); before it writes it takes the earlier blocks' counts.
// ONE: a unit fits the tile (or the cluster's tiles), which stays in registers; otherwise the tiles are read again for every
// step.
template <int IPT, bool ONE, bool SPREAD>
__global__ void __launch_bounds__(kSelectThreads) select_rows_kernel(const SelectArgs a, const __grid_constant__ SelectCounts counts, int cluster) {
    static_assert(ONE || !SPREAD, "a cluster's blocks take one tile each");
    // (a spread unit's passes have a histogram each: the other blocks may still read the last one's)
    __shared__ __align__(16) int hists[SPREAD ? 3 : 1][kSelectBins];
    __shared__ __align__(16) int merged[SPREAD ? kSelectBins : 4];
    __shared__ int warp_gt[32], warp_eq[32];
    __shared__ __align__(8) int block_counts[2];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need;
    const int unit = SPREAD ? blockIdx.x / cluster : blockIdx.x, rank = SPREAD ? blockIdx.x - unit * cluster : 0;
    const long long u = a.unit0 + unit;
    // (in a normal build the compiler drops the check)
    auto fits = [&](int at) { return KVS_BOUNDS_OK(at, 1, a.keep_stride, a.status) && KVS_BOUNDS_OK(unit, 1, a.units, a.status); };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, threads = blockDim.x, warps = threads >> 5;
    const int n = a.unit_len ? a.unit_len[u] : a.n;
    const int want = counts.n[unit] - a.n_recent;     // rows chosen by total
    const int old = n - a.n_recent;                         // rows they are chosen from
    const float* total = a.total + u * a.total_stride;
    const int tile = threads * IPT, first = warp * 32 * IPT + lane;
    uint32_t key[IPT];
    auto load = [&](int base) {
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const int j = base + first + 32 * i;
            key[i] = __float_as_uint(j < old && KVS_BOUNDS_OK(j, 1, a.total_stride, a.status) ? total[j] : __uint_as_float(0x7fffffffu));
        }
#pragma unroll
        for (int i = 0; i < IPT; ++i) key[i] = order_key(__uint_as_float(key[i]));
    };
    // the digit of the s_need-th largest key in hist[0 .. 2^bits): called by warp 0
    auto find = [&](const int* hist, uint32_t prefix, int low, int bits) {
        // lane i first sums the 64 (32) digits of the i-th largest run, then the warp looks into the run it is in
        const int run = 1 << (bits - 5), need = s_need;
        int top0 = (1 << bits) - 1, before = 0;                      // digits top0, top0 - 1, ...; rows above them
        for (int level = 0; level < 2; ++level) {
            const int width = level == 0 ? run : run / 32, top = top0 - width * lane;
            int sum = 0;
#pragma unroll 8
            for (int i = 0; i < width; ++i) sum += hist[top - ((i + lane) & (width - 1))];     // (rotated: other banks)
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            const int at = __ffs(__ballot_sync(0xffffffffu, before + upto >= need)) - 1;
            before += __shfl_sync(0xffffffffu, upto - sum, at);
            top0 -= width * at;
        }
        if (run == 64 && before + hist[top0] < need) before += hist[top0--];
        __syncwarp();
        if (lane == 0) {
            s_prefix = prefix | (uint32_t)top0 << low;
            s_need = need - before;
        }
    };
    if (want > 0) {
        if (ONE) load(rank * tile);
        if (tid == 0) s_need = want;
        uint32_t prefix = 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int low = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
            int* hist = hists[SPREAD ? pass : 0];
            for (int i = tid; i < kSelectBins; i += threads) hist[i] = 0;
            __syncthreads();
            for (int base = 0; base < (ONE ? 1 : old); base += tile) {
                if (!ONE) load(base);
#pragma unroll
                for (int i = 0; i < IPT; ++i)
                    if (pass == 0 || (key[i] ^ prefix) >> (low + bits & 31) == 0u) atomicAdd(&hist[key[i] >> low & ((1u << bits) - 1u)], 1);
            }
            if constexpr (SPREAD) {
                cluster_sync();
                // each block sums a share of the digits over all blocks and hands every block the sums
                const int part = (1 << bits) / cluster;
                for (int i = 4 * tid; i < part; i += 4 * threads) {
                    const int at = rank * part + i;
                    int4 sum = make_int4(0, 0, 0, 0);
#pragma unroll 4
                    for (int r = 0; r < cluster; ++r) {
                        const int4 x = ld_cluster4(in_block(hist + at, r));
                        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
                    }
                    for (int r = 0; r < cluster; ++r) st_cluster4(in_block(merged + at, r), sum);
                }
                cluster_sync();
            }
            __syncthreads();
            if (warp == 0) find(SPREAD ? merged : hist, prefix, low, bits);
            __syncthreads();
            prefix = s_prefix;
        }
    }
    int* keep = a.keep + u * a.keep_stride;
    float* kept = a.kept ? a.kept + u * a.keep_stride : nullptr;
    if (want > 0) {
        const uint32_t last = s_prefix;    // the smallest key kept; of the rows that have it the first `ties` stay
        const int ties = s_need;
        const uint32_t below = (1u << lane) - 1u;
        int gt_done = 0, eq_done = 0;      // rows of earlier tiles
        const int base0 = rank * tile;
        for (int base = base0; base < (ONE ? base0 + 1 : old); base += tile) {
            if (!ONE) load(base);
            int gt = 0, eq = 0;
#pragma unroll
            for (int i = 0; i < IPT; ++i) {
                gt += key[i] > last ? 1 : 0;
                eq += key[i] == last ? 1 : 0;
            }
            gt = __reduce_add_sync(0xffffffffu, gt);
            eq = __reduce_add_sync(0xffffffffu, eq);
            if (lane == 0) {
                warp_gt[warp] = gt;
                warp_eq[warp] = eq;
            }
            __syncthreads();
            int gt_w = lane < warps ? warp_gt[lane] : 0, eq_w = lane < warps ? warp_eq[lane] : 0;
            const int gt_all = __reduce_add_sync(0xffffffffu, gt_w), eq_all = __reduce_add_sync(0xffffffffu, eq_w);
            gt_w = __reduce_add_sync(0xffffffffu, lane < warp ? gt_w : 0);
            eq_w = __reduce_add_sync(0xffffffffu, lane < warp ? eq_w : 0);
            if constexpr (SPREAD) {
                if (tid == 0) {
                    block_counts[0] = gt_all;
                    block_counts[1] = eq_all;
                }
                cluster_sync();
                int2 c = make_int2(0, 0);
                if (lane < rank) c = ld_cluster2(in_block(block_counts, lane));
                gt_done = __reduce_add_sync(0xffffffffu, c.x);
                eq_done = __reduce_add_sync(0xffffffffu, c.y);
                // (nothing of another block is read after this: its end waits at the last line)
                asm volatile("barrier.cluster.arrive.release;" ::: "memory");
            }
            int seen = eq_done + eq_w;                               // rows with the last key before this warp's turn
            int pos = gt_done + gt_w + min(seen, ties);
            const float* from = total + base + first;
            if (seen + eq <= ties || seen >= ties) {                 // the warp's rows with the last key stay all, or none
                const uint32_t least = seen < ties || eq == 0 ? last : last + 1u;
#pragma unroll
                for (int i = 0; i < IPT; ++i) {
                    const bool take = key[i] >= least;
                    const uint32_t taken = __ballot_sync(0xffffffffu, take);
                    if (take) {
                        const int at = pos + __popc(taken & below);
                        if (fits(at)) {
                            keep[at] = base + first + 32 * i;
                            if (kept) kept[at] = total_of(key[i], from + 32 * i);
                        }
                    }
                    pos += __popc(taken);
                }
            } else {
#pragma unroll
                for (int i = 0; i < IPT; ++i) {
                    const uint32_t same = __ballot_sync(0xffffffffu, key[i] == last);
                    const bool take = key[i] > last || (key[i] == last && seen + __popc(same & below) < ties);
                    const uint32_t taken = __ballot_sync(0xffffffffu, take);
                    if (take) {
                        const int at = pos + __popc(taken & below);
                        if (fits(at)) {
                            keep[at] = base + first + 32 * i;
                            if (kept) kept[at] = total_of(key[i], from + 32 * i);
                        }
                    }
                    pos += __popc(taken);
                    seen += __popc(same);
                }
            }
            gt_done += gt_all;
            eq_done += eq_all;
            if (!ONE) __syncthreads();     // warp_gt, warp_eq are written again
        }
    }
    for (int j = old + rank * threads + tid; j < n; j += (SPREAD ? cluster : 1) * threads) {
        if (!fits(want + j - old) || !KVS_BOUNDS_OK(j, 1, a.total_stride, a.status)) continue;
        keep[want + j - old] = j;
        if (kept) kept[want + j - old] = total[j];
    }
    if constexpr (SPREAD) {
        __syncwarp();
        if (want > 0) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
}

__global__ void put_counts_kernel(int* out, const __grid_constant__ SelectCounts counts, int units) {
    for (int u = threadIdx.x; u < units; u += blockDim.x) out[u] = counts.n[u];
}

template <int IPT, bool ONE, bool SPREAD>
cudaError_t select_attr() {
    return cudaFuncSetAttribute(select_rows_kernel<IPT, ONE, SPREAD>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
}

// `old`: rows chosen from, of the longest unit.
template <int IPT, bool ONE, bool SPREAD = false>
cudaError_t launch_select_one(const SelectArgs& a, const SelectCounts& counts, int old, cudaStream_t stream, int cluster = 1) {
    // no more warps than a block's share has rows for
    const int share = (old + cluster - 1) / cluster, warps = std::max(1, (share + 32 * IPT - 1) / (32 * IPT));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.units * cluster));
    cfg.blockDim = dim3((unsigned)std::min(kSelectThreads, 32 * warps));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = SPREAD ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, select_rows_kernel<IPT, ONE, SPREAD>, a, counts, cluster);
}

}  // namespace

cudaError_t init_weights_kernels() {
    cudaError_t e = select_attr<8, true, false>();
    if (e == cudaSuccess) e = select_attr<8, true, true>();
    if (e == cudaSuccess) e = select_attr<32, true, true>();
    if (e == cudaSuccess) e = select_attr<32, true, false>();
    return e == cudaSuccess ? select_attr<16, false, false>() : e;
}

cudaError_t launch_put_counts(int* out, const int* n, int units, cudaStream_t stream) {
    for (int u0 = 0; u0 < units; u0 += SelectCounts::kMax) {
        const int count = std::min(units - u0, (int)SelectCounts::kMax);
        SelectCounts counts;
        for (int i = 0; i < count; ++i) counts.n[i] = n[u0 + i];
        const cudaError_t e = launch_kernel(put_counts_kernel, dim3(1), dim3(256), 0, stream, false, out + u0, counts, count);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_weights_finish(const DecodeArgs& a, const DecodePlan& plan, const float* total_in, float* total_out,
                                  int total_stride, int sm_count, cudaStream_t stream) {
    FinishArgs f;
    f.part_o = a.part_o;
    f.part_ml = a.part_ml;
    f.scores = a.scores;
    f.total_in = total_in;
    f.total_out = total_out;
    f.out = a.out;
    f.T = plan.T;
    f.total_stride = total_stride;
    f.score_stride = a.score_stride;
    f.G = a.G;
    f.tpu = plan.tpu;
    f.NC = plan.NC;
    f.n = a.n;
    f.tile_rows = plan.tile_rows;
    f.units = a.units;
    f.cap = a.capacity;
    f.n_extra = a.n_extra;
    f.unit_len = a.unit_len;
    f.score_count = a.score_count;
    f.status = a.status;
    const int turns = ((a.n_extra ? a.capacity : a.n) + kFinishRows - 1) / kFinishRows;      // of a unit's longest run of rows
    // several turns per block once eight blocks per SM are there without (640 units of 8192 rows: 2 blocks each)
    f.turns = (int)std::min<long long>(turns, std::max<long long>(1, (long long)a.units * turns / (8ll * sm_count)));
    f.chunks = (turns + f.turns - 1) / f.turns;
    f.vec = total_stride % 4 == 0 && (uintptr_t)total_in % 16 == 0 && (uintptr_t)total_out % 16 == 0;
    const dim3 grid((unsigned)(a.units * (f.chunks + a.G)));
    return a.D == 128 ? launch_kernel(weights_finish_kernel<128>, grid, dim3(kFinishThreads), 0, stream, a.programmatic, f)
                      : launch_kernel(weights_finish_kernel<64>, grid, dim3(kFinishThreads), 0, stream, a.programmatic, f);
}

cudaError_t launch_select(const SelectArgs& a, const SelectCounts& counts, cudaStream_t stream) {
    const int old = std::max(0, a.n - a.n_recent);     // of the longest unit
    // Few units, up to 8192 rows: a block of 8 rows per lane; more units: 32 rows per lane, blocks small enough that an SM holds
    // several (8192 rows, 128 units 10.3 us against 12.3, 640 units 30.8 against 26.7).
    if (old <= 2048 || (old <= 8 * kSelectThreads && a.units <= 2 * a.sm_count)) return launch_select_one<8, true>(a, counts, old, stream);
    // Longer ones: as many blocks per unit as there are SMs for, twice that if only then it stays in registers (a block alone
    // / the cluster: 8 units of 16384 rows 14.4 / 12.4 us, of 32768 20.5 / 12.6, of 131072 74 / 19; 64 units of 32768
    // 20.6 / 18.5, of 70000 49 / 37; beyond that it loses: 128 units of 32768 20.6 / 24.7, of 70000 49 / 70).
    int cluster = 1;
    while (old > 8 * kSelectThreads && cluster < kSelectCluster &&
           2ll * cluster * a.units <= (old > cluster * 32 * kSelectThreads ? 2 : 1) * a.sm_count)
        cluster *= 2;
    if (cluster > 1 && old <= cluster * 8 * kSelectThreads) return launch_select_one<8, true, true>(a, counts, old, stream, cluster);
    if (cluster > 1 && old <= cluster * 32 * kSelectThreads) return launch_select_one<32, true, true>(a, counts, old, stream, cluster);
    if (old <= 32 * kSelectThreads) return launch_select_one<32, true>(a, counts, old, stream);
    return launch_select_one<16, false>(a, counts, old, stream);
}

}  // namespace kvs
