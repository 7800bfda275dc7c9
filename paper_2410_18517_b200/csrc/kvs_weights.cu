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
// Blocks 0 .. chunks-1 of a unit take 1024 rows each, blocks chunks .. chunks+G-1 one head's output each; every
// block works M and L out for itself from the pieces' (max, sum) pairs, which are few and in L2.
// Bound: HBM / L2 for the scores and totals, (4 G + 8) bytes per row beside the step's 4 D or 8 D bytes.
// --------------------------------------------------------------------------------------
constexpr int kFinishThreads = 256;
constexpr int kFinishRows = 1024;

struct FinishArgs {
    const float* part_o;
    const float* part_ml;
    const float* scores;
    const float* total_in;     // nullptr: totals start at zero
    float* total_out;
    float* out;
    long long T;
    int total_stride, row_stride, G, tpu, NC, n, tile_rows, units, cap, chunks;
    const int* n_extra;
    const int* unit_len;
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
    const int np = block_of_tile((u + 1) * a.tpu - 1, a.T, a.NC) - c0 + 1;
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + (u + c0) * a.G;    // piece c, head g: ml[c * G + g]
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
        const int n = a.unit_len ? min(a.unit_len[u], a.cap) : a.n;
        const float* sc = a.scores + u * a.G * a.row_stride;
        const long long tot = u * (long long)a.total_stride;
#pragma unroll
        for (int i = 0; i < kFinishRows / kFinishThreads; ++i) {
            const int j = part * kFinishRows + i * kFinishThreads + threadIdx.x;
            if (j >= n) break;
            float sum = 0.f;
            for (int g = 0; g < a.G; ++g) sum = fmaf(fast_exp2(sc[(long long)g * a.row_stride + j] - s_max[g]), s_inv[g], sum);
            a.total_out[tot + j] = a.total_in ? a.total_in[tot + j] + sum : sum;
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
// Radix select on order-preserving 32-bit keys, eight bits per pass from the top: after four passes the key of the last
// row kept is known exactly, and how many rows with that very key stay.  One block per unit; a warp then walks its own
// contiguous stretch of rows twice (count, write), so that one scan over the 32 warps orders the whole list.
// --------------------------------------------------------------------------------------
constexpr int kSelectThreads = 1024;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kSelectCached = 49152;     // keys a block holds in shared memory; longer units are read again per pass

__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0u;                            // NaN: below minus infinity (whose key is 0x007fffff)
    const uint32_t b = __float_as_uint(x + 0.0f);     // -0 becomes +0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kSelectThreads) select_rows_kernel(const SelectArgs a, const __grid_constant__ SelectCounts counts,
                                                                     int cached) {
    extern __shared__ uint32_t cache[];
    __shared__ int hist[256];
    __shared__ int warp_gt[kSelectWarps], warp_eq[kSelectWarps];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need;
    const long long u = a.unit0 + blockIdx.x;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int n = a.unit_len ? a.unit_len[u] : a.n;
    const int want = counts.n[blockIdx.x] - a.n_recent;     // rows chosen by total
    const int old = n - a.n_recent;                         // rows they are chosen from
    const float* total = a.total + u * a.total_stride;
    const bool held = old <= cached;
    if (held) {
        for (int j = tid; j < old; j += kSelectThreads) cache[j] = order_key(total[j]);
    }
    auto key = [&](int j) { return held ? cache[j] : order_key(total[j]); };
    if (tid == 0) {
        s_prefix = 0;
        s_need = want;
    }
    __syncthreads();
    // `need` rows are still to be taken among the keys that begin with `prefix`
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        const uint32_t prefix = s_prefix;
        for (int j = tid; j < old; j += kSelectThreads) {
            const uint32_t k = key(j);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        if (warp == 0) {
            // lane i holds the counts of digits 255 - 8 i .. 248 - 8 i: largest first
            int c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = hist[255 - 8 * lane - i];
                sum += c[i];
            }
            int before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += y;
            }
            before -= sum;
            const int need = s_need;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < need && before + c[i] >= need) {      // exactly one digit of one lane
                    s_prefix = prefix | (uint32_t)(255 - 8 * lane - i) << shift;
                    s_need = need - before;
                }
                before += c[i];
            }
        }
        __syncthreads();
    }
    const uint32_t last = s_prefix;        // the smallest key kept; of the rows that have it the first `ties` stay
    const int ties = want > 0 ? s_need : 0;
    // contiguous stretches per warp, in multiples of 32 rows
    const int per = ((old + kSelectWarps - 1) / kSelectWarps + 31) / 32 * 32;
    const int j0 = min(old, warp * per), j1 = min(old, j0 + per);
    int gt = 0, eq = 0;
    if (want > 0)
        for (int j = j0; j < j1; j += 32) {
            const uint32_t k = j + lane < j1 ? key(j + lane) : 0u;
            const bool in = j + lane < j1;
            gt += __popc(__ballot_sync(0xffffffffu, in && k > last));
            eq += __popc(__ballot_sync(0xffffffffu, in && k == last));
        }
    if (lane == 0) {
        warp_gt[warp] = gt;
        warp_eq[warp] = eq;
    }
    __syncthreads();
    int eq_before = 0, pos = 0;
    for (int w = 0; w < warp; ++w) {
        pos += warp_gt[w];
        eq_before += warp_eq[w];
    }
    pos += min(eq_before, ties);
    int* keep = a.keep + u * a.keep_stride;
    float* kept = a.kept ? a.kept + u * a.keep_stride : nullptr;
    const uint32_t below = (1u << lane) - 1;
    if (want > 0)
        for (int j = j0; j < j1; j += 32) {
            const bool in = j + lane < j1;
            const uint32_t k = in ? key(j + lane) : 0u;
            const uint32_t meq = __ballot_sync(0xffffffffu, in && k == last);
            const bool take = in && (k > last || (k == last && eq_before + __popc(meq & below) < ties));
            const uint32_t mt = __ballot_sync(0xffffffffu, take);
            if (take) {
                const int p = pos + __popc(mt & below);
                keep[p] = j + lane;
                if (kept) kept[p] = total[j + lane];
            }
            pos += __popc(mt);
            eq_before += __popc(meq);
        }
    for (int j = old + tid; j < n; j += kSelectThreads) {
        keep[want + j - old] = j;
        if (kept) kept[want + j - old] = total[j];
    }
}

}  // namespace

cudaError_t init_weights_kernels() {
    return cudaFuncSetAttribute(select_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelectCached * 4);
}

cudaError_t launch_weights_finish(const DecodeArgs& a, const DecodePlan& plan, const float* total_in, float* total_out,
                                  int total_stride, cudaStream_t stream) {
    FinishArgs f;
    f.part_o = a.part_o;
    f.part_ml = a.part_ml;
    f.scores = a.scores;
    f.total_in = total_in;
    f.total_out = total_out;
    f.out = a.out;
    f.T = plan.T;
    f.total_stride = total_stride;
    f.row_stride = a.row_stride;
    f.G = a.G;
    f.tpu = plan.tpu;
    f.NC = plan.NC;
    f.n = a.n;
    f.tile_rows = plan.tile_rows;
    f.units = a.units;
    f.cap = a.capacity;
    f.n_extra = a.n_extra;
    f.unit_len = a.unit_len;
    f.chunks = ((a.n_extra ? a.capacity : a.n) + kFinishRows - 1) / kFinishRows;
    const dim3 grid((unsigned)(a.units * (f.chunks + a.G)));
    return a.D == 128 ? launch_kernel(weights_finish_kernel<128>, grid, dim3(kFinishThreads), 0, stream, a.programmatic, f)
                      : launch_kernel(weights_finish_kernel<64>, grid, dim3(kFinishThreads), 0, stream, a.programmatic, f);
}

cudaError_t launch_select(const SelectArgs& a, const SelectCounts& counts, cudaStream_t stream) {
    const int cached = std::min(kSelectCached, std::max(0, a.n - a.n_recent));
    select_rows_kernel<<<(unsigned)a.units, kSelectThreads, (size_t)cached * 4, stream>>>(a, counts, cached);
    return cudaGetLastError();
}

}  // namespace kvs
