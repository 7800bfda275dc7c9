// 4-bit caches: storing rows, reading them back, and decode attention over them for fp32 storage.
#include <algorithm>

#include "kvs_kernels.h"
#include "kvs_pack4.cuh"

namespace kvs {

namespace {

// --------------------------------------------------------------------------------------
// Storing.  A lane takes a group of a row, four lanes a row, rows dealt out with the tokens of a head in a run, so that what a
// warp writes is contiguous (see pack_group).
// Bound: HBM, 2 D e bytes in and D + 32 out per token and head, once the instructions are few: 4 x 4096 tokens of 8 heads of 128 took
// 67 us with 64-bit divisions and ties settled in fp64, 46 without, 24 with a group per lane, 22.8 without fp64 (88 MB: 3.9 TB/s).
// --------------------------------------------------------------------------------------
constexpr int kPackThreads = 256;

struct PackKernelArgs {
    const char* k;
    const char* v;
    char* kplane;
    char* vplane;
    long long src_b, src_t, src_h;      // bytes between sequences, tokens, heads of the source
    uint32_t rows;                      // batch * n_new * Hkv
    FastDiv by_token, by_head;          // n_new, Hkv
    int n_new, row_stride, len0, cap;
    const int* unit_len;
    const int* n_extra;
    int* status;
    long long plane_bytes;
};

template <typename T, int D>
__global__ void __launch_bounds__(kPackThreads) pack4_kernel(const PackKernelArgs a_in) {
    using R = Pack4Row<D>;
    constexpr int RPB = kPackThreads / 4;       // rows of a block's turn
    constexpr int WORDS = R::GROUP / 8;         // words of codes a lane makes
    constexpr int V = sizeof(T) / 2;            // 16-byte pieces of eight elements
    PackKernelArgs a = a_in;
    pdl_launch_dependents();
    pdl_wait();
    if (a.n_extra) a.len0 += *a.n_extra;        // replayed launch: the slot has grown since the launch was recorded
    if (!a.unit_len && a.len0 + a.n_new > a.cap) {
        if (threadIdx.x == 0 && blockIdx.x == 0) atomicExch(a.status, 4);
        return;
    }
    const char* src = blockIdx.y == 0 ? a.k : a.v;
    char* dst = blockIdx.y == 0 ? a.kplane : a.vplane;
    const uint32_t group = threadIdx.x % 4;
    for (uint32_t r = blockIdx.x * RPB + threadIdx.x / 4; r < a.rows; r += gridDim.x * RPB) {
        const uint32_t u = a.by_token.div(r), t = r - u * a.n_new;          // (sequence, head), token
        const uint32_t seq = a.by_head.div(u), h = u - seq * a.by_head.d;
        const uint4* p = reinterpret_cast<const uint4*>(src + seq * a.src_b + t * a.src_t + h * a.src_h) + group * WORDS * V;
        uint4 in[WORDS * V];
#pragma unroll
        for (int i = 0; i < WORDS * V; ++i) in[i] = p[i];
        const int first = a.unit_len ? a.unit_len[u] : a.len0;      // ragged slots append per unit
        if (first + (int)t >= a.cap) {     // only a replay that outran the capacity gets here
            atomicExch(a.status, 4);
            continue;
        }
        uint32_t pair, words[WORDS];
        pack_group<T, D>(in, &pair, words);
        const long long to = ((long long)u * a.row_stride + first + t) * R::RB;
        if (!KVS_BOUNDS_OK(to, R::RB, a.plane_bytes, a.status)) continue;
        uint32_t* row = reinterpret_cast<uint32_t*>(dst + to);
        store_group<D>(row, group, pair, words);
    }
}

// --------------------------------------------------------------------------------------
// Reading rows back, to [b][t][h] places of any strides.  packed: the values of a 4-bit row, eight per lane; otherwise a
// copy of the storage type's row.  Rows a unit does not hold become zeros.  Bound: HBM.
// --------------------------------------------------------------------------------------
// RUNS (long reads): a block takes a run of tokens of one unit, and offsets advance by additions; otherwise the rows of all units are
// dealt out one after the other.  (2 x 4096 tokens of 8 heads of 128: 16.2 us without runs, 11.9 with; storing gained nothing.)
constexpr int kReadRows = 4;        // rows a lane has in flight
constexpr int kRunRows = 256;       // tokens of a run

struct ReadKernelArgs {
    const char* kplane;
    const char* vplane;
    char* k_out;
    char* v_out;
    long long dst_b, dst_t, dst_h;      // bytes
    uint32_t rows;                      // batch * n * Hkv
    FastDiv by_token, by_head;          // n, Hkv
    int n, row_stride, first;
    const int* unit_len;
    int* status;
    long long plane_bytes, out_bytes;
};

// bf16 values of a word's eight codes, in order
__device__ __forceinline__ uint4 pack4_expand(uint32_t w, uint32_t pair) {
    const uint32_t s2 = __byte_perm(pair, pair, 0x1010), b2 = __byte_perm(pair, pair, 0x3232);
    const uint32_t v04 = fma_bf16x2(pack4_pair<0>(w), s2, b2), v15 = fma_bf16x2(pack4_pair<1>(w), s2, b2);
    const uint32_t v26 = fma_bf16x2(pack4_pair<2>(w), s2, b2), v37 = fma_bf16x2(pack4_pair<3>(w), s2, b2);
    return make_uint4(__byte_perm(v04, v15, 0x5410), __byte_perm(v26, v37, 0x5410), __byte_perm(v04, v15, 0x7632), __byte_perm(v26, v37, 0x7632));
}

template <typename T, int D, bool PACKED, bool RUNS>
__global__ void __launch_bounds__(256) read_rows_kernel(const ReadKernelArgs a) {
    constexpr int LPR = D / 8;
    constexpr int RPB = 256 / LPR;
    constexpr int RB = PACKED ? Pack4Row<D>::RB : D * (int)sizeof(T);
    constexpr int V = sizeof(T) / 2;            // 16-byte pieces of eight elements
    pdl_launch_dependents();
    pdl_wait();
    const char* src = blockIdx.y == 0 ? a.kplane : a.vplane;
    char* dst = blockIdx.y == 0 ? a.k_out : a.v_out;
    const uint32_t lane = threadIdx.x % LPR, step = RUNS ? RPB : gridDim.x * RPB;
    // RUNS: rows are numbered within the block's unit
    uint32_t base = threadIdx.x / LPR, end = a.rows;
    long long src0 = 0, dst0 = 0;
    int held = 0;
    if constexpr (RUNS) {
        const uint32_t runs = (a.n + kRunRows - 1) / kRunRows, u = blockIdx.x / runs, run = blockIdx.x - u * runs;
        const uint32_t seq = a.by_head.div(u), h = u - seq * a.by_head.d;
        base += run * kRunRows;
        end = min((uint32_t)a.n, (run + 1) * kRunRows);
        src0 = ((long long)u * a.row_stride + a.first) * RB;
        dst0 = seq * a.dst_b + h * a.dst_h;
        held = a.unit_len ? a.unit_len[u] - a.first : a.n;
    } else {
        base += blockIdx.x * RPB;
    }
    for (; base < end; base += kReadRows * step) {
        uint4 x[kReadRows][PACKED ? 1 : V];         // packed: the codes and the pair
        long long to[kReadRows];
        bool have[kReadRows];
#pragma unroll
        for (int j = 0; j < kReadRows; ++j) {
            const uint32_t r = base + j * step;
            to[j] = -1;
            have[j] = false;
            if (r >= end) continue;
            long long at;
            if constexpr (RUNS) {
                at = src0 + (long long)r * RB;
                to[j] = dst0 + r * a.dst_t;
                have[j] = (int)r < held;
            } else {
                const uint32_t u = a.by_token.div(r), t = r - u * a.n;
                const uint32_t seq = a.by_head.div(u), h = u - seq * a.by_head.d;
                at = ((long long)u * a.row_stride + a.first + t) * RB;
                to[j] = seq * a.dst_b + t * a.dst_t + h * a.dst_h;
                have[j] = !a.unit_len || a.first + (int)t < a.unit_len[u];
            }
            if (!KVS_BOUNDS_OK(at, RB, a.plane_bytes, a.status)) have[j] = false;
            if (!have[j]) continue;
            if constexpr (PACKED) {
                const uint32_t* row = reinterpret_cast<const uint32_t*>(src + at);
                x[j][0].x = row[4 + lane];
                x[j][0].y = row[lane / (LPR / 4)];
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) x[j][i] = reinterpret_cast<const uint4*>(src + at)[lane * V + i];
            }
        }
#pragma unroll
        for (int j = 0; j < kReadRows; ++j) {
            if (to[j] < 0) break;
            uint4 y[V];
            if (!have[j]) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = make_uint4(0u, 0u, 0u, 0u);
            } else if constexpr (!PACKED) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = x[j][i];
            } else if constexpr (V == 1) {
                y[0] = pack4_expand(x[j][0].x, x[j][0].y);
            } else {
                const uint32_t w = x[j][0].x;
                const float s = bf16_lo(x[j][0].y), b = bf16_hi(x[j][0].y);
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = pack4_value(w >> (4 * i) & 15u, s, b);
                y[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                y[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
            }
            if (KVS_BOUNDS_OK(to[j], D * (int)sizeof(T), a.out_bytes, a.status))
#pragma unroll
                for (int i = 0; i < V; ++i) reinterpret_cast<uint4*>(dst + to[j])[lane * V + i] = y[i];
        }
    }
}

// --------------------------------------------------------------------------------------
// Decode attention over a 4-bit cache, fp32 storage (the small configuration): plain fp32 arithmetic.  A block walks its
// share of the line of 64-row tiles (see DecodePlan); per tile four threads share a key, one group of the row each; a warp
// then owns a q-head's softmax; then a thread owns an output column over its part of the tile's rows.  Pieces are merged by
// the combine kernel.
// --------------------------------------------------------------------------------------
constexpr int kF32Tile = 64;

struct Pack4F32Args {
    const float* q;
    const char* kplane;
    const char* vplane;
    float* part_o;
    float* part_ml;
    int* status;
    int n, row_stride, cap, units, tpu;
    long long T;
    float scale_log2;
    const int* unit_len;
    const int* n_extra;
    long long plane_bytes;
};

template <int D, int G>
__global__ void __launch_bounds__(256) decode_pack4_f32(const Pack4F32Args a_in) {
    using R = Pack4Row<D>;
    constexpr int PARTS = 256 / D;
    Pack4F32Args a = a_in;
    __shared__ __align__(16) unsigned char tile[2][kF32Tile * R::RB];
    __shared__ float s_q[G][4][R::GROUP + 1];       // a group's elements apart, so that four threads read four banks
    __shared__ float s_p[G][kF32Tile];
    __shared__ float s_alpha[G];
    __shared__ float s_o[PARTS][G][D];
    pdl_wait();
    pdl_launch_dependents();      // in this order, as in every split-K kernel (see safe_rows_of)
    if (a.n_extra) {    // replayed launch: the lengths have grown on the device
        a.n = min(a.n + *a.n_extra, a.cap);
        a.tpu = (a.n + kF32Tile - 1) / kF32Tile;
        a.T = (long long)a.units * a.tpu;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long t1 = ((long long)(blockIdx.x + 1) * a.T) / gridDim.x;
    long long gt = ((long long)blockIdx.x * a.T) / gridDim.x;
    while (gt < t1) {
        const long long u = gt / a.tpu;
        const int ti0 = (int)(gt - u * a.tpu);
        const int piece_tiles = (int)min((long long)(a.tpu - ti0), t1 - gt);
        const int n_u = a.unit_len ? min(a.unit_len[u], a.cap) : a.n;
        float m = -1.0e30f, l = 0.f;                // of q-head `warp`, the same in all its lanes
        float o[G];
#pragma unroll
        for (int g = 0; g < G; ++g) o[g] = 0.f;
        __syncthreads();                            // the previous piece's readers are done
        for (int i = tid; i < G * D; i += 256) s_q[i / D][i % D / R::GROUP][i % R::GROUP] = a.q[u * G * D + i];
        for (int k = 0; k < piece_tiles; ++k) {
            const int row0 = (ti0 + k) * kF32Tile, valid = min(kF32Tile, n_u - row0);
            if (valid <= 0) break;                  // a ragged unit ended before this tile
            const long long at = (u * a.row_stride + row0) * (long long)R::RB;
            __syncthreads();
            if (KVS_BOUNDS_OK(at, valid * R::RB, a.plane_bytes, a.status))
                for (int i = tid; i < valid * R::RB / 16; i += 256) {
                    reinterpret_cast<uint4*>(tile[0])[i] = reinterpret_cast<const uint4*>(a.kplane + at)[i];
                    reinterpret_cast<uint4*>(tile[1])[i] = reinterpret_cast<const uint4*>(a.vplane + at)[i];
                }
            __syncthreads();
            {
                const int key = tid >> 2, part = tid & 3;
                float acc[G];
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g] = 0.f;
                if (key < valid) {
                    const uint32_t* row = reinterpret_cast<const uint32_t*>(tile[0] + key * R::RB);
                    const float s = bf16_lo(row[part]), b = bf16_hi(row[part]);
#pragma unroll
                    for (int x = 0; x < R::GROUP / 8; ++x) {
                        const uint32_t w = row[4 + part * (R::GROUP / 8) + x];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float val = pack4_value(w >> (4 * i) & 15u, s, b);
#pragma unroll
                            for (int g = 0; g < G; ++g) acc[g] = fmaf(s_q[g][part][8 * x + i], val, acc[g]);
                        }
                    }
                }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    acc[g] += __shfl_xor_sync(0xffffffffu, acc[g], 1);
                    acc[g] += __shfl_xor_sync(0xffffffffu, acc[g], 2);
                    if (part == 0) s_p[g][key] = key < valid ? acc[g] * a.scale_log2 : -INFINITY;
                }
            }
            __syncthreads();
            if (warp < G) {
                const float s0 = s_p[warp][lane], s1 = s_p[warp][lane + 32];
                float top = fmaxf(s0, s1);
#pragma unroll
                for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                const float m_new = fmaxf(m, top), alpha = fast_exp2(m - m_new);
                const float p0 = fast_exp2(s0 - m_new), p1 = fast_exp2(s1 - m_new);
                float sum = p0 + p1;
#pragma unroll
                for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                l = fmaf(l, alpha, sum);
                m = m_new;
                s_p[warp][lane] = p0;
                s_p[warp][lane + 32] = p1;
                if (lane == 0) s_alpha[warp] = alpha;
            }
            __syncthreads();
            const int d = tid % D, part = tid / D;
#pragma unroll
            for (int g = 0; g < G; ++g) o[g] *= s_alpha[g];
            for (int key = part; key < valid; key += PARTS) {
                const unsigned char* row = tile[1] + key * R::RB;
                const uint32_t pair = reinterpret_cast<const uint32_t*>(row)[d / R::GROUP];
                const uint32_t c = (uint32_t)(row[16 + d / 2] >> (4 * (d & 1))) & 15u;
                const float val = pack4_value(c, bf16_lo(pair), bf16_hi(pair));
#pragma unroll
                for (int g = 0; g < G; ++g) o[g] = fmaf(s_p[g][key], val, o[g]);
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) s_o[tid / D][g][tid % D] = o[g];
        __syncthreads();
        const long long pid = u + blockIdx.x;
        if (KVS_BOUNDS_OK(pid, 1, a.units + (long long)gridDim.x, a.status)) {
            for (int i = tid; i < G * D; i += 256) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < PARTS; ++j) sum += s_o[j][i / D][i % D];
                a.part_o[pid * G * D + i] = sum;
            }
            if (warp < G && lane == 0) {
                a.part_ml[(pid * G + warp) * 2] = m;
                a.part_ml[(pid * G + warp) * 2 + 1] = l;
            }
        }
        gt += piece_tiles;
    }
}

template <int D>
cudaError_t launch_f32_groups(int G, const Pack4F32Args& ka, int NC, bool pdl, cudaStream_t st) {
    switch (G) {
        case 1: return launch_kernel(decode_pack4_f32<D, 1>, dim3(NC), dim3(256), 0, st, pdl, ka);
        case 2: return launch_kernel(decode_pack4_f32<D, 2>, dim3(NC), dim3(256), 0, st, pdl, ka);
        case 4: return launch_kernel(decode_pack4_f32<D, 4>, dim3(NC), dim3(256), 0, st, pdl, ka);
        case 8: return launch_kernel(decode_pack4_f32<D, 8>, dim3(NC), dim3(256), 0, st, pdl, ka);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace

cudaError_t launch_pack4(const PackArgs& p, cudaStream_t stream) {
    PackKernelArgs a;
    const long long e = p.dtype == 0 ? 2 : 4;
    a.k = static_cast<const char*>(p.k);
    a.v = static_cast<const char*>(p.v);
    a.kplane = static_cast<char*>(p.kplane);
    a.vplane = static_cast<char*>(p.vplane);
    a.src_b = p.src_b * e;
    a.src_t = p.src_t * e;
    a.src_h = p.src_h * e;
    a.rows = (uint32_t)p.batch * p.n_new * p.Hkv;
    a.n_new = p.n_new;
    a.by_token = FastDiv(p.n_new);
    a.by_head = FastDiv(p.Hkv);
    a.row_stride = p.row_stride;
    a.len0 = p.len0;
    a.cap = p.capacity;
    a.unit_len = p.unit_len;
    a.n_extra = p.n_extra;
    a.status = p.status;
    a.plane_bytes = p.plane_bytes;
    const int rpb = kPackThreads / 4;
    if ((long long)p.batch * p.n_new * p.Hkv > 0x7fffffffll) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)std::min<long long>((a.rows + rpb - 1) / rpb, p.sm_count * 16), 2), block(kPackThreads);
    if (p.dtype == 0)
        return p.D == 128 ? launch_kernel(pack4_kernel<__nv_bfloat16, 128>, grid, block, 0, stream, p.programmatic, a)
                          : launch_kernel(pack4_kernel<__nv_bfloat16, 64>, grid, block, 0, stream, p.programmatic, a);
    return p.D == 128 ? launch_kernel(pack4_kernel<float, 128>, grid, block, 0, stream, p.programmatic, a)
                      : launch_kernel(pack4_kernel<float, 64>, grid, block, 0, stream, p.programmatic, a);
}

cudaError_t launch_read_rows(const ReadArgs& p, cudaStream_t stream) {
    ReadKernelArgs a;
    const long long e = p.dtype == 0 ? 2 : 4;
    a.kplane = static_cast<const char*>(p.kplane);
    a.vplane = static_cast<const char*>(p.vplane);
    a.k_out = static_cast<char*>(p.k_out);
    a.v_out = static_cast<char*>(p.v_out);
    a.dst_b = p.dst_b * e;
    a.dst_t = p.dst_t * e;
    a.dst_h = p.dst_h * e;
    a.rows = (uint32_t)p.batch * p.n * p.Hkv;
    a.n = p.n;
    a.by_token = FastDiv(p.n);
    a.by_head = FastDiv(p.Hkv);
    a.row_stride = p.row_stride;
    a.first = p.first;
    a.unit_len = p.unit_len;
    a.status = p.status;
    a.plane_bytes = p.plane_bytes;
    a.out_bytes = ((p.batch - 1) * p.dst_b + (p.n - 1) * p.dst_t + (p.Hkv - 1) * p.dst_h + p.D) * e;
    const int rpb = 256 / (p.D / 8);
    if ((long long)p.batch * p.n * p.Hkv > 0x7fffffffll) return cudaErrorInvalidValue;
    const bool runs = p.n >= kRunRows / 2;       // (a run as long as that occupies its block)
    const long long blocks = runs ? (long long)p.batch * p.Hkv * ((p.n + kRunRows - 1) / kRunRows)
                                  : std::min<long long>((a.rows + rpb - 1) / rpb, p.sm_count * 16);
    const dim3 grid((unsigned)blocks, 2), block(256);
#define KVS_READ2(T, D, P) (runs ? launch_kernel(read_rows_kernel<T, D, P, true>, grid, block, 0, stream, p.programmatic, a) \
                                 : launch_kernel(read_rows_kernel<T, D, P, false>, grid, block, 0, stream, p.programmatic, a))
#define KVS_READ(T, D) (p.packed ? KVS_READ2(T, D, true) : KVS_READ2(T, D, false))
    if (p.dtype == 0) return p.D == 128 ? KVS_READ(__nv_bfloat16, 128) : KVS_READ(__nv_bfloat16, 64);
    return p.D == 128 ? KVS_READ(float, 128) : KVS_READ(float, 64);
#undef KVS_READ
#undef KVS_READ2
}

void plan_decode_pack4_f32(int units, int n, int sm_count, int max_ctas, DecodePlan* plan) {
    int cap = sm_count * 2;
    if (max_ctas > 0) cap = std::min(cap, max_ctas);
    cap = std::min(cap, kMaxCtas);
    plan->tile_rows = kF32Tile;
    plan->tpu = (n + kF32Tile - 1) / kF32Tile;
    plan->T = (long long)units * plan->tpu;
    plan->NC = (int)std::min<long long>(plan->T, cap);
    plan->kernel = 4;
}

cudaError_t launch_decode_pack4_f32(const DecodeArgs& a, const DecodePlan& plan, cudaStream_t stream) {
    Pack4F32Args ka;
    ka.q = static_cast<const float*>(a.q);
    ka.kplane = static_cast<const char*>(a.kplane);
    ka.vplane = static_cast<const char*>(a.vplane);
    ka.part_o = a.part_o;
    ka.part_ml = a.part_ml;
    ka.status = a.status;
    ka.n = a.n;
    ka.row_stride = a.row_stride;
    ka.cap = a.capacity;
    ka.units = a.units;
    ka.tpu = plan.tpu;
    ka.T = plan.T;
    ka.scale_log2 = a.scale_log2;
    ka.unit_len = a.unit_len;
    ka.n_extra = a.n_extra;
    ka.plane_bytes = a.plane_bytes;
    return a.D == 128 ? launch_f32_groups<128>(a.G, ka, plan.NC, a.programmatic, stream)
                      : launch_f32_groups<64>(a.G, ka, plan.NC, a.programmatic, stream);
}

}  // namespace kvs
