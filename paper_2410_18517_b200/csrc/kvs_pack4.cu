// 4-bit caches: storing rows, reading them back, and decode attention over them for fp32 storage.
#include <algorithm>

#include "kvs_kernels.h"
#include "kvs_pack4.cuh"

namespace kvs {

namespace {

// --------------------------------------------------------------------------------------
// Storing.  A lane takes eight neighbouring elements of a row: their smallest and largest go around the D/32 lanes of the
// group by shuffles, the eight codes make one word of the row.  Rows are dealt out with the tokens of a head in a run, so
// that what a warp writes is contiguous.  In fp32 the quotient, at most 32, is off by less than 1e-5: a code next to the
// border between two is settled by the sign of x - b - (k + 1/2) s, which two fp32 operations and their remainders give exactly.
// (Ties are real, bf16 elements lie on few values: of normal draws 1 in 300, so that two warps in five have one.)
// Bound: HBM, 2 D e bytes in and D + 32 out per token and head.
// --------------------------------------------------------------------------------------
constexpr int kPackThreads = 256;
constexpr int kPackRows = 2;        // rows a lane has in flight

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

__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.4028234e38f; }

__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// smallest and largest of a lane's eight elements
__device__ __forceinline__ void range_of(const uint4 (&in)[1], float* lo, float* hi) {      // bf16: two at a time
    const uint32_t l = min_bf16x2(min_bf16x2(in[0].x, in[0].y), min_bf16x2(in[0].z, in[0].w));
    const uint32_t h = max_bf16x2(max_bf16x2(in[0].x, in[0].y), max_bf16x2(in[0].z, in[0].w));
    *lo = min_nan(bf16_lo(l), bf16_hi(l));
    *hi = max_nan(bf16_lo(h), bf16_hi(h));
}
__device__ __forceinline__ void range_of(const uint4 (&in)[2], float* lo, float* hi) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(in);
    *lo = *hi = __uint_as_float(w[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        *lo = min_nan(*lo, __uint_as_float(w[i]));
        *hi = max_nan(*hi, __uint_as_float(w[i]));
    }
}

// The group's pair s | b << 16 and the lane's eight codes.  All lanes of a group call it together; LANES per group.
template <int LANES>
__device__ __forceinline__ void pack_eight(const float (&x)[8], float lo, float hi, uint32_t* pair, uint32_t* codes) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    const float step = __fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f);
    const float s = __uint_as_float((__float_as_uint(step) + 0xffffu) & 0xffff0000u);
    const float b = __bfloat162float(__float2bfloat16_rn(__fsub_rn(lo, 16.f * s)));
    const bool broken = !(finite(step) && finite(s) && finite(b));
    // rint by adding 1.5 * 2^23; the codes are the lowest four bits of 16 + c
    constexpr float kRint = 12582912.f;
    const float inv = 1.f / s;
    float f[8], worst = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(__fsub_rn(x[i], b), inv);
    // Clamped to 16 .. 31 only where the rounding of b, up to 2^-8 |b|, can take the quotient past 15.5 or 31.5.
    if (fabsf(b) > 100.f * s)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = fminf(fmaxf(f[i], 16.f), 31.f);
    uint32_t word = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
        const float r = __fadd_rn(f[i], kRint);
        worst = fmaxf(worst, fabsf(__fsub_rn(f[i], __fsub_rn(r, kRint))));
        word = word * 16 + (__float_as_uint(r) & 15u);
    }
    if (__any_sync(0xffffffffu, worst > 0.4999f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float r = __fsub_rn(__fadd_rn(f[i], kRint), kRint);
            const float rest = __fsub_rn(f[i], r);
            const bool near = fabsf(rest) > 0.4999f;
            if (!__any_sync(0xffffffffu, near)) continue;
            const float below = rest >= 0.f ? r : r - 1.f;              // the border next to f is below + 1/2
            const float d = __fsub_rn(x[i], b), back = __fsub_rn(x[i], d);
            const float lost = __fadd_rn(__fsub_rn(x[i], __fadd_rn(d, back)), __fsub_rn(back, b));      // x - b = d + lost exactly
            const float side = __fadd_rn(__fmaf_rn(-(below + 0.5f), s, d), lost);
            r = side > 0.f ? below + 1.f : side < 0.f ? below : below + ((int)below & 1);
            r = fminf(fmaxf(r, 16.f), 31.f);
            if (near) word = (word & ~(15u << (4 * i))) | ((uint32_t)r & 15u) << (4 * i);
        }
    }
    if (s < 1e-30f && !broken) {                // s = 0, or its reciprocal may overflow and products may lose bits
        word = 0;
        if (s > 0.f)
            for (int i = 7; i >= 0; --i) {
                const double q = rint(((double)x[i] - (double)b) / (double)s);
                word = word * 16 + (uint32_t)(fmin(fmax(q, 16.0), 31.0) - 16.0);
            }
    }
    *pair = broken ? 0x7fc07fc0u : (__float_as_uint(s) >> 16) | (__float_as_uint(b) & 0xffff0000u);
    *codes = broken ? 0u : word;
}

template <typename T, int D>
__global__ void __launch_bounds__(kPackThreads) pack4_kernel(const PackKernelArgs a_in) {
    using R = Pack4Row<D>;
    constexpr int LPR = D / 8;                  // lanes per row
    constexpr int RPB = kPackThreads / LPR;     // rows of a block's turn
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
    const uint32_t lane = threadIdx.x % LPR, step = gridDim.x * RPB;
    for (uint32_t base = blockIdx.x * RPB; base < a.rows; base += kPackRows * step) {
        constexpr int V = sizeof(T) / 2;        // 16-byte pieces of eight elements
        uint4 in[kPackRows][V];
        long long to[kPackRows];
#pragma unroll
        for (int j = 0; j < kPackRows; ++j) {
            const uint32_t r = base + threadIdx.x / LPR + j * step;
            to[j] = -1;
            if (r < a.rows) {
                const uint32_t u = a.by_token.div(r), t = r - u * a.n_new;          // (sequence, head), token
                const uint32_t seq = a.by_head.div(u), h = u - seq * a.by_head.d;
                const uint4* p = reinterpret_cast<const uint4*>(src + seq * a.src_b + t * a.src_t + h * a.src_h) + lane * V;
#pragma unroll
                for (int i = 0; i < V; ++i) in[j][i] = __ldcs(p + i);
                const int first = a.unit_len ? a.unit_len[u] : a.len0;      // ragged slots append per unit
                if (first + (int)t < a.cap) {
                    to[j] = ((long long)u * a.row_stride + first + t) * R::RB;
                    if (!KVS_BOUNDS_OK(to[j], R::RB, a.plane_bytes, a.status)) to[j] = -1;
                } else if (lane == 0) {     // only a replay that outran the capacity gets here
                    atomicExch(a.status, 4);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) in[j][i] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
#pragma unroll
        for (int j = 0; j < kPackRows; ++j) {
            float x[8];
            if constexpr (V == 1) {
                Unpack<T>::run(in[j][0], x);
            } else {
                Unpack<T>::run(in[j][0], *reinterpret_cast<float(*)[4]>(x));
                Unpack<T>::run(in[j][1], *reinterpret_cast<float(*)[4]>(x + 4));
            }
            float lo, hi;
            range_of(in[j], &lo, &hi);
            uint32_t pair, codes;
            pack_eight<R::GROUP / 8>(x, lo, hi, &pair, &codes);
            if (to[j] >= 0) {
                uint32_t* row = reinterpret_cast<uint32_t*>(dst + to[j]);
                row[4 + lane] = codes;
                if (lane % (R::GROUP / 8) == 0) row[lane / (R::GROUP / 8)] = pair;
            }
        }
    }
}

// --------------------------------------------------------------------------------------
// Reading rows back, to [b][t][h] places of any strides.  packed: the values of a 4-bit row, eight per lane; otherwise a
// copy of the storage type's row.  Rows a unit does not hold become zeros.  Bound: HBM.
// --------------------------------------------------------------------------------------
constexpr int kReadRows = 4;        // rows a lane has in flight

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

template <typename T, int D, bool PACKED>
__global__ void __launch_bounds__(256) read_rows_kernel(const ReadKernelArgs a) {
    constexpr int LPR = D / 8;
    constexpr int RPB = 256 / LPR;
    constexpr int RB = PACKED ? Pack4Row<D>::RB : D * (int)sizeof(T);
    constexpr int V = sizeof(T) / 2;            // 16-byte pieces of eight elements
    pdl_launch_dependents();
    pdl_wait();
    const char* src = blockIdx.y == 0 ? a.kplane : a.vplane;
    char* dst = blockIdx.y == 0 ? a.k_out : a.v_out;
    const uint32_t lane = threadIdx.x % LPR, step = gridDim.x * RPB;
    for (uint32_t base = blockIdx.x * RPB + threadIdx.x / LPR; base < a.rows; base += kReadRows * step) {
        uint4 x[kReadRows][PACKED ? 1 : V];         // packed: the codes and the pair
        long long to[kReadRows];
        bool have[kReadRows];
#pragma unroll
        for (int j = 0; j < kReadRows; ++j) {
            const uint32_t r = base + j * step;
            to[j] = -1;
            have[j] = false;
            if (r >= a.rows) continue;
            const uint32_t u = a.by_token.div(r), t = r - u * a.n;
            const uint32_t seq = a.by_head.div(u), h = u - seq * a.by_head.d;
            const long long at = ((long long)u * a.row_stride + a.first + t) * RB;
            to[j] = seq * a.dst_b + t * a.dst_t + h * a.dst_h;
            have[j] = !a.unit_len || a.first + (int)t < a.unit_len[u];
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
    pdl_launch_dependents();
    pdl_wait();
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
    const int rpb = kPackThreads / (p.D / 8);
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
    const dim3 grid((unsigned)std::min<long long>((a.rows + rpb - 1) / rpb, p.sm_count * 16), 2), block(256);
#define KVS_READ(T, D) (p.packed ? launch_kernel(read_rows_kernel<T, D, true>, grid, block, 0, stream, p.programmatic, a) \
                                 : launch_kernel(read_rows_kernel<T, D, false>, grid, block, 0, stream, p.programmatic, a))
    if (p.dtype == 0) return p.D == 128 ? KVS_READ(__nv_bfloat16, 128) : KVS_READ(__nv_bfloat16, 64);
    return p.D == 128 ? KVS_READ(float, 128) : KVS_READ(float, 64);
#undef KVS_READ
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
