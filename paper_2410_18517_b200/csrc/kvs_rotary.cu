// Rotary append: new tokens enter a layer's slot through one pass that normalises every query and key head
// (root mean square over the head, optional), rotates them to their positions and stores keys and values
// straight into the planes, queries into the caller's buffer.
//
//   x' = x * rsqrt(mean(x^2) + eps) * w               per (token, head); left out where no weight is given
//   pair (x0, x1) of index i -> (x0 c - x1 s, x1 c + x0 s),  c, s = cos, sin(position * inv_freq[i])
//
// Everything is fp32 and rounded to the storage type once, at the store.  Only the angle needs more: positions
// reach 10^6 and more, where an fp32 angle is off by hundredths of a radian, so position * inv_freq / 2 pi is
// formed in fp64, reduced to half a turn there, and only the remainder goes to fp32 (one fp64 product per
// (token, pair), shared by all heads of the token).
//
// Bound: HBM for prompts (each byte read and written once), launch latency for decode steps.  One block per
// token (several where a token has many heads): a head row is read by row_bytes / 16 lanes, 16 bytes each; the block
// issues its loads before it works out the cos / sin table, so that the table's latency hides behind them.
#include <algorithm>

#include "kvs_device.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotVecs = 4;      // 16-byte vectors a thread has in flight

struct RotaryKernelArgs {
    const char* q;
    const char* k;
    const char* v;
    long long q_stride, k_stride, v_stride;     // bytes between consecutive tokens
    const int* positions;                       // [tokens]
    const char* q_weight;                       // [D] or nullptr
    const char* k_weight;
    char* q_out;                                // [tokens][Hq][D]
    char* kplane;
    char* vplane;
    int Hq, Hkv;                                // Hkv = 0: queries only (a layer that shares its cache)
    int n_new;
    int row_stride;
    int len0;
    const int* unit_len;
    const int* n_extra;
    int capacity;
    int* status;
    long long plane_bytes;
    int half;                                   // rotated pairs per head
    float eps;
    double turns[64];                           // inv_freq[i] / 2 pi
};

template <typename T>
__device__ __forceinline__ uint4 pack_row(const float (&f)[16 / sizeof(T)]) {
    uint4 r;
    if constexpr (sizeof(T) == 2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&p);
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        r = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    return r;
}

// INTERLEAVED: pairs are neighbours (2i, 2i+1); else pair i is (i, i + half), half a multiple of a lane's elements.
template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotThreads) append_rotary_kernel(const __grid_constant__ RotaryKernelArgs a) {
    constexpr int EPL = 16 / (int)sizeof(T);
    constexpr int LPR = D / EPL;
    constexpr int ROWS = kRotThreads / LPR;       // head rows the block works on at once
    constexpr int RB = D * (int)sizeof(T);
    __shared__ float2 cs[D / 2];
    pdl_launch_dependents();
    pdl_wait();
    const int extra = a.n_extra ? *a.n_extra : 0;    // replayed launch: the slot has grown since it was recorded
    const long long tok = blockIdx.x;
    const int b = (int)(tok / a.n_new), t = (int)(tok - (long long)b * a.n_new);
    const int heads = a.Hq + 2 * a.Hkv;
    const int lig = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    // this block's share of the token's head rows (blockIdx.y of gridDim.y)
    const int r0 = (int)((long long)heads * blockIdx.y / gridDim.y), r1 = (int)((long long)heads * (blockIdx.y + 1) / gridDim.y);
    bool table = false;
    for (int rb = r0; rb < r1; rb += ROWS * kRotVecs) {
        uint4 raw[kRotVecs];
#pragma unroll
        for (int i = 0; i < kRotVecs; ++i) {
            const int r = rb + i * ROWS + slot;
            raw[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < r1) {
                const char* src = r < a.Hq ? a.q + tok * a.q_stride + (long long)r * RB
                                 : r < a.Hq + a.Hkv ? a.k + tok * a.k_stride + (long long)(r - a.Hq) * RB
                                                    : a.v + tok * a.v_stride + (long long)(r - a.Hq - a.Hkv) * RB;
                raw[i] = *reinterpret_cast<const uint4*>(src + lig * 16);
            }
        }
        if (!table) {
            for (int i = threadIdx.x; i < a.half; i += kRotThreads) {
                double turn = (double)a.positions[tok] * a.turns[i];
                turn -= rint(turn);
                float sn, cn;
                sincospif(2.0f * (float)turn, &sn, &cn);
                cs[i] = make_float2(cn, sn);
            }
            __syncthreads();
            table = true;
        }
#pragma unroll
        for (int i = 0; i < kRotVecs; ++i) {
            // (whole warps agree on r >= r1 only by chance: the exchange below needs every lane, the store is guarded)
            const int r = rb + i * ROWS + slot;
            const bool is_v = r >= a.Hq + a.Hkv;
            uint4 res = raw[i];
            float x[EPL];
            Unpack<T>::run(raw[i], x);
            const char* w = r < a.Hq ? a.q_weight : a.k_weight;
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int o = LPR / 2; o >= 1; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            if (w != nullptr) {
                const float inv = rsqrtf(ss * (1.0f / D) + a.eps);
                float wf[EPL];
                Unpack<T>::run(*reinterpret_cast<const uint4*>(w + lig * 16), wf);
#pragma unroll
                for (int e = 0; e < EPL; ++e) x[e] = x[e] * inv * wf[e];
            }
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < EPL; e += 2) {
                    const int p = (lig * EPL + e) / 2;
                    if (p < a.half) {
                        const float2 c = cs[p];
                        const float x0 = x[e], x1 = x[e + 1];
                        x[e] = x0 * c.x - x1 * c.y;
                        x[e + 1] = x1 * c.x + x0 * c.y;
                    }
                }
            } else {
                const int hl = a.half / EPL;           // lanes that hold first elements of pairs
                const bool first = lig < hl;
                const int partner = first ? lig + hl : (lig < 2 * hl ? lig - hl : lig);
                float y[EPL];
#pragma unroll
                for (int e = 0; e < EPL; ++e) y[e] = __shfl_sync(0xffffffffu, x[e], partner, LPR);
                if (lig < 2 * hl) {
                    const int p = (first ? lig : lig - hl) * EPL;
#pragma unroll
                    for (int e = 0; e < EPL; ++e) {
                        const float2 c = cs[p + e];
                        x[e] = first ? x[e] * c.x - y[e] * c.y : x[e] * c.x + y[e] * c.y;
                    }
                }
            }
            if (!is_v) res = pack_row<T>(x);
            if (r >= r1) continue;
            if (r < a.Hq) {
                *reinterpret_cast<uint4*>(a.q_out + (tok * a.Hq + r) * RB + lig * 16) = res;
            } else {
                const int h = is_v ? r - a.Hq - a.Hkv : r - a.Hq;
                const long long u = (long long)b * a.Hkv + h;
                const int row = (a.unit_len ? a.unit_len[u] : a.len0) + (a.unit_len ? 0 : extra) + t;
                if (row >= a.capacity) {               // only a replay that outran the capacity gets here
                    if (lig == 0) atomicExch(a.status, 4);
                    continue;
                }
                const long long dst = (u * a.row_stride + row) * (long long)RB + lig * 16;
                if (!KVS_BOUNDS_OK(dst, 16, a.plane_bytes, a.status)) continue;
                *reinterpret_cast<uint4*>((is_v ? a.vplane : a.kplane) + dst) = res;
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch_one(const RotaryKernelArgs& ka, bool interleaved, dim3 grid, bool pdl, cudaStream_t stream) {
    return interleaved ? launch_kernel(append_rotary_kernel<T, D, true>, grid, dim3(kRotThreads), 0, stream, pdl, ka)
                       : launch_kernel(append_rotary_kernel<T, D, false>, grid, dim3(kRotThreads), 0, stream, pdl, ka);
}

}  // namespace

cudaError_t launch_append_rotary(const RotaryArgs& r, cudaStream_t stream) {
    RotaryKernelArgs ka;
    const int e = r.dtype == 0 ? 2 : 4;
    ka.q = static_cast<const char*>(r.q);
    ka.k = static_cast<const char*>(r.k);
    ka.v = static_cast<const char*>(r.v);
    ka.q_stride = r.q_stride * e;
    ka.k_stride = r.k_stride * e;
    ka.v_stride = r.v_stride * e;
    ka.positions = r.positions;
    ka.q_weight = static_cast<const char*>(r.q_weight);
    ka.k_weight = static_cast<const char*>(r.k_weight);
    ka.q_out = static_cast<char*>(r.q_out);
    ka.kplane = static_cast<char*>(r.kplane);
    ka.vplane = static_cast<char*>(r.vplane);
    ka.Hq = r.Hq;
    ka.Hkv = r.Hkv;
    ka.n_new = r.n_new;
    ka.row_stride = r.row_stride;
    ka.len0 = r.len0;
    ka.unit_len = r.unit_len;
    ka.n_extra = r.n_extra;
    ka.capacity = r.capacity;
    ka.status = r.status;
    ka.plane_bytes = r.plane_bytes;
    ka.half = r.rotary_dim / 2;
    ka.eps = r.eps;
    for (int i = 0; i < 64; ++i) ka.turns[i] = i < ka.half ? r.inv_freq[i] * 0.15915494309189533577 : 0.0;   // 1 / 2 pi
    const long long tokens = (long long)r.batch * r.n_new;
    const dim3 grid((unsigned)tokens, 1);
    if (r.dtype == 0)
        return r.D == 128 ? launch_one<__nv_bfloat16, 128>(ka, r.interleaved, grid, r.programmatic, stream)
                          : launch_one<__nv_bfloat16, 64>(ka, r.interleaved, grid, r.programmatic, stream);
    return r.D == 128 ? launch_one<float, 128>(ka, r.interleaved, grid, r.programmatic, stream)
                      : launch_one<float, 64>(ka, r.interleaved, grid, r.programmatic, stream);
}

}  // namespace kvs
