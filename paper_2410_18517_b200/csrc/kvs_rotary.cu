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
// Bound: HBM for prompts (each byte read and written once), launch latency for decode steps.  A head row is read by
// D / 8 lanes of eight elements each: four neighbours and the four they are rotated with, so that no value has to cross
// lanes but the norm's sum (a layout of 16 contiguous bytes per lane needs eight shuffles a row for that).  A block
// takes several tokens of a long prompt: its threads work out one (token, pair) angle each while the first rows are on
// their way, and every block needs the table's latency only once.
#include <algorithm>

#include "kvs_device.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 4;    // tokens per block of a long prompt: as many rows a group of lanes has in flight

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
    int tokens;                                 // batch * n_new
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

// Four elements of storage: 8 (bf16) or 16 (fp32) bytes.
template <typename T>
struct Quad;
template <>
struct Quad<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void unpack(float* f) const {
        f[0] = __uint_as_float(v.x << 16);
        f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16);
        f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    __device__ __forceinline__ void pack(const float* f) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2], f[3]);
        v = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
};
template <>
struct Quad<float> {
    float4 v;
    __device__ __forceinline__ void unpack(float* f) const {
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    }
    __device__ __forceinline__ void pack(const float* f) { v = make_float4(f[0], f[1], f[2], f[3]); }
};

// INTERLEAVED: pairs are neighbours (2i, 2i+1); else pair i is (i, i + half).  TOKENS: tokens per block.
template <typename T, int D, bool INTERLEAVED, int TOKENS>
__global__ void __launch_bounds__(kRotThreads, 4) append_rotary_kernel(const __grid_constant__ RotaryKernelArgs a) {
    constexpr int LPR = D / 8;                    // lanes per head row, two quads each
    constexpr int ROWS = kRotThreads / LPR;       // head rows the block works on at once
    constexpr int RB = D * (int)sizeof(T);
    constexpr int QB = 4 * (int)sizeof(T);        // bytes of a quad
    // cos and sin apart: the lanes' 16-byte reads then hit different banks
    __shared__ __align__(16) float cos_t[TOKENS][D / 2], sin_t[TOKENS][D / 2];
    __shared__ int seq[TOKENS], row_in[TOKENS];
    pdl_launch_dependents();
    const int heads = a.Hq + 2 * a.Hkv;
    const int lig = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    // This lane's two quads of a row: its pairs' first and second elements; the quads that are not rotated are dealt
    // out to the lanes left over.  Interleaved pairs lie inside a quad.
    const int hq = a.half / 4;                    // quads of first elements
    int c0, c1;
    bool turn0, turn1;
    if (INTERLEAVED) {
        c0 = lig;
        c1 = lig + LPR;
        turn0 = c0 < 2 * hq;
        turn1 = c1 < 2 * hq;
    } else {
        turn0 = turn1 = lig < hq;
        c0 = turn0 ? lig : hq + lig;                              // 2 hq + (lig - hq)
        c1 = turn0 ? lig + hq : hq + lig + (LPR - hq);            // as many quads further on as are left over
    }
    const int passes = (heads + ROWS - 1) / ROWS;
    const int tok0 = blockIdx.x * TOKENS, ntok = min(TOKENS, a.tokens - tok0);
    // grid.y = 1: the block goes through all passes; else each block has one of them
    const int pass0 = gridDim.y == 1 ? 0 : blockIdx.y, pass1 = gridDim.y == 1 ? passes : pass0 + 1;
    pdl_wait();
    const int extra = a.n_extra ? *a.n_extra : 0;    // replayed launch: the slot has grown since it was recorded
    for (int pass = pass0; pass < pass1; ++pass) {
        // A group of lanes keeps its head row of the pass for all tokens of the block.
        const int r = pass * ROWS + slot;
        const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv, there = r < heads;
        const int h = is_q ? r : (is_v ? r - a.Hq - a.Hkv : r - a.Hq);
        const long long step = is_q ? a.q_stride : (is_v ? a.v_stride : a.k_stride);
        const char* src = (is_q ? a.q : (is_v ? a.v : a.k)) + tok0 * step + (long long)h * RB;
        const char* w = is_q ? a.q_weight : (is_v ? nullptr : a.k_weight);
        Quad<T> raw[TOKENS][2], w0 = {}, w1 = {};
#pragma unroll
        for (int i = 0; i < TOKENS; ++i)
            if (there && i < ntok) {
                raw[i][0] = *reinterpret_cast<const Quad<T>*>(src + i * step + c0 * QB);
                raw[i][1] = *reinterpret_cast<const Quad<T>*>(src + i * step + c1 * QB);
            }
        if (w != nullptr) {
            w0 = *reinterpret_cast<const Quad<T>*>(w + c0 * QB);
            w1 = *reinterpret_cast<const Quad<T>*>(w + c1 * QB);
        }
        if (pass == pass0) {
            for (int i = threadIdx.x; i < ntok * a.half; i += kRotThreads) {
                const int tk = i / a.half, pr = i - tk * a.half;
                double turn = (double)a.positions[tok0 + tk] * a.turns[pr];
                turn -= rint(turn);
                // the angle as hi + lo: rounding it to fp32 alone would cost as much again as the functions' own error
                const float hi = (float)turn, lo = (float)(turn - (double)hi) * 6.2831853f;
                float sn, cn;
                sincospif(2.0f * hi, &sn, &cn);
                cos_t[tk][pr] = fmaf(-sn, lo, cn);
                sin_t[tk][pr] = fmaf(cn, lo, sn);
            }
            if (threadIdx.x < ntok) {
                // where the token's row of unit 0 of its sequence goes (a ragged slot adds the unit's length later)
                const int tok = tok0 + threadIdx.x, b = tok / a.n_new, t = tok - b * a.n_new;
                seq[threadIdx.x] = b;
                row_in[threadIdx.x] = t + (a.unit_len ? 0 : a.len0 + extra);
            }
            __syncthreads();
        }
        if (!there) continue;
        float wf[8];
        w0.unpack(wf);
        w1.unpack(wf + 4);
        char* q_dst = a.q_out + ((long long)tok0 * a.Hq + r) * RB;      // (used where the row is a query's)
        const long long q_step = (long long)a.Hq * RB;
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            if (i >= ntok) break;
            if (!is_v) {
                float x[8];
                raw[i][0].unpack(x);
                raw[i][1].unpack(x + 4);
                if (w != nullptr) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
                    // (the lanes of a row come here together, other rows of the warp perhaps not)
                    const uint32_t group = LPR == 16 ? 0xffffu << (threadIdx.x & 16) : 0xffu << (threadIdx.x & 24);
#pragma unroll
                    for (int o = LPR / 2; o >= 1; o >>= 1) ss += __shfl_xor_sync(group, ss, o);
                    const float inv = rsqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * wf[e];
                }
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < 2 ? turn0 : turn1) {
                            const int pr = 2 * (q < 2 ? c0 : c1) + (q & 1);
                            const float c = cos_t[i][pr], sn = sin_t[i][pr], f = x[2 * q], g = x[2 * q + 1];
                            x[2 * q] = f * c - g * sn;
                            x[2 * q + 1] = g * c + f * sn;
                        }
                } else if (turn0) {
                    const float4 c4 = *reinterpret_cast<const float4*>(&cos_t[i][4 * c0]), s4 = *reinterpret_cast<const float4*>(&sin_t[i][4 * c0]);
                    const float c[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float f = x[q], g = x[4 + q];
                        x[q] = f * c[q] - g * sn[q];
                        x[4 + q] = g * c[q] + f * sn[q];
                    }
                }
                raw[i][0].pack(x);
                raw[i][1].pack(x + 4);
            }
            char* dst;
            if (is_q) {
                dst = q_dst + i * q_step;
            } else {
                const int u = seq[i] * a.Hkv + h;
                const int row = row_in[i] + (a.unit_len ? a.unit_len[u] : 0);
                if (row >= a.capacity) {               // only a replay that outran the capacity gets here
                    if (lig == 0) atomicExch(a.status, 4);
                    continue;
                }
                const long long off = ((long long)u * a.row_stride + row) * RB;
                if (!KVS_BOUNDS_OK(off, RB, a.plane_bytes, a.status)) continue;
                dst = (is_v ? a.vplane : a.kplane) + off;
            }
            *reinterpret_cast<Quad<T>*>(dst + c0 * QB) = raw[i][0];
            *reinterpret_cast<Quad<T>*>(dst + c1 * QB) = raw[i][1];
        }
    }
}

template <typename T, int D, int TOKENS>
cudaError_t launch_one(const RotaryKernelArgs& ka, bool interleaved, int passes, bool pdl, cudaStream_t stream) {
    const dim3 grid((unsigned)((ka.tokens + TOKENS - 1) / TOKENS), (unsigned)passes), block(kRotThreads);
    return interleaved ? launch_kernel(append_rotary_kernel<T, D, true, TOKENS>, grid, block, 0, stream, pdl, ka)
                       : launch_kernel(append_rotary_kernel<T, D, false, TOKENS>, grid, block, 0, stream, pdl, ka);
}

// Several tokens per block, and all head rows of a token in it, once that still leaves every SM its four blocks; below,
// one token per block and a block for every pass over its heads spread the few rows there are over the SMs.
template <typename T, int D>
cudaError_t launch_tokens(const RotaryKernelArgs& ka, bool interleaved, bool pdl, cudaStream_t stream) {
    if (ka.tokens >= kRotTokens * 4 * 148) return launch_one<T, D, kRotTokens>(ka, interleaved, 1, pdl, stream);
    const int rows = kRotThreads / (D / 8);
    return launch_one<T, D, 1>(ka, interleaved, (ka.Hq + 2 * ka.Hkv + rows - 1) / rows, pdl, stream);
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
    ka.tokens = r.batch * r.n_new;
    if (r.dtype == 0)
        return r.D == 128 ? launch_tokens<__nv_bfloat16, 128>(ka, r.interleaved, r.programmatic, stream)
                          : launch_tokens<__nv_bfloat16, 64>(ka, r.interleaved, r.programmatic, stream);
    return r.D == 128 ? launch_tokens<float, 128>(ka, r.interleaved, r.programmatic, stream)
                      : launch_tokens<float, 64>(ka, r.interleaved, r.programmatic, stream);
}

}  // namespace kvs
