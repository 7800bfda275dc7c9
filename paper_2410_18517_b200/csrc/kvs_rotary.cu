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
// lanes but the norm's sum (a layout of 16 contiguous bytes per lane needs eight shuffles a row for that).  Long prompts
// go through persistent blocks whose rows arrive by bulk copies ahead of their use; what then holds them is as much the
// issue of some 130 instructions per eight elements and lane as the memory, hence the packed two-float products.
// 16384 bf16 tokens of 32 + 2 x 8 heads of 128, norm and rotation: 73 us for 403 MB, 5.5 TB/s (82 us with a block per
// four tokens, 77 us before the packed products); eight tokens of them 2.9 us.
#include <algorithm>

#include "kvs_device.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

constexpr int kRotThreads = 256;

struct RotaryKernelArgs {
    const char* q;
    const char* k;
    const char* v;
    long long q_stride, k_stride, v_stride;     // bytes between consecutive tokens
    const int* positions;                       // [tokens]; may be nullptr where half is 0
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

// This lane's two quads of a row: its pairs' first and second elements; the quads that are not rotated are dealt out to the
// lanes left over.  Interleaved pairs lie inside a quad.
template <int LPR, bool INTERLEAVED>
struct Lane {
    int c0, c1;
    bool turn0, turn1;
    __device__ __forceinline__ Lane(int lig, int half) {
        const int hq = half / 4;                      // quads of first elements
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
    }
};

// Entry `pr` of a token's table: cos and sin of position * inv_freq.
__device__ __forceinline__ void table_entry(int position, double turns, float* c, float* s) {
    double turn = (double)position * turns;
    turn -= rint(turn);
    // the angle as hi + lo: rounding it to fp32 alone would cost as much again as the functions' own error
    const float hi = (float)turn, lo = (float)(turn - (double)hi) * 6.2831853f;
    float sn, cn;
    sincospif(2.0f * hi, &sn, &cn);
    *c = fmaf(-sn, lo, cn);
    *s = fmaf(cn, lo, sn);
}

// Norm (where there is a weight, wf) and rotation of a row's eight elements in this lane.
template <int LPR, int D, bool INTERLEAVED>
__device__ __forceinline__ void finish_row(float (&x)[8], bool norm, const float (&wf)[8], float eps, const Lane<LPR, INTERLEAVED>& ln,
                                           const float* cos_t, const float* sin_t) {
    if (norm) {
        float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 8; e += 2) s2 = __ffma2_rn(make_float2(x[e], x[e + 1]), make_float2(x[e], x[e + 1]), s2);
        float ss = s2.x + s2.y;
        // (the lanes of a row come here together, other rows of the warp perhaps not)
        const uint32_t group = LPR == 16 ? 0xffffu << (threadIdx.x & 16) : 0xffu << (threadIdx.x & 24);
#pragma unroll
        for (int o = LPR / 2; o >= 1; o >>= 1) ss += __shfl_xor_sync(group, ss, o);
        const float inv = rsqrtf(ss * (1.0f / D) + eps);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float2 p = __fmul2_rn(__fmul2_rn(make_float2(x[e], x[e + 1]), make_float2(inv, inv)), make_float2(wf[e], wf[e + 1]));
            x[e] = p.x;
            x[e + 1] = p.y;
        }
    }
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < 2 ? ln.turn0 : ln.turn1) {
                const int pr = 2 * (q < 2 ? ln.c0 : ln.c1) + (q & 1);
                const float c = cos_t[pr], sn = sin_t[pr], f = x[2 * q], g = x[2 * q + 1];
                x[2 * q] = f * c - g * sn;
                x[2 * q + 1] = g * c + f * sn;
            }
    } else if (ln.turn0) {
        const float4 c4 = *reinterpret_cast<const float4*>(cos_t + 4 * ln.c0), s4 = *reinterpret_cast<const float4*>(sin_t + 4 * ln.c0);
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            const float2 f = make_float2(x[q], x[q + 1]), g = make_float2(x[4 + q], x[5 + q]);
            const float2 cc = make_float2(c[q], c[q + 1]), s2 = make_float2(sn[q], sn[q + 1]);
            const float2 u = __ffma2_rn(f, cc, __fmul2_rn(g, make_float2(-s2.x, -s2.y))), v = __ffma2_rn(g, cc, __fmul2_rn(f, s2));
            x[q] = u.x, x[q + 1] = u.y, x[4 + q] = v.x, x[5 + q] = v.y;
        }
    }
}

// Where row r of a token goes: nullptr past the capacity (only a replay that outran it gets there).  `seq`, `row`: the
// token's sequence and row in its units (of a ragged slot: behind the unit's length).
template <int RB>
__device__ __forceinline__ char* target(const RotaryKernelArgs& a, long long tok, int r, int h, bool is_q, bool is_v, int seq, int row, bool report) {
    if (is_q) return KVS_BOUNDS_OK(tok, 1, a.tokens, a.status) ? a.q_out + (tok * a.Hq + r) * RB : nullptr;
    const int u = seq * a.Hkv + h;
    if (a.unit_len) row += a.unit_len[u];
    if (row >= a.capacity) {
        if (report) atomicExch(a.status, 4);
        return nullptr;
    }
    const long long off = ((long long)u * a.row_stride + row) * RB;
    if (!KVS_BOUNDS_OK(off, RB, a.plane_bytes, a.status)) return nullptr;
    return (is_v ? a.vplane : a.kplane) + off;
}

// Few or short tokens: block (token, pass) takes as many of the token's head rows as it has threads for.
template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotThreads) append_rotary_kernel(const __grid_constant__ RotaryKernelArgs a) {
    constexpr int LPR = D / 8;                    // lanes per head row, two quads each
    constexpr int RB = D * (int)sizeof(T);
    constexpr int QB = 4 * (int)sizeof(T);        // bytes of a quad
    // cos and sin apart: the lanes' 16-byte reads then hit different banks
    __shared__ __align__(16) float cos_t[D / 2], sin_t[D / 2];
    pdl_launch_dependents();
    const int lig = threadIdx.x % LPR, slot = threadIdx.x / LPR, tok = blockIdx.x;
    const Lane<LPR, INTERLEAVED> ln(lig, a.half);
    const int r = blockIdx.y * (blockDim.x / LPR) + slot;
    const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv, there = r < a.Hq + 2 * a.Hkv;
    const int h = is_q ? r : (is_v ? r - a.Hq - a.Hkv : r - a.Hq);
    const char* src = (is_q ? a.q + tok * a.q_stride : (is_v ? a.v + tok * a.v_stride : a.k + tok * a.k_stride)) + (long long)h * RB;
    const char* w = is_q ? a.q_weight : (is_v ? nullptr : a.k_weight);
    pdl_wait();
    const int extra = a.n_extra ? *a.n_extra : 0;    // replayed launch: the slot has grown since it was recorded
    Quad<T> q0 = {}, q1 = {}, w0 = {}, w1 = {};
    if (there) {
        q0 = *reinterpret_cast<const Quad<T>*>(src + ln.c0 * QB);
        q1 = *reinterpret_cast<const Quad<T>*>(src + ln.c1 * QB);
        if (w != nullptr) {
            w0 = *reinterpret_cast<const Quad<T>*>(w + ln.c0 * QB);
            w1 = *reinterpret_cast<const Quad<T>*>(w + ln.c1 * QB);
        }
    }
    // the table while the rows are on their way
    for (int i = threadIdx.x; i < a.half; i += blockDim.x) table_entry(a.positions[tok], a.turns[i], &cos_t[i], &sin_t[i]);
    __syncthreads();
    if (!there) return;
    if (!is_v) {
        float x[8], wf[8];
        q0.unpack(x);
        q1.unpack(x + 4);
        w0.unpack(wf);
        w1.unpack(wf + 4);
        finish_row<LPR, D, INTERLEAVED>(x, w != nullptr, wf, a.eps, ln, cos_t, sin_t);
        q0.pack(x);
        q1.pack(x + 4);
    }
    const int b = tok / a.n_new;
    char* dst = target<RB>(a, tok, r, h, is_q, is_v, b, tok - b * a.n_new + (a.unit_len ? 0 : a.len0 + extra), lig == 0);
    if (dst == nullptr) return;
    *reinterpret_cast<Quad<T>*>(dst + ln.c0 * QB) = q0;
    *reinterpret_cast<Quad<T>*>(dst + ln.c1 * QB) = q1;
}

// Many tokens: persistent blocks, each with a ring of tokens in shared memory.  The producer warp works out a token's table
// (two entries a lane) and asks for its rows by bulk copies several tokens ahead, eight warps finish the rows of one
// token after the other.  Weights stay in registers.
constexpr int kStreamWarps = 8;
constexpr int kStreamThreads = (kStreamWarps + 1) * 32;
constexpr int kStreamBlocks = 3;                  // per SM
constexpr int kStreamSmem = 72 * 1024;            // ring of a block
constexpr int kStreamMaxStages = 6;
constexpr int kStreamToken = 8 * 1024;            // bytes

struct StreamMeta {
    int seq, row;      // the token's sequence and row in its units
};

template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kStreamThreads, kStreamBlocks) append_rotary_stream(const __grid_constant__ RotaryKernelArgs a, int stages, int stage_bytes) {
    constexpr int LPR = D / 8;
    constexpr int ROWS = kStreamWarps * 32 / LPR;
    constexpr int RB = D * (int)sizeof(T);
    constexpr int QB = 4 * (int)sizeof(T);
    extern __shared__ __align__(128) unsigned char ring[];      // stages x [head rows][cos][sin]
    __shared__ uint64_t full[kStreamMaxStages], empty[kStreamMaxStages];
    __shared__ StreamMeta meta[kStreamMaxStages];
    __shared__ volatile int abort_flag[2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int heads = a.Hq + 2 * a.Hkv;
    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&full[i], 2);      // the copies, the table
            mbar_init(&empty[i], kStreamWarps);
        }
        abort_flag[0] = abort_flag[1] = 0;
        fence_mbar_init();
    }
    __syncthreads();
    pdl_wait();
    if (warp == kStreamWarps) {
        const int extra = a.n_extra ? *a.n_extra : 0;
        const uint32_t q_bytes = (uint32_t)a.Hq * RB, kv_bytes = (uint32_t)a.Hkv * RB;
        int it = 0;
        bool ok = true;
        // (nothing is rotated: there may be no positions)
        const bool turned = a.half > 0;
        int position = turned && blockIdx.x < a.tokens ? a.positions[blockIdx.x] : 0;
        for (int tok = blockIdx.x; tok < a.tokens; tok += gridDim.x, ++it) {
            const int st = it % stages;
            if (it >= stages) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&empty[st], (uint32_t)(it / stages - 1) & 1u, abort_flag, a.status)) != 0;
            if (!ok) break;
            unsigned char* base = ring + st * stage_bytes;
            if (lane == 0) {
                mbar_arrive_expect_tx(&full[st], q_bytes + 2 * kv_bytes);
                bulk_g2s(base, a.q + tok * a.q_stride, q_bytes, &full[st]);
                if (a.Hkv > 0) {
                    bulk_g2s(base + q_bytes, a.k + tok * a.k_stride, kv_bytes, &full[st]);
                    bulk_g2s(base + q_bytes + kv_bytes, a.v + tok * a.v_stride, kv_bytes, &full[st]);
                }
                const int b = tok / a.n_new;
                meta[st].seq = b;
                meta[st].row = tok - b * a.n_new + (a.unit_len ? 0 : a.len0 + extra);
            }
            // the next token's position is on its way while this one's table is worked out
            const int now = position, next = tok + (int)gridDim.x;
            if (turned && next < a.tokens) position = a.positions[next];
            float* cos_t = reinterpret_cast<float*>(base + heads * RB);
            for (int i = lane; i < a.half; i += 32) table_entry(now, a.turns[i], &cos_t[i], &cos_t[D / 2 + i]);
            __syncwarp();
            // (releases the table and the token's place to the other warps)
            if (lane == 0) mbar_arrive(&full[st]);
        }
        if ((!ok || abort_flag[0] != 0) && lane == 0) {
            // gave up: the copies already issued end (bounded) before the block gives its memory back
            for (int j = max(0, it - stages); j < it; ++j)
                mbar_wait_bounded(&full[j % stages], (uint32_t)(j / stages) & 1u, abort_flag + 1, a.status);
        }
        return;
    }
    const int lig = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const Lane<LPR, INTERLEAVED> ln(lig, a.half);
    float wq[8], wk[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
    if (a.q_weight != nullptr) {
        reinterpret_cast<const Quad<T>*>(a.q_weight)[ln.c0].unpack(wq);
        reinterpret_cast<const Quad<T>*>(a.q_weight)[ln.c1].unpack(wq + 4);
    }
    if (a.k_weight != nullptr) {
        reinterpret_cast<const Quad<T>*>(a.k_weight)[ln.c0].unpack(wk);
        reinterpret_cast<const Quad<T>*>(a.k_weight)[ln.c1].unpack(wk + 4);
    }
    int it = 0;
    for (int tok = blockIdx.x; tok < a.tokens; tok += gridDim.x, ++it) {
        const int st = it % stages;
        if (!mbar_wait_bounded(&full[st], (uint32_t)(it / stages) & 1u, abort_flag, a.status)) return;
        const unsigned char* base = ring + st * stage_bytes;
        const float* cos_t = reinterpret_cast<const float*>(base + heads * RB);
        const int seq = meta[st].seq, row = meta[st].row;
        for (int r = slot; r < heads; r += ROWS) {
            const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv;
            Quad<T> q0 = *reinterpret_cast<const Quad<T>*>(base + r * RB + ln.c0 * QB);
            Quad<T> q1 = *reinterpret_cast<const Quad<T>*>(base + r * RB + ln.c1 * QB);
            if (!is_v) {
                float x[8];
                q0.unpack(x);
                q1.unpack(x + 4);
                if (is_q) finish_row<LPR, D, INTERLEAVED>(x, a.q_weight != nullptr, wq, a.eps, ln, cos_t, cos_t + D / 2);
                else finish_row<LPR, D, INTERLEAVED>(x, a.k_weight != nullptr, wk, a.eps, ln, cos_t, cos_t + D / 2);
                q0.pack(x);
                q1.pack(x + 4);
            }
            char* dst = target<RB>(a, tok, r, is_q ? r : (is_v ? r - a.Hq - a.Hkv : r - a.Hq), is_q, is_v, seq, row, lig == 0);
            if (dst == nullptr) continue;
            *reinterpret_cast<Quad<T>*>(dst + ln.c0 * QB) = q0;
            *reinterpret_cast<Quad<T>*>(dst + ln.c1 * QB) = q1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[st]);
    }
}

template <typename T, int D, bool INTERLEAVED>
cudaError_t launch_one(const RotaryKernelArgs& ka, int sm_count, bool pdl, cudaStream_t stream) {
    const int heads = ka.Hq + 2 * ka.Hkv, stage = heads * D * (int)sizeof(T) + D * (int)sizeof(float);
    const int stages = std::min(kStreamMaxStages, kStreamSmem / stage);
    // The ring needs several tokens a block, room for two of them, and enough rows in a token for its eight warps: their
    // waits on it are once a token.  Measured as us through the ring / a block per token and pass: tokens of 12 KB,
    // 1024 7.9 / 8.7, 16384 73 / 115; of 30 KB, 256 7.0 / 6.5, 1024 12.9 / 18.8, 16384 190 / 291; of 2.5 KB, 16384 42 / 28;
    // of 4 KB, 16384 44 / 42.
    if (stages >= 2 && stage >= kStreamToken && ka.tokens >= 2 * kStreamBlocks * sm_count)
        return launch_kernel(append_rotary_stream<T, D, INTERLEAVED>, dim3(kStreamBlocks * sm_count), dim3(kStreamThreads), (size_t)stages * stage,
                             stream, pdl, ka, stages, stage);
    const int lpr = D / 8, threads = std::min(kRotThreads, (heads * lpr + 31) / 32 * 32), rows = threads / lpr;
    return launch_kernel(append_rotary_kernel<T, D, INTERLEAVED>, dim3((unsigned)ka.tokens, (unsigned)((heads + rows - 1) / rows)), dim3(threads), 0,
                         stream, pdl, ka);
}

template <typename T, int D>
cudaError_t launch_either(const RotaryKernelArgs& ka, bool interleaved, int sm_count, bool pdl, cudaStream_t stream) {
    return interleaved ? launch_one<T, D, true>(ka, sm_count, pdl, stream) : launch_one<T, D, false>(ka, sm_count, pdl, stream);
}

template <typename T, int D>
cudaError_t stream_attr() {
    const cudaError_t e = cudaFuncSetAttribute(append_rotary_stream<T, D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(append_rotary_stream<T, D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
}

}  // namespace

cudaError_t init_rotary_kernels() {
    cudaError_t e;
    if ((e = stream_attr<__nv_bfloat16, 128>()) != cudaSuccess || (e = stream_attr<__nv_bfloat16, 64>()) != cudaSuccess ||
        (e = stream_attr<float, 128>()) != cudaSuccess)
        return e;
    return stream_attr<float, 64>();
}

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
        return r.D == 128 ? launch_either<__nv_bfloat16, 128>(ka, r.interleaved, r.sm_count, r.programmatic, stream)
                          : launch_either<__nv_bfloat16, 64>(ka, r.interleaved, r.sm_count, r.programmatic, stream);
    return r.D == 128 ? launch_either<float, 128>(ka, r.interleaved, r.sm_count, r.programmatic, stream)
                      : launch_either<float, 64>(ka, r.interleaved, r.sm_count, r.programmatic, stream);
}

}  // namespace kvs
