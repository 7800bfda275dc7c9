// Beam search around the cache: the best continuations of every request's beams, and the sequences of every slot taking the
// rows of the beams they continue.
#include <algorithm>

#include "kvs_device.cuh"
#include "kvs_kernels.h"

namespace kvs {

namespace {

// --------------------------------------------------------------------------------------
// Selection.  score(b, v) = scores[b] + x_bv - lse_b,  lse_b = log sum_v exp x_bv;  of a request's W beams x V tokens the K
// best, equal scores by the lowest beam, within it the higher logit, then the lower token.
//
// First kernel: every logits row is cut into segments, a block each: running maximum and sum of exponentials per thread, then
// the segment's K best by a threshold: the K-th largest of the threads' own maxima.  K elements at least reach it and hardly
// more do, and only the logits of threads whose maximum does are read again (from L2, a warp for a thread's pieces).  Where
// too many reach it (equal logits, sorted ones) the candidates become 64-bit keys - order of the value, then the lower index, all different - and the
// threads' best of those bound them, a run of logits at a time: exactly K threads reach the K-th largest.
// Second kernel, a block per request: the segments' sums merged and scores formed in fp64 (the order within a beam is then the
// logits', rows with equal bits tie exactly, and no rounding of a score near -20, 1e-6, decides between beams), the lists'
// entries by the same kind of threshold, and the K best in order.  The sums themselves are of fp32 exponentials (ex2.approx, 2^-22)
// added in fp32 within a segment: lse was off by 2.3e-7 at most over random rows of 1000 to 1000003 logits, and beams whose scores
// are closer than that may come in either order.
// Bound: HBM for the logits, once; small calls: two launches.
// --------------------------------------------------------------------------------------
constexpr int kBeamThreads = 256;
constexpr int kBeamAhead = 4;                             // 16-byte pieces of logits a thread has in flight
constexpr int kBeamRoom = 2048;                           // candidates a block has room for
constexpr int kBeamRun = 8;                               // logits of a thread at a time where there are too many
// Up to so many continuations the threshold is taken from the maxima of four threads each, a quarter of the numbers to rank; with
// more it falls so low that too many logits reach it (16 x 8 beams x 131071 bf16, 4 / 16 / 24 / 32 continuations: 16.4 / 20.3 /
// 22.5 / 28.0 us by fours, 22.0 / 24.8 / 26.4 / 28.9 by threads; 4 beams x 32000 fp32: 6.7 / 10.7 / 13.4 / 36.2 and 9.0 / 12.4 /
// 14.9 / 18.4).
constexpr int kBeamQuads = 24;
static_assert(kBeamQuads <= kBeamThreads / 4 && kBeamMaxOut <= kBeamThreads, "at least as many maxima as continuations");
static_assert(kBeamMaxOut * (kBeamRun + 1) * 2 <= kBeamRoom, "what is kept, and what a run adds");

__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);          // -0 and 0 are equal
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ uint64_t order_of(double x) {
    const uint64_t u = __double_as_longlong(x + 0.0);
    return u ^ (u >> 63 ? 0xffffffffffffffffull : 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(uint64_t o) { return __longlong_as_double(o ^ (o >> 63 ? 0x8000000000000000ull : 0xffffffffffffffffull)); }

// exp(t), t <= 0 (or NaN)
__device__ __forceinline__ float exp_below(float t) { return fast_exp2(t * 1.44269504f); }

// The second kernel's keys need more bits than one word.  By score, then by the lower beam, the higher logit and the lower
// token: within a beam that is the order by which the segments' lists are cut, also where fp64 scores are equal and logits are not.
struct Wide {
    uint64_t v;      // order of the fp64 score
    uint64_t t;      // from the top: beams after this one, order of the logit (32 bits), tokens after this one (token_bits)
};
__device__ __forceinline__ bool above(uint64_t a, uint64_t b) { return a > b; }
__device__ __forceinline__ bool above(const Wide& a, const Wide& b) { return a.v > b.v || (a.v == b.v && a.t > b.t); }

// The K-th largest of `n` numbers s_x[0 .. n-1] (n a multiple of four, at least K), of which thread t < n holds `mine`, as
// order_of: into *cut, which is to hold the highest order before.  Ends with a barrier.
__device__ __forceinline__ void kth_of(const float* s_x, int n, float mine, int K, uint32_t* cut) {
    if ((int)threadIdx.x < n) {
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; j += 4) {
            const float4 x = *reinterpret_cast<const float4*>(s_x + j);
            rank += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
        }
        if (rank < K) atomicMin(cut, order_of(mine));
    }
    __syncthreads();
}

// The K-th largest of all threads' keys into *cut, for every thread (keys that differ, except `lowest`, which nothing is
// below).  `keys`: a shared array of a key per thread.
template <typename Key>
__device__ __noinline__ void kth_of_threads(Key mine, int K, Key lowest, Key* keys, Key* cut) {
    keys[threadIdx.x] = mine;
    __syncthreads();
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < kBeamThreads; ++j) rank += above(keys[j], mine) ? 1 : 0;
    if (rank == K - 1 || (rank < K - 1 && !above(mine, lowest))) *cut = mine;        // (several lowest keys: the same value)
    __syncthreads();
}

// Keeps of the `n` keys in `list` (at most kBeamRoom) those that reach the K-th largest of the threads' best: at most
// K * kBeamRoom / 256, the K best among them.  *count receives how many; returns the threshold.
template <typename Key>
__device__ __noinline__ Key prune(Key* list, int n, int* count, int K, Key lowest, Key* keys, Key* cut) {
    constexpr int MOST = (kBeamRoom + kBeamThreads - 1) / kBeamThreads;
    Key mine[MOST], top = lowest;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
        const int at = threadIdx.x + j * kBeamThreads;
        mine[j] = at < n ? list[at] : lowest;
        if (above(mine[j], top)) top = mine[j];
    }
    kth_of_threads(top, K, lowest, keys, cut);
    const Key c = *cut;
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MOST; ++j)
        if (above(mine[j], lowest) && !above(c, mine[j])) list[atomicAdd(count, 1)] = mine[j];
    __syncthreads();
    return c;
}

// Of the *count keys in `list` the K best, in order, to put(rank, key).
template <typename Key, typename Put>
__device__ __forceinline__ void best_in_order(Key* list, int* count, int K, Key lowest, Key* keys, Key* cut, Put put) {
    int n = *count;
    while (n > kBeamThreads) {
        prune(list, n, count, K, lowest, keys, cut);
        n = *count;
        __syncthreads();
    }
    if ((int)threadIdx.x < n) {
        const Key mine = list[threadIdx.x];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += above(list[j], mine) ? 1 : 0;
        if (rank < K) put(rank, mine);
    }
}

struct BeamKernelArgs {
    const void* logits;
    long long stride;        // elements between rows
    int vocab, rows, segs, seg_len;
    bool vec;                // rows start on 16 bytes
    const float* scores;
    int W, K;
    int token_bits;          // of vocab - 1; with a beam's they are 32 at most (beams * vocab is below 2^31)
    float* out_scores;
    int* out_tokens;
    int* out_parents;
    uint64_t* lists;         // [rows][segs][K] keys, best first, 0 where there are fewer
    float2* sums;            // [rows][segs] maximum, sum of exponentials below it
    int* status;
    long long list_count, sum_count;
};

// 16 bytes of logits that are all minus infinity, and 16 bytes that lie anywhere
template <typename T>
__device__ __forceinline__ uint4 masked_piece() {
    constexpr uint32_t w = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    return make_uint4(w, w, w, w);
}
__device__ __forceinline__ uint4 gather_piece(const __nv_bfloat16* p) {
    auto bits = [&](int i) { return (uint32_t)__bfloat16_as_ushort(p[i]); };
    return make_uint4(bits(0) | bits(1) << 16, bits(2) | bits(3) << 16, bits(4) | bits(5) << 16, bits(6) | bits(7) << 16);
}
__device__ __forceinline__ uint4 gather_piece(const float* p) {
    return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
}

template <typename T>
__global__ void __launch_bounds__(kBeamThreads, 5) beam_segments_kernel(const BeamKernelArgs a) {
    __shared__ uint64_t s_list[kBeamRoom];
    __shared__ uint64_t s_keys[kBeamThreads];
    __shared__ __align__(16) float s_max[kBeamThreads];
    __shared__ uint64_t s_kth;
    __shared__ uint32_t s_cut;
    __shared__ int s_count, s_found, s_who[kBeamThreads];
    __shared__ float2 s_sum[kBeamThreads / 32];
    const int seg = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
    if (tid == 0) {
        s_count = s_found = 0;
        s_cut = 0xffffffffu;
    }
    pdl_launch_dependents();
    pdl_wait();
    const int v0 = seg * a.seg_len, len = min(a.seg_len, a.vocab - v0);      // (v0 + seg_len may pass 31 bits)
    const T* x_row = static_cast<const T*>(a.logits) + row * a.stride;
    const uint64_t none = (uint64_t)order_of(-INFINITY) << 32 | 0xffffffffu;     // minus infinity is no candidate
    constexpr int PER16 = 16 / (int)sizeof(T);       // logits per piece
    constexpr int AHEAD = kBeamAhead, TURN = AHEAD * kBeamThreads;
    auto key = [&](float x, int v) { return (uint64_t)order_of(x) << 32 | (uint32_t)~v; };
    // thread t takes pieces t, t + 256, ...: the same logits whether they can be loaded as vectors or not; what is left of the
    // row behind the last whole piece goes to the first threads, a logit each
    const int pieces = len / PER16, rest = len - pieces * PER16, at_rest = v0 + pieces * PER16 + min(tid, rest);
    const float extra = tid < rest ? (float)x_row[at_rest] : -INFINITY;
    auto piece = [&](int p) {
        if (p >= pieces) return masked_piece<T>();
        const T* at = x_row + v0 + p * PER16;
        return a.vec ? *reinterpret_cast<const uint4*>(at) : gather_piece(at);
    };
    float m = extra, sum = extra > -INFINITY ? 1.f : extra != extra ? extra : 0.f;
    for (int p0 = tid; p0 < pieces; p0 += TURN) {
        uint4 x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) x[j] = piece(p0 + j * kBeamThreads);
        float top = m;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float f[PER16];
            Unpack<T>::run(x[j], f);
#pragma unroll
            for (int i = 0; i < PER16; ++i) top = fmaxf(top, f[i]);
        }
        // exp(x - top), two at a time (a product's rounding costs 2^-24 |x - top| of it: next to nothing where a term counts)
        const float ref = top == -INFINITY ? 0.f : top;
        const uint64_t minus = pair_of(-ref, -ref), scale = pair_of(1.44269504f, 1.44269504f);
        uint64_t sums[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float f[PER16];
            Unpack<T>::run(x[j], f);
#pragma unroll
            for (int i = 0; i < PER16; i += 2) {
                const uint64_t y = mul2(add2(pair_of(f[i], f[i + 1]), minus), scale);
                sums[i / 2 % 2] = add2(sums[i / 2 % 2], pair_of(fast_exp2(low_of(y)), fast_exp2(high_of(y))));
            }
        }
        const uint64_t both = add2(sums[0], sums[1]);
        sum = sum * exp_below(m - ref) + (low_of(both) + high_of(both));    // a NaN among the logits makes it, and the row's sum, NaN
        m = top;
    }
    // the threshold; for few continuations the maxima of four threads each are enough of them
    const bool quads = a.K <= kBeamQuads;
    float most = m;
    if (quads) {
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    }
    if (!quads || tid % 4 == 0) s_max[quads ? tid / 4 : tid] = most;
    __syncthreads();
    kth_of(s_max, quads ? kBeamThreads / 4 : kBeamThreads, s_max[quads ? tid % (kBeamThreads / 4) : tid], a.K, &s_cut);
    const float cut = value_of(s_cut);
    auto offer = [&](float x, int v) {
        if (x >= cut && x > -INFINITY) {
            const int at = atomicAdd(&s_count, 1);
            if (at < kBeamRoom) s_list[at] = key(x, v);
        }
    };
    if (m >= cut && m > -INFINITY) {
        s_who[atomicAdd(&s_found, 1)] = tid;
        offer(extra, at_rest);
    }
    __syncthreads();
    const int found = s_found;
    for (int i = tid / 32; i < found; i += kBeamThreads / 32)
        for (int p = s_who[i] + tid % 32 * kBeamThreads; p < pieces; p += 32 * kBeamThreads) {
            float f[PER16];
            Unpack<T>::run(piece(p), f);
            float high = f[0];
#pragma unroll
            for (int j = 1; j < PER16; ++j) high = fmaxf(high, f[j]);
            if (high >= cut)
#pragma unroll
                for (int j = 0; j < PER16; ++j) offer(f[j], v0 + p * PER16 + j);
        }
    __syncthreads();
    if (s_count > kBeamRoom) {
        // too many: with keys, a few logits of a thread and the extra one at a time
        __syncthreads();
        if (tid == 0) s_count = 0;
        int held = 0;
        constexpr int RUN = kBeamRun / PER16;
#pragma unroll 1
        for (int p0 = 0; p0 < max(pieces, 1); p0 += RUN * kBeamThreads) {
            uint64_t k[kBeamRun + 1];
            k[kBeamRun] = p0 == 0 ? key(extra, at_rest) : none;
#pragma unroll
            for (int j = 0; j < RUN; ++j) {
                float f[PER16];
                const int p = p0 + j * kBeamThreads + tid;
                Unpack<T>::run(piece(p), f);
#pragma unroll
                for (int i = 0; i < PER16; ++i) k[j * PER16 + i] = key(f[i], v0 + p * PER16 + i);
            }
            uint64_t first = none;
#pragma unroll
            for (int i = 0; i <= kBeamRun; ++i) first = max(first, k[i]);
            kth_of_threads(first, a.K, none, s_keys, &s_kth);
            uint64_t least = s_kth;
            __syncthreads();
            if (held > kBeamRoom / 2) least = max(least, prune(s_list, held, &s_count, a.K, none, s_keys, &s_kth));
#pragma unroll
            for (int i = 0; i <= kBeamRun; ++i)
                if (k[i] >= least && k[i] > none) s_list[atomicAdd(&s_count, 1)] = k[i];
            __syncthreads();
            held = s_count;
            __syncthreads();
        }
    }
    // the segment's maximum and sum, in a fixed order
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, d), sum2 = __shfl_xor_sync(0xffffffffu, sum, d);
        const float top = fmaxf(m, m2), ref2 = top == -INFINITY ? 0.f : top;
        const float lo = m <= m2 ? sum * exp_below(m - ref2) : sum2 * exp_below(m2 - ref2), hi = m <= m2 ? sum2 : sum;
        sum = m == m2 ? sum + sum2 : hi + lo;
        m = top;
    }
    if ((tid & 31) == 0) s_sum[tid >> 5] = make_float2(m, sum);
    __syncthreads();
    const long long at = (long long)row * a.segs + seg;
    if (tid == 0 && KVS_BOUNDS_OK(at, 1, a.sum_count, a.status)) {
        float top = -INFINITY, total = 0.f;
        for (int w = 0; w < kBeamThreads / 32; ++w) top = fmaxf(top, s_sum[w].x);
        for (int w = 0; w < kBeamThreads / 32; ++w) total += s_sum[w].x == top ? s_sum[w].y : s_sum[w].y * exp_below(s_sum[w].x - top);
        a.sums[at] = make_float2(top, total);
    }
    uint64_t* out = a.lists + at * a.K;
    const bool room = KVS_BOUNDS_OK(at * a.K, a.K, a.list_count, a.status);
    best_in_order(s_list, &s_count, a.K, none, s_keys, &s_kth, [&](int rank, uint64_t k) {
        if (room) out[rank] = k;
    });
    if (room && tid < a.K && tid >= s_count) out[tid] = 0;
}

// Blocks that start early settle where the first kernel's blocks leave room, several on an SM, and then wait for one another's
// fp64 arithmetic.  Shared memory that nothing uses keeps them apart as long as each can have an SM (16 requests x 8 beams x
// 131071 logits, 16 / 17 / 32 continuations: 21.9 / 29.4 / 34.4 us without, 20.3 / 24.8 / 28.7 with it; 148 requests x 4 x 32000
// 18.4 and 18.1); with more requests they have to share (200 x 1 x 32000: 11.9 and 14.3, 1024 x 2 x 2000: 19.0 and 32.5).
constexpr int kFinishApart = 80 * 1024;

__global__ void __launch_bounds__(kBeamThreads) beam_finish_kernel(const BeamKernelArgs a) {
    __shared__ Wide s_list[kBeamRoom];
    __shared__ Wide s_keys[kBeamThreads];
    __shared__ __align__(16) float s_head[kBeamThreads];
    __shared__ Wide s_kth;
    __shared__ double s_base[kBeamMaxBeams];      // scores[b] - log of the sum below the row's maximum
    __shared__ float s_top[kBeamMaxBeams];
    __shared__ uint32_t s_cut;
    __shared__ int s_count, s_equal[kBeamMaxOut];
    const int req = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row0 = (long long)req * a.W;
    const int lists = a.W * a.segs, entries = lists * a.K;
    if (tid == 0) {
        s_cut = 0xffffffffu;
        s_count = 0;
    }
    pdl_launch_dependents();
    pdl_wait();
    const uint64_t* list = a.lists + row0 * a.segs * a.K;
    constexpr int AHEAD = 4;                      // entries a thread has in flight
    uint64_t ahead[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) ahead[j] = tid + j * kBeamThreads < entries ? __ldcg(list + tid + j * kBeamThreads) : 0;
    for (int b = warp; b < a.W; b += kBeamThreads / 32) {
        const float2* sums = a.sums + (row0 + b) * a.segs;
        float top = -INFINITY;
        for (int i = lane; i < a.segs; i += 32) top = fmaxf(top, __ldcg(&sums[i].x));
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        double total = 0;
        for (int i = lane; i < a.segs; i += 32) {
            const float2 s = __ldcg(sums + i);
            total += (double)s.y * (s.x == top ? 1.0 : exp((double)s.x - (double)top));
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
        if (lane == 0) {
            const double base = (double)a.scores[row0 + b] - log(total);
            s_base[b] = isfinite(base) ? base : -(double)INFINITY;      // such a row has no candidates
            s_top[b] = top;
        }
    }
    __syncthreads();
    const Wide lowest = {order_of(-(double)INFINITY), 0ull};      // scores of minus infinity and NaN are no candidates
    // an entry's score (as an order), and its key once that is known
    auto score_of = [&](uint64_t k, int beam) {
        if (k == 0) return lowest.v;
        const double score = s_base[beam] + ((double)value_of((uint32_t)(k >> 32)) - (double)s_top[beam]);
        return score > -(double)INFINITY ? order_of(score) : lowest.v;
    };
    auto key_of = [&](uint64_t v, uint64_t k, int beam) {
        const uint32_t tokens_after = (uint32_t)a.vocab - 1 - ~(uint32_t)k;
        return Wide{v, (uint64_t)(a.W - 1 - beam) << (32 + a.token_bits) | (k >> 32) << a.token_bits | tokens_after};
    };
    // The threads' best entries, in fp32 (whose rounding keeps the order), or the best of four threads each: what is below the
    // K-th largest of those is not among the K best.
    const int per = a.segs * a.K;                 // entries of a beam
    float most = -INFINITY;
    uint64_t scores[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int e = tid + j * kBeamThreads;
        scores[j] = e < entries ? score_of(ahead[j], e / per) : lowest.v;
        most = fmaxf(most, (float)value_of(scores[j]));
    }
    for (int e = tid + AHEAD * kBeamThreads; e < entries; e += kBeamThreads)
        most = fmaxf(most, (float)value_of(score_of(__ldcg(list + e), e / per)));
    const bool quads = a.K <= kBeamQuads;
    if (quads) {
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    }
    if (!quads || tid % 4 == 0) s_head[quads ? tid / 4 : tid] = most;
    __syncthreads();
    kth_of(s_head, quads ? kBeamThreads / 4 : kBeamThreads, s_head[quads ? tid % (kBeamThreads / 4) : tid], a.K, &s_cut);
    const float cut = value_of(s_cut);
    auto reaches = [&](uint64_t v) { return v > lowest.v && (float)value_of(v) >= cut; };
    auto offer = [&](uint64_t v, uint64_t k, int e) {
        if (reaches(v)) {
            const int at = atomicAdd(&s_count, 1);
            if (at < kBeamRoom) s_list[at] = key_of(v, k, e / per);
        }
    };
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) offer(scores[j], ahead[j], tid + j * kBeamThreads);
    for (int e = tid + AHEAD * kBeamThreads; e < entries; e += kBeamThreads) {
        const uint64_t k = __ldcg(list + e);
        offer(score_of(k, e / per), k, e);
    }
    __syncthreads();
    if (s_count > kBeamRoom) {
        // more than there is room for (many equal scores): a row of entries of all threads at a time, keeping the best so far
        __syncthreads();
        if (tid == 0) s_count = 0;
        __syncthreads();
        int held = 0;
        Wide least = lowest;
        for (int e0 = 0; e0 < entries; e0 += kBeamThreads) {
            const int e = e0 + tid;
            const uint64_t k = e < entries ? __ldcg(list + e) : 0;
            Wide w = lowest;
            if (k) w = key_of(score_of(k, e / per), k, e / per);
            const bool in = reaches(w.v) && !above(least, w);
            if (in) s_list[atomicAdd(&s_count, 1)] = w;
            held += __syncthreads_count(in);
            if (held > kBeamRoom - kBeamThreads) {
                least = prune(s_list, held, &s_count, a.K, lowest, s_keys, &s_kth);
                held = s_count;
                __syncthreads();
            }
        }
    }
    // in order: by the fp32 scores, in which a hundred candidates compare quickly, equal ones by their keys
    const long long o = (long long)req * a.K;
    int n = s_count;
    while (n > kBeamThreads) {
        __syncthreads();
        prune(s_list, n, &s_count, a.K, lowest, s_keys, &s_kth);
        n = s_count;
    }
    Wide w = lowest;
    if (tid < n) w = s_list[tid];
    s_head[tid] = tid < n ? (float)value_of(w.v) : -INFINITY;
    if (tid < a.K) s_equal[tid] = 0;
    __syncthreads();
    int rank = a.K;
    const float x = s_head[tid];
    if (tid < n) {
        rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; j += 4) {
            const float4 y = *reinterpret_cast<const float4*>(s_head + j);
            rank += (y.x > x) + (y.y > x) + (y.z > x) + (y.w > x);
        }
        if (rank < a.K) atomicAdd(&s_equal[rank], 1);
    }
    __syncthreads();
    if (rank < a.K) {
        if (s_equal[rank] > 1)
            for (int j = 0; j < n; ++j) rank += s_head[j] == x && above(s_list[j], w) ? 1 : 0;
        if (rank < a.K) {
            a.out_scores[o + rank] = x;
            a.out_tokens[o + rank] = a.vocab - 1 - (int)(w.t & ((1ull << a.token_bits) - 1));
            a.out_parents[o + rank] = (int)(row0 + a.W - 1 - (int)(w.t >> (32 + a.token_bits)));
        }
    }
    if (tid < a.K && tid >= s_count) {     // fewer candidates than places
        a.out_scores[o + tid] = -INFINITY;
        a.out_tokens[o + tid] = -1;
        a.out_parents[o + tid] = (int)row0;
    }
}

// --------------------------------------------------------------------------------------
// Reordering.  Sequence b of every plane takes rows first .. n-1 of sequence parent[b].  In place: a block takes one run of
// bytes of one head's rows, the same run of every sequence; it brings the runs of all sequences that another one takes
// into shared memory (bulk copies), waits, and sends them to their takers (bulk copies).  A source is read once however many
// take it, a sequence that stays as it is costs nothing.  Bound: HBM, bytes read and written once.
// --------------------------------------------------------------------------------------
constexpr int kReorderThreads = 128;
constexpr int kReorderBytes = 64 * 1024;       // shared memory for the runs; three blocks per SM

struct ReorderKernelArgs {
    char* pool;
    const int* parent;
    long long plane_bytes;
    int planes, Hkv, row_bytes, row_stride, first, cap, old_batch, new_batch;
    const int* n_extra;
    int* status;
    unsigned long long wait_ns;
};

__global__ void __launch_bounds__(kReorderThreads) reorder_kernel(const ReorderKernelArgs a, const ReorderRows rows) {
    extern __shared__ __align__(128) unsigned char run[];
    int* from = reinterpret_cast<int*>(run + kReorderBytes);       // [sources]: the sequences to read
    int* place = from + a.old_batch;                              // [old_batch]: where a sequence's run lies, or -1
    int* to = place + a.old_batch;                                // [takers]: sequence
    int* what = to + a.new_batch;                                 // [takers]: its source, then where that lies
    __shared__ uint64_t bar;
    __shared__ int s_sources, s_takers, s_abort, s_gave_up;
    const int tid = threadIdx.x;
    if (tid == 0) {
        mbar_init(&bar, 1);
        fence_mbar_init();
        s_sources = s_takers = s_abort = s_gave_up = 0;
    }
    for (int b = tid; b < a.old_batch; b += kReorderThreads) place[b] = -1;
    pdl_launch_dependents();
    pdl_wait();
    __syncthreads();
    // who takes from whom; a parent out of range leaves its sequence as it is
    for (int b = tid; b < a.new_batch; b += kReorderThreads) {
        const int p = a.parent[b];
        if (p < 0 || p >= a.old_batch) {
            if (blockIdx.x == 0) atomicExch(a.status, 1);
            continue;
        }
        if (p == b) continue;
        const int i = atomicAdd(&s_takers, 1);
        to[i] = b;
        what[i] = p;
        if (atomicExch(&place[p], -2) == -1) from[atomicAdd(&s_sources, 1)] = p;
    }
    __syncthreads();
    const int sources = s_sources, takers = s_takers;
    if (takers == 0) return;
    for (int i = tid; i < sources; i += kReorderThreads) place[from[i]] = i;
    __syncthreads();
    for (int i = tid; i < takers; i += kReorderThreads) what[i] = place[what[i]];      // (read again by the same thread)
    const int chunk = kReorderBytes / sources / 16 * 16;
    const int extra = a.n_extra ? *a.n_extra : 0;
    int longest = 0;
    for (int s = 0; s < a.planes / 2; ++s) longest = max(longest, min(rows.n[s] + extra, a.cap));
    const long long most = (long long)max(0, longest - a.first) * a.row_bytes;      // bytes of a unit's rows that move
    const long long chunks = (most + chunk - 1) / chunk, items = chunks * a.planes * a.Hkv;
    int turn = 0;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const long long head = it / chunks, c = it - head * chunks;
        const int plane = (int)(head / a.Hkv), h = (int)(head - (long long)plane * a.Hkv);
        const int n = min(rows.n[plane / 2] + extra, a.cap);
        const long long len = (long long)max(0, n - a.first) * a.row_bytes, at = c * chunk;
        if (at >= len) continue;            // a slot with fewer rows than others
        const uint32_t bytes = (uint32_t)min((long long)chunk, len - at);
        const long long off0 = ((long long)h * a.row_stride + a.first) * a.row_bytes + at;
        const long long seq = (long long)a.Hkv * a.row_stride * a.row_bytes;
        char* base = a.pool + plane * a.plane_bytes;
        // the previous item's runs have left shared memory before they are overwritten
        if (turn) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncthreads();
        if (tid == 0) mbar_arrive_expect_tx(&bar, bytes * (uint32_t)sources);
        __syncthreads();
        for (int i = tid; i < sources; i += kReorderThreads) {
            long long off = from[i] * seq + off0;
            if (!KVS_BOUNDS_OK(off, bytes, a.plane_bytes, a.status)) off = 0;
            bulk_g2s(run + (size_t)i * chunk, base + off, bytes, &bar);
        }
        const bool ok = mbar_wait_bounded(&bar, turn & 1, &s_abort, a.status, a.wait_ns);
        ++turn;
        if (__syncthreads_or(!ok)) {     // give up, with nothing of this item written, once the copies have landed
            mbar_wait_bounded(&bar, (turn + 1) & 1, &s_gave_up, a.status, a.wait_ns);
            break;
        }
        for (int i = tid; i < takers; i += kReorderThreads) {
            const long long off = to[i] * seq + off0;
            if (KVS_BOUNDS_OK(off, bytes, a.plane_bytes, a.status))
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(base + off),
                             "r"(smem_u32(run + (size_t)what[i] * chunk)), "r"(bytes)
                             : "memory");
        }
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

size_t reorder_smem(int old_batch, int new_batch) { return kReorderBytes + 2ull * (old_batch + new_batch) * sizeof(int); }

}  // namespace

cudaError_t init_beam_kernels() {
    const cudaError_t e = cudaFuncSetAttribute(beam_finish_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFinishApart);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(reorder_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)reorder_smem(kReorderMaxBatch, kReorderMaxBatch));
}

cudaError_t launch_beam_select(const BeamArgs& p, cudaStream_t stream) {
    BeamKernelArgs a;
    a.logits = p.logits;
    a.stride = p.stride;
    a.vocab = p.vocab;
    a.rows = p.requests * p.beams;
    // Segments: as many as make the blocks fill the SMs once, five on each, but none shorter than a piece per thread; at most 256
    // lists (a thread each in the second kernel) per request, and no more than there is room for.
    const int e = p.dtype == 0 ? 2 : 4, piece = kBeamThreads * (16 / e);
    const int most = std::min({(p.vocab - 1) / piece + 1, kBeamThreads / p.beams, std::max(1, kBeamMaxLists / a.rows)});
    a.segs = std::min(std::max(1, p.sm_count * 5 / a.rows), most);
    a.seg_len = ((p.vocab - 1) / a.segs + 1 + 15) / 16 * 16;
    a.segs = (p.vocab - 1) / a.seg_len + 1;
    a.vec = (uintptr_t)p.logits % 16 == 0 && p.stride * e % 16 == 0;
    a.scores = p.scores;
    a.W = p.beams;
    a.K = p.n_out;
    a.token_bits = 0;
    while ((long long)p.vocab > 1ll << a.token_bits) ++a.token_bits;
    a.out_scores = p.out_scores;
    a.out_tokens = p.out_tokens;
    a.out_parents = p.out_parents;
    a.lists = static_cast<uint64_t*>(p.scratch);
    a.list_count = beam_lists(a.rows) * kBeamMaxOut;
    a.sums = reinterpret_cast<float2*>(a.lists + a.list_count);
    a.sum_count = beam_lists(a.rows);
    a.status = p.status;
    const dim3 grid(a.segs, a.rows);
    const cudaError_t err = p.dtype == 0 ? launch_kernel(beam_segments_kernel<__nv_bfloat16>, grid, dim3(kBeamThreads), 0, stream, p.programmatic, a)
                                         : launch_kernel(beam_segments_kernel<float>, grid, dim3(kBeamThreads), 0, stream, p.programmatic, a);
    if (err != cudaSuccess) return err;
    return launch_kernel(beam_finish_kernel, dim3(p.requests), dim3(kBeamThreads), p.requests <= p.sm_count ? kFinishApart : 0, stream,
                         p.programmatic, a);
}

cudaError_t launch_reorder(const ReorderArgs& p, const ReorderRows& rows, cudaStream_t stream) {
    ReorderKernelArgs a;
    a.pool = static_cast<char*>(p.pool);
    a.parent = p.parent;
    a.plane_bytes = p.plane_bytes;
    a.planes = 2 * p.slots;
    a.Hkv = p.Hkv;
    a.row_bytes = p.row_bytes;
    a.row_stride = p.row_stride;
    a.first = p.first;
    a.cap = p.capacity;
    a.old_batch = p.old_batch;
    a.new_batch = p.new_batch;
    a.n_extra = p.n_extra;
    a.status = p.status;
    a.wait_ns = p.wait_ns;
    // no more blocks than there can be items: every run at least a sixteen-byte piece per sequence
    long long bytes = 0;
    for (int s = 0; s < p.slots; ++s) bytes = std::max(bytes, (long long)(p.n_extra ? p.capacity : rows.n[s]) * p.row_bytes);
    const long long smallest = std::max(16, kReorderBytes / std::min(p.old_batch, p.new_batch) / 16 * 16);
    const long long items = (bytes + smallest - 1) / smallest * a.planes * p.Hkv;
    const unsigned blocks = (unsigned)std::max(1ll, std::min<long long>(items, p.sm_count * 3));
    return launch_kernel(reorder_kernel, dim3(blocks), dim3(kReorderThreads), reorder_smem(p.old_batch, p.new_batch), stream, p.programmatic, a, rows);
}

}  // namespace kvs
