// Host side of the C ABI declared in include/kvs.h: the layer -> slot indirection
// table, slot lengths, capacity and state checks, byte accounting, and the launches.
#include "../../include/kvs.h"

#include "kvs_kernels.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include <new>
#include <vector>

namespace {

constexpr size_t kAlign = 256;
constexpr int kRowStrideQuantum = 128;
constexpr size_t kScoreBytes = 64u << 20;     // scores of one pass of kvs_decode_attention_weights
constexpr size_t kPlainRowBytes = 64u << 20;  // 4-bit cache: rows in the storage type of one pass of the calls that need them so
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace

// ---------------------------------------------------------------------------------------
// Scratch of kvs_decode_attention_static: attention without any caller- or library-allocated
// scratch memory.
//
// The split-K partial results and the device status word of that one entry point live in a
// fixed array that is part of the loaded library image.  Every GPU that loads the library
// carries these kStaticScratchBytes until the process exits, and every call, from every
// context, uses the same bytes.
// ---------------------------------------------------------------------------------------
constexpr size_t kStaticScratchBytes = 2u << 20;  // 2 MiB
constexpr size_t kStaticStatusBytes = 256;        // first 256 bytes: device status word
// then the per-unit hand-over flags, at a fixed place and of a fixed size, so that no call's partial results
// (which follow) ever lie where another call, of another size, keeps its flags: they are zero when the library
// is loaded and every launch leaves them zero
constexpr size_t kStaticFlagBytes = 32768;        // 8192 (sequence, kv-head) units
static __device__ __align__(256) unsigned char g_static_scratch[kStaticScratchBytes];

namespace {

// In host code `g_static_scratch` is only a handle for the symbol, not an address the GPU can
// use, so the device address is looked up once per device, with that device current, as part of
// the per-device set-up that kvs_bind_memory runs (see init_device_once).  The look-up is also
// what makes the driver load this file's module and reserve the array on that GPU, so it happens
// where allocating is still allowed and no stream is being captured; the entry point itself then
// only reads the cached address.
cudaError_t g_static_err[64];
unsigned char* g_static_ptr[64];

cudaError_t resolve_static_scratch(int device) {
    void* p = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&p, g_static_scratch);
    g_static_err[device] = e;
    g_static_ptr[device] = e == cudaSuccess ? static_cast<unsigned char*>(p) : nullptr;
    return e;
}

}  // namespace

struct kvs_ctx {
    kvs_config cfg;
    int G = 1;
    int elem = 2;
    int format = KVS_CACHE_PLAIN;
    int row_bytes = 0;         // of a cached row
    int row_stride = 0;        // rows between units of a plane
    size_t plane_bytes = 0;
    float scale = 0.f;

    std::vector<int32_t> share_map, root, slot_of_layer;
    int n_slots = 0;
    std::vector<int32_t> slot_len;
    int cur_batch = 0;         // batch the cached rows were appended for (0 = none yet)

    // Ragged slots: after kvs_evict the units of a slot differ in length; the lengths then live in
    // a device array (one per slot, in the workspace) with a host mirror.
    std::vector<char> ragged;                       // per slot
    std::vector<std::vector<int32_t>> unit_len_host;  // per slot, [max_batch * Hkv]

    bool bound = false;
    char* pool = nullptr;
    char* ws = nullptr;
    int sm_count = 148;
    long long l2_bytes = 64ll << 20;

    // workspace carve-up (byte offsets)
    size_t off_status = 0, off_part_o = 0, off_part_ml = 0, off_stage_q = 0, off_stage_k = 0, off_stage_v = 0,
           off_stage_out = 0, off_unit_len = 0, off_counts = 0, off_search = 0, off_replay = 0, off_flags = 0, off_scores = 0,
           off_tree_o = 0, off_tree_ml = 0, ws_bytes = 0, search_bytes = 0,
           score_bytes = 0, off_plain = 0, plain_bytes = 0;

    alignas(64) unsigned char tensor_map[128];  // TMA view of the pool (bf16 storage only), 64-row boxes
    alignas(64) unsigned char tensor_map_tail[128];   // the same view with 16-row boxes (partly filled tiles)
    bool have_tensor_map = false;
    alignas(64) unsigned char plain_map[128];         // 4-bit cache: the scratch of storage-type rows

    // Launch bookkeeping for early-start (programmatic) launches.  Every kernel of this context
    // gets a sequence number.  A split-K kernel lets its successor start only after its own
    // wait, so when any later kernel runs, everything before the latest split-K kernel is
    // complete; appends newer than that may still be in flight.
    uint64_t seq = 0;
    uint64_t last_splitk_seq = 0;
    std::vector<uint64_t> app_seq_latest, app_seq_prev;   // per slot, 0 = none
    std::vector<int32_t> app_start_latest;                // first row the latest append wrote

    // kvs_step_host: second stream and events that overlap the host copies with the layers
    static constexpr int kChunks = 8;
    bool copy_ready = false;
    cudaStream_t copy_stream = nullptr, out_stream = nullptr;
    cudaEvent_t ev_in[kChunks] = {}, ev_done[kChunks] = {}, ev_start = nullptr;
    // kvs_layer_distances: a second stream on which the pair sums of one slab run beside the averaging of the next

    int opt_max_ctas = 0;
    int opt_kernel = 0;
    int opt_pdl = 1;
    int opt_host_chunks = 4;
    // tracing build: where the next attention launch stamps its timeline (kvs_trace_begin / kvs_trace_end)
    unsigned long long* trace_buf = nullptr;
    int trace_capacity = 0, trace_launch = 0;
    int opt_wait_us = 2000000;   // limit of the waits inside the split-K kernels, microseconds
    long long stall_tile = -1;   // kvs_selftest_stalled_copy: tile whose copies the next attention launch withholds
    int opt_finish = 1;   // units of at most two pieces are finished by the split-K kernel itself (no combine launch)
    int opt_replay = 0;   // launches carry the device-side growth counter (for CUDA-graph replay)
    // The split-K kernels read the growth counter before their wait.  That is safe because the
    // first launch after anything wrote the counter never starts early (full dependency): it and
    // everything after it then begin with the write complete.
    bool counter_written = false;
    kvs::DecodePlan last_plan{};
    kvs_stats_t stats{};
};

namespace {

void resolve_map(kvs_ctx* c) {
    const int L = c->cfg.n_layers;
    c->root.assign(L, 0);
    c->slot_of_layer.assign(L, -1);
    int n = 0;
    for (int l = 0; l < L; ++l) {
        if (c->share_map[l] == l) {
            c->root[l] = l;
            c->slot_of_layer[l] = n++;
        } else {
            // sources precede targets, so the source is already resolved
            c->root[l] = c->root[c->share_map[l]];
            c->slot_of_layer[l] = c->slot_of_layer[c->root[l]];
        }
    }
    c->n_slots = n;
    c->slot_len.assign(n, 0);
    c->cur_batch = 0;
    c->app_seq_latest.assign(n, 0);
    c->app_seq_prev.assign(n, 0);
    c->app_start_latest.assign(n, 0);
    c->ragged.assign(n, 0);
    c->unit_len_host.assign(n, std::vector<int32_t>());
}

// Whether the next launch may start early; consumes the "counter was just written" mark.
bool take_early_start(kvs_ctx* c) {
    const bool early = c->opt_pdl != 0 && !c->counter_written;
    c->counter_written = false;
    return early;
}

const int* replay_counter(const kvs_ctx* c) {
    return c->opt_replay ? reinterpret_cast<const int*>(c->ws + c->off_replay) : nullptr;
}

int* unit_len_dev(const kvs_ctx* c, int slot) {
    return reinterpret_cast<int*>(c->ws + c->off_unit_len) + (size_t)slot * c->cfg.max_batch * c->cfg.n_kv_heads;
}

// Rows of `slot` that no kernel possibly still in flight writes (see kvs_ctx::seq).
int safe_rows_of(const kvs_ctx* c, int slot) {
    const uint64_t complete_upto = c->last_splitk_seq ? c->last_splitk_seq - 1 : 0;
    if (c->app_seq_latest[slot] <= complete_upto) return c->slot_len[slot];
    if (c->app_seq_prev[slot] <= complete_upto) return c->app_start_latest[slot];
    return 0;
}

void layout_workspace(kvs_ctx* c) {
    const kvs_config& f = c->cfg;
    c->row_bytes = c->format == KVS_CACHE_4BIT ? kvs::pack4_row_bytes(f.head_dim) : f.head_dim * c->elem;
    c->plane_bytes = (size_t)f.max_batch * f.n_kv_heads * c->row_stride * c->row_bytes;
    const size_t units = (size_t)f.max_batch * f.n_kv_heads;
    const size_t pieces = units + kvs::kMaxCtas;
    size_t off = 0;
    c->off_status = off;
    off += kAlign;
    c->off_part_o = off;
    off = align_up(off + pieces * c->G * f.head_dim * sizeof(float), kAlign);
    c->off_part_ml = off;
    off = align_up(off + pieces * c->G * 2 * sizeof(float), kAlign);
    const size_t L = f.n_layers;
    c->off_stage_q = off;
    off = align_up(off + L * f.max_batch * f.n_q_heads * f.head_dim * c->elem, kAlign);
    c->off_stage_k = off;
    off = align_up(off + L * f.max_batch * f.n_kv_heads * f.head_dim * c->elem, kAlign);
    c->off_stage_v = off;
    off = align_up(off + L * f.max_batch * f.n_kv_heads * f.head_dim * c->elem, kAlign);
    c->off_stage_out = off;
    off = align_up(off + L * f.max_batch * f.n_q_heads * f.head_dim * sizeof(float), kAlign);
    c->off_unit_len = off;      // per slot (at most one per layer): int32 [max_batch * Hkv]
    off = align_up(off + L * units * sizeof(int32_t), kAlign);
    c->off_counts = off;        // staging for the kept-row counts of one kvs_evict call
    off = align_up(off + units * sizeof(int32_t), kAlign);
    c->off_replay = off;        // one int: rows every slot has grown by since a recorded launch
    off += kAlign;
    c->off_flags = off;         // one int per unit: "second piece written" (zero between launches)
    off = align_up(off + units * sizeof(int32_t), kAlign);
    c->off_search = off;        // per-block partial sums of the strategy-search reductions, and more (below)
    {
        // at most one slot per layer, at most max_seq rows: enough for every strategy and length
        const size_t need = std::max(kvs::distance_scratch_bytes(f.n_layers <= kvs::kMaxLayersSearch ? f.n_layers : 4,
                                                                 2LL * f.n_kv_heads * f.max_seq * f.head_dim),
                                     (size_t)kvs::kCosineMaxBlocks * 3 * sizeof(double));
        c->search_bytes = need;
        // The same bytes serve the other calls whose scratch lives no longer than the call (every kernel writes it
        // only after its wait for the previous one):
        // kvs_decode_attention_weights: one score per (unit, q-head of its group, row), for as many units at a time as
        // kScoreBytes hold, so that contexts of long and wide caches do not pay for a call they may never make
        const size_t unit_scores = (size_t)c->G * c->row_stride * sizeof(float);
        const size_t scores = std::min(units, std::max<size_t>(1, kScoreBytes / unit_scores)) * unit_scores;
        c->off_scores = off;
        c->score_bytes = scores;
        // kvs_tree_attention: two cut pieces per thread block at most
        const size_t tree_rows = (size_t)kvs::tree_piece_rows(c->G);
        const size_t tree_o = align_up(tree_rows * f.head_dim * sizeof(float), kAlign);
        c->off_tree_o = off;
        c->off_tree_ml = off + tree_o;
        // kvs_beam_select: the segments' lists and sums
        const size_t beam = kvs::beam_scratch_bytes(f.max_batch);
        // 4-bit cache: K and V rows in the storage type, of at least one sequence as long as the cache
        c->off_plain = off;
        c->plain_bytes = 0;
        if (c->format == KVS_CACHE_4BIT) {
            const size_t seq = 2ull * f.n_kv_heads * c->row_stride * f.head_dim * c->elem;
            c->plain_bytes = std::max(seq, std::min(f.max_batch * seq, kPlainRowBytes / kAlign * kAlign));
        }
        off = align_up(off + std::max({need, scores, tree_o + tree_rows * 2 * sizeof(float), beam, c->plain_bytes}), kAlign);
    }
    c->ws_bytes = off;
}

std::once_flag g_init_flag[64];
cudaError_t g_init_err[64];

cudaError_t init_device_once(int device) {
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    std::call_once(g_init_flag[device], [device]() {
        g_init_err[device] = kvs::init_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_mma_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_prefill_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_rotary_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_tree_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_weights_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_pack4_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = kvs::init_beam_kernels();
        if (g_init_err[device] == cudaSuccess) g_init_err[device] = resolve_static_scratch(device);
    });
    return g_init_err[device];
}

// RAII: make ctx's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
        target = dev;
    }
    ~DeviceGuard() {
        if (ok && prev != target) cudaSetDevice(prev);
    }
    int target = -1;
};

kvs_status check_append(kvs_ctx* c, int layer, const void* k, const void* v, int batch, int n_new, bool* sharing) {
    if (!c) return KVS_ERR_INVALID_ARG;
    if (!c->bound) return KVS_ERR_STATE;
    if (layer < 0 || layer >= c->cfg.n_layers) return KVS_ERR_INVALID_ARG;
    if (batch < 1 || batch > c->cfg.max_batch || n_new < 1) return KVS_ERR_INVALID_ARG;
    *sharing = c->share_map[layer] != layer;
    if (*sharing) return KVS_OK;
    if (!k || !v) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)k % 16) != 0 || ((uintptr_t)v % 16) != 0) return KVS_ERR_INVALID_ARG;   // 16-byte vector loads
    if (c->cur_batch != 0 && batch != c->cur_batch) return KVS_ERR_INVALID_ARG;
    const int slot = c->slot_of_layer[layer];
    if ((long long)c->slot_len[slot] + n_new > c->cfg.max_seq) return KVS_ERR_CAPACITY;
    return KVS_OK;
}

kvs_status check_attention(kvs_ctx* c, int layer, const void* q, const void* out, int batch) {
    if (!c) return KVS_ERR_INVALID_ARG;
    if (!c->bound) return KVS_ERR_STATE;
    if (layer < 0 || layer >= c->cfg.n_layers || !q || !out) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)q % 16) != 0 || ((uintptr_t)out % 4) != 0) return KVS_ERR_INVALID_ARG;   // q is fetched by bulk copies
    if (batch < 1 || batch > c->cfg.max_batch) return KVS_ERR_INVALID_ARG;
    const int slot = c->slot_of_layer[layer];
    if (c->slot_len[slot] == 0) return KVS_ERR_STATE;
    if (batch > c->cur_batch) return KVS_ERR_INVALID_ARG;
    return KVS_OK;
}

kvs_status appended(kvs_ctx* c, int slot, int batch, int n_new, cudaStream_t st);

// Stores rows of sequences seq0 .. seq0+batch-1 behind the ones a 4-bit slot holds; strides of k and v in elements.
cudaError_t store_packed(kvs_ctx* c, int slot, const void* k, const void* v, long long src_b, long long src_t, long long src_h,
                         int seq0, int batch, int n_new, cudaStream_t st) {
    const size_t skipped = (size_t)seq0 * c->cfg.n_kv_heads * c->row_stride * c->row_bytes;
    kvs::PackArgs p = {};
    p.k = k;
    p.v = v;
    p.src_b = src_b;
    p.src_t = src_t;
    p.src_h = src_h;
    p.kplane = c->pool + (size_t)(2 * slot) * c->plane_bytes + skipped;
    p.vplane = static_cast<char*>(p.kplane) + c->plane_bytes;
    p.batch = batch;
    p.n_new = n_new;
    p.Hkv = c->cfg.n_kv_heads;
    p.D = c->cfg.head_dim;
    p.dtype = c->cfg.dtype;
    p.row_stride = c->row_stride;
    p.len0 = c->slot_len[slot];
    p.capacity = c->cfg.max_seq;
    p.unit_len = c->ragged[slot] ? unit_len_dev(c, slot) + (size_t)seq0 * p.Hkv : nullptr;
    p.n_extra = replay_counter(c);
    p.status = reinterpret_cast<int*>(c->ws + c->off_status);
    p.plane_bytes = (long long)(c->plane_bytes - skipped);
    p.sm_count = c->sm_count;
    p.programmatic = take_early_start(c);
    return kvs::launch_pack4(p, st);
}

kvs_status do_append(kvs_ctx* c, int layer, const void* k, const void* v, int batch, int n_new, cudaStream_t st) {
    const int slot = c->slot_of_layer[layer];
    if (c->format == KVS_CACHE_4BIT) {
        const long long D = c->cfg.head_dim, token = c->cfg.n_kv_heads * D;
        if (store_packed(c, slot, k, v, n_new * token, token, D, 0, batch, n_new, st) != cudaSuccess) return KVS_ERR_CUDA;
        return appended(c, slot, batch, n_new, st);
    }
    char* kp = c->pool + (size_t)(2 * slot) * c->plane_bytes;
    char* vp = kp + c->plane_bytes;
    const bool rag = c->ragged[slot] != 0;
    if (kvs::launch_append(k, v, kp, vp, batch, n_new, c->cfg.n_kv_heads, c->row_bytes, c->row_stride,
                           c->slot_len[slot], rag ? unit_len_dev(c, slot) : nullptr, replay_counter(c), c->cfg.max_seq,
                           reinterpret_cast<int*>(c->ws + c->off_status), (long long)c->plane_bytes, take_early_start(c),
                           st) != cudaSuccess)
        return KVS_ERR_CUDA;
    return appended(c, slot, batch, n_new, st);
}

// Bookkeeping of a kernel just launched that stores n_new rows at the end of every unit of `slot`.
kvs_status appended(kvs_ctx* c, int slot, int batch, int n_new, cudaStream_t st) {
    if (c->ragged[slot]) {
        const int units = batch * c->cfg.n_kv_heads;
        if (kvs::launch_add_len(unit_len_dev(c, slot), n_new, units, c->opt_pdl != 0, st) != cudaSuccess)
            return KVS_ERR_CUDA;
        for (int u = 0; u < units; ++u) c->unit_len_host[slot][u] += n_new;
        c->seq += 1;
    }
    c->seq += 1;
    c->app_seq_prev[slot] = c->app_seq_latest[slot];
    c->app_seq_latest[slot] = c->seq;
    c->app_start_latest[slot] = c->slot_len[slot];
    c->slot_len[slot] += n_new;
    c->cur_batch = batch;
    c->stats.append_launches += 1;
    c->stats.kv_bytes_appended += 2ull * batch * c->cfg.n_kv_heads * n_new * c->row_bytes;
    return KVS_OK;
}

// Where one attention call keeps its split-K partial results and reports device-side trouble.
struct AttentionScratch {
    float* part_o;
    float* part_ml;
    int* flags;          // [units] ints, zero between launches
    int* status;
    bool programmatic;   // early-start launches (only when the call follows this context's own kernels)
    bool tracked;        // the call is part of the context's one ordered chain of launches (see kvs_ctx::seq)
};

// Which kernel serves the context's shape and how the call is cut into work.  bf16 groups of three
// or more q-heads per kv-head are a real (if thin) contraction and go to the tensor cores.
bool choose_plan(const kvs_ctx* c, int units, int n, kvs::DecodePlan* plan) {
    if (c->format == KVS_CACHE_4BIT) {
        if (c->cfg.dtype == KVS_BF16)
            kvs::plan_decode_pack4(units, n, c->sm_count, c->opt_max_ctas, plan);
        else
            kvs::plan_decode_pack4_f32(units, n, c->sm_count, c->opt_max_ctas, plan);
        return false;
    }
    const bool use_mma = c->have_tensor_map && (c->opt_kernel == 2 || (c->opt_kernel == 0 && c->G >= 3));
    if (use_mma)
        kvs::plan_decode_mma(units, n, c->cfg.head_dim, c->sm_count, c->opt_max_ctas, plan);
    else
        kvs::plan_decode_scalar(units, n, c->G, c->cfg.head_dim, c->cfg.dtype, c->sm_count, c->opt_max_ctas, plan);
    return use_mma;
}

// Where kvs_decode_attention_weights reads and leaves the running totals of the rows' softmax weights.
struct WeightTotals {
    const float* in;     // nullptr: totals start at zero
    float* out;
    int stride;
    int score_stride;    // floats between the scores of consecutive q-heads
};

// Split-K kernel + combine kernel of one layer, with the given plan and scratch, over `units` (sequence, kv-head) units of
// the slot from unit0 on.  q and out: of the whole batch.
// With k_new / v_new the split-K kernel also appends that one row per unit (the slot's length must
// already count it).
kvs_status run_attention(kvs_ctx* c, int slot, const void* q, float* out, int unit0, int units, const kvs::DecodePlan& plan,
                         bool use_mma, const AttentionScratch& scratch, cudaStream_t st, const void* k_new = nullptr,
                         const void* v_new = nullptr, const WeightTotals* totals = nullptr) {
    kvs::DecodeArgs a;
    const size_t skipped = (size_t)unit0 * c->row_stride * c->row_bytes, heads0 = (size_t)unit0 * c->G * c->cfg.head_dim;
    a.q = static_cast<const char*>(q) + heads0 * c->elem;
    a.kplane = c->pool + (size_t)(2 * slot) * c->plane_bytes + skipped;
    a.vplane = c->pool + (size_t)(2 * slot + 1) * c->plane_bytes + skipped;
    a.part_o = scratch.part_o;
    a.part_ml = scratch.part_ml;
    a.out = out + heads0;
    a.status = scratch.status;
    a.n = c->slot_len[slot];
    a.row_stride = c->row_stride;
    a.capacity = c->cfg.max_seq;
    a.units = units;
    a.G = c->G;
    a.D = c->cfg.head_dim;
    a.dtype = c->cfg.dtype;
    a.scale_log2 = c->scale * 1.4426950408889634f;
    a.programmatic = scratch.programmatic;
    a.safe_rows = scratch.programmatic ? safe_rows_of(c, slot) : 0;
    a.unit_len = c->ragged[slot] ? unit_len_dev(c, slot) + unit0 : nullptr;
    a.n_extra = replay_counter(c);
    a.k_new = k_new;
    a.v_new = v_new;
    if (k_new) a.safe_rows = std::min(a.safe_rows, a.n - 1);   // the new row is fetched after the kernel has stored it
    a.plane_bytes = (long long)(c->plane_bytes - skipped);
    a.wait_ns = 1000ull * (unsigned long long)c->opt_wait_us;
    a.trace = nullptr;
    if (c->trace_buf && c->trace_launch < c->trace_capacity)
        a.trace = c->trace_buf + (size_t)(c->trace_launch++) * kvs::kTraceLaunchWords;
    a.stall_tile = c->stall_tile >= 0 ? std::min<long long>(c->stall_tile, plan.T - 1) : -1;
    c->stall_tile = -1;
    // with totals the unit's (max, sum) are needed beyond its output: always the separate finishing kernel
    a.finish_in_kernel = c->opt_finish != 0 && kvs::can_finish_in_kernel(plan, a.units) && totals == nullptr;
    a.scores = totals ? reinterpret_cast<float*>(c->ws + c->off_scores) : nullptr;
    a.score_stride = totals ? totals->score_stride : 0;
    a.score_count = (long long)(c->score_bytes / sizeof(float));
    a.flags = scratch.flags;
    if (scratch.tracked) {
        c->seq += a.finish_in_kernel ? 1 : 2;     // split-K kernel, then (unless it finishes the units itself) combine
        c->last_splitk_seq = a.finish_in_kernel ? c->seq : c->seq - 1;
    }
    if (c->format == KVS_CACHE_4BIT) {
        if ((plan.kernel == 3 ? kvs::launch_decode_pack4(a, plan, st) : kvs::launch_decode_pack4_f32(a, plan, st)) != cudaSuccess)
            return KVS_ERR_CUDA;
    } else if (use_mma) {
        const long long plane_rows = (long long)c->cfg.max_batch * c->cfg.n_kv_heads * c->row_stride;
        const long long row0 = (long long)unit0 * c->row_stride;
        if (kvs::launch_decode_mma(a, plan, c->tensor_map, c->tensor_map_tail, plane_rows * (2 * slot) + row0,
                                   plane_rows * (2 * slot + 1) + row0, st) != cudaSuccess)
            return KVS_ERR_CUDA;
    } else {
        if (kvs::launch_decode_scalar(a, plan, st) != cudaSuccess) return KVS_ERR_CUDA;
    }
    if (!a.finish_in_kernel) {
        const size_t total0 = totals ? (size_t)unit0 * totals->stride : 0;
        const cudaError_t e = totals ? kvs::launch_weights_finish(a, plan, totals->in ? totals->in + total0 : nullptr, totals->out + total0,
                                                                  totals->stride, c->sm_count, st)
                                     : kvs::launch_combine(a, plan, st);
        if (e != cudaSuccess) return KVS_ERR_CUDA;
        c->stats.combine_launches += 1;
    }
    c->last_plan = plan;
    c->stats.attention_launches += 1;
    if (c->ragged[slot]) {
        unsigned long long rows = 0;
        for (int u = unit0; u < unit0 + a.units; ++u) rows += c->unit_len_host[slot][u];
        c->stats.kv_bytes_read += 2ull * rows * c->row_bytes;
    } else {
        c->stats.kv_bytes_read += 2ull * a.units * a.n * c->row_bytes;
    }
    return KVS_OK;
}

// Whether the attention kernel of the slot can store the step's new rows itself (all but the one over 4-bit rows for fp32).
bool can_fuse_append(const kvs_ctx* c, int slot) {
    return !c->ragged[slot] && (c->format == KVS_CACHE_PLAIN || c->cfg.dtype == KVS_BF16);
}

// One decode step of a computing layer with the append riding in the split-K kernel (the caller
// has checked the arguments; the slot is not ragged).
kvs_status do_fused_step(kvs_ctx* c, int layer, const void* q, const void* k, const void* v, float* out, int batch,
                         cudaStream_t st) {
    const int slot = c->slot_of_layer[layer];
    const int old_len = c->slot_len[slot];
    kvs::DecodePlan plan;
    const bool use_mma = choose_plan(c, batch * c->cfg.n_kv_heads, old_len + 1, &plan);
    const AttentionScratch scratch = {reinterpret_cast<float*>(c->ws + c->off_part_o),
                                      reinterpret_cast<float*>(c->ws + c->off_part_ml),
                                      reinterpret_cast<int*>(c->ws + c->off_flags),
                                      reinterpret_cast<int*>(c->ws + c->off_status), take_early_start(c), true};
    // run_attention works out which rows are stable from the appends before this one
    c->slot_len[slot] = old_len + 1;
    const kvs_status s = run_attention(c, slot, q, out, 0, batch * c->cfg.n_kv_heads, plan, use_mma, scratch, st, k, v);
    if (s != KVS_OK) {
        c->slot_len[slot] = old_len;
        return s;
    }
    c->app_seq_prev[slot] = c->app_seq_latest[slot];
    c->app_seq_latest[slot] = c->last_splitk_seq;   // the kernel that appended is the split-K kernel itself
    c->app_start_latest[slot] = old_len;
    c->cur_batch = batch;
    c->stats.fused_appends += 1;
    c->stats.kv_bytes_appended += 2ull * batch * c->cfg.n_kv_heads * c->row_bytes;
    return KVS_OK;
}

kvs_status do_attention(kvs_ctx* c, int layer, const void* q, float* out, int batch, cudaStream_t st,
                        WeightTotals* totals = nullptr) {
    const int slot = c->slot_of_layer[layer], units = batch * c->cfg.n_kv_heads;
    int step = units;
    if (totals) {
        // as many units at a time as there is room for their scores; a recorded launch grows up to the capacity
        totals->score_stride = c->opt_replay ? c->row_stride : (int)align_up(c->slot_len[slot], kRowStrideQuantum);
        const int most = (int)std::min<size_t>(units, c->score_bytes / ((size_t)c->G * totals->score_stride * sizeof(float)));
        const int passes = (units + most - 1) / most;
        step = (units + passes - 1) / passes;
    }
    for (int u0 = 0; u0 < units; u0 += step) {
        const int count = std::min(step, units - u0);
        kvs::DecodePlan plan;
        const bool use_mma = choose_plan(c, count, c->slot_len[slot], &plan);
        const AttentionScratch scratch = {reinterpret_cast<float*>(c->ws + c->off_part_o),
                                          reinterpret_cast<float*>(c->ws + c->off_part_ml),
                                          reinterpret_cast<int*>(c->ws + c->off_flags),
                                          reinterpret_cast<int*>(c->ws + c->off_status), take_early_start(c), true};
        const kvs_status s = run_attention(c, slot, q, out, u0, count, plan, use_mma, scratch, st, nullptr, nullptr, totals);
        if (s != KVS_OK) return s;
    }
    return KVS_OK;
}

// Rows of unit `u` of `slot` as the host knows them.
int unit_rows(const kvs_ctx* c, int slot, int u) { return c->ragged[slot] ? c->unit_len_host[slot][u] : c->slot_len[slot]; }

// Whether every unit of the slot's first `batch` sequences holds at least `rows` rows.
bool holds_rows(const kvs_ctx* c, int slot, int batch, int rows) {
    if (!c->ragged[slot]) return c->slot_len[slot] >= rows;
    for (int u = 0; u < batch * c->cfg.n_kv_heads; ++u)
        if (c->unit_len_host[slot][u] < rows) return false;
    return true;
}

// Rows of a 4-bit slot in the storage type, into the scratch: sequences seq0 .. seq0+seqs-1, rows 0 .. n-1, laid out as planes
// [seqs][Hkv][stride][D] of K, then of V.
cudaError_t plain_rows(kvs_ctx* c, int slot, int seq0, int seqs, int n, int stride, cudaStream_t st) {
    const size_t skipped = (size_t)seq0 * c->cfg.n_kv_heads * c->row_stride * c->row_bytes;
    const long long D = c->cfg.head_dim, head = stride * D, seq = c->cfg.n_kv_heads * head;
    kvs::ReadArgs r = {};
    r.kplane = c->pool + (size_t)(2 * slot) * c->plane_bytes + skipped;
    r.vplane = static_cast<const char*>(r.kplane) + c->plane_bytes;
    r.packed = true;
    r.row_stride = c->row_stride;
    r.first = 0;
    r.n = n;
    r.k_out = c->ws + c->off_plain;
    r.v_out = c->ws + c->off_plain + (size_t)seqs * seq * c->elem;
    r.dst_b = seq;
    r.dst_t = D;
    r.dst_h = head;
    r.batch = seqs;
    r.Hkv = c->cfg.n_kv_heads;
    r.D = c->cfg.head_dim;
    r.dtype = c->cfg.dtype;
    r.status = reinterpret_cast<int*>(c->ws + c->off_status);
    r.plane_bytes = (long long)(c->plane_bytes - skipped);
    r.sm_count = c->sm_count;
    r.programmatic = take_early_start(c);
    return kvs::launch_read_rows(r, st);
}

// Sequences whose rows, `stride` of them per head, the scratch holds at a time.
int plain_seqs(const kvs_ctx* c, int batch, int stride) {
    const size_t seq = 2ull * c->cfg.n_kv_heads * stride * c->cfg.head_dim * c->elem;
    return (int)std::min<size_t>(batch, c->plain_bytes / seq);
}

// Every row of the slot may just have moved: nothing of it may be fetched early.
void rows_moved(kvs_ctx* c, int slot) {
    c->app_seq_prev[slot] = c->seq;
    c->app_seq_latest[slot] = c->seq;
    c->app_start_latest[slot] = 0;
}

}  // namespace

extern "C" {

kvs_status kvs_create(const kvs_config* cfg, kvs_ctx** out) {
    if (!cfg || !out) return KVS_ERR_INVALID_ARG;
    *out = nullptr;
    if (cfg->n_layers < 1 || cfg->n_q_heads < 1 || cfg->n_kv_heads < 1 || cfg->max_batch < 1 || cfg->max_seq < 1)
        return KVS_ERR_INVALID_ARG;
    if (cfg->n_q_heads % cfg->n_kv_heads != 0) return KVS_ERR_INVALID_ARG;
    const int G = cfg->n_q_heads / cfg->n_kv_heads;
    const bool pow2_group = (G == 1 || G == 2 || G == 4 || G == 8);
    if (G > 8) return KVS_ERR_INVALID_ARG;
    // groups of 3, 5, 6 or 7 q-heads exist only on the tensor-core kernel, which is bf16-only
    if (!pow2_group && cfg->dtype != KVS_BF16) return KVS_ERR_INVALID_ARG;
    if (cfg->head_dim != 64 && cfg->head_dim != 128) return KVS_ERR_INVALID_ARG;
    if (cfg->dtype != KVS_BF16 && cfg->dtype != KVS_F32) return KVS_ERR_INVALID_ARG;
    if (cfg->device < 0 || cfg->device >= 64) return KVS_ERR_INVALID_ARG;
    if (!(cfg->softmax_scale >= 0.f) || std::isinf(cfg->softmax_scale)) return KVS_ERR_INVALID_ARG;
    if (cfg->max_seq > (1 << 30) - kRowStrideQuantum) return KVS_ERR_INVALID_ARG;
    kvs_ctx* c = new (std::nothrow) kvs_ctx();
    if (!c) return KVS_ERR_OOM;
    c->cfg = *cfg;
    c->G = G;
    c->elem = cfg->dtype == KVS_BF16 ? 2 : 4;
    c->row_stride = (cfg->max_seq + kRowStrideQuantum - 1) / kRowStrideQuantum * kRowStrideQuantum;
    c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt((float)cfg->head_dim);
    c->share_map.resize(cfg->n_layers);
    for (int l = 0; l < cfg->n_layers; ++l) c->share_map[l] = l;
    resolve_map(c);
    layout_workspace(c);
    *out = c;
    return KVS_OK;
}

kvs_status kvs_destroy(kvs_ctx* ctx) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (ctx->copy_ready) {
        DeviceGuard guard(ctx->cfg.device);
        if (guard.ok) {
            for (int i = 0; i < kvs_ctx::kChunks; ++i) {
                cudaEventDestroy(ctx->ev_in[i]);
                cudaEventDestroy(ctx->ev_done[i]);
            }
            cudaEventDestroy(ctx->ev_start);
            cudaStreamDestroy(ctx->copy_stream);
            cudaStreamDestroy(ctx->out_stream);
        }
    }
    delete ctx;
    return KVS_OK;
}

kvs_status kvs_set_share_map(kvs_ctx* ctx, const int32_t* share_map) {
    if (!ctx || !share_map) return KVS_ERR_INVALID_ARG;
    for (int s = 0; s < ctx->n_slots; ++s)
        if (ctx->slot_len[s] != 0) return KVS_ERR_STATE;
    const int L = ctx->cfg.n_layers;
    for (int l = 0; l < L; ++l)
        if (share_map[l] < 0 || share_map[l] > l) return KVS_ERR_BAD_SHARE_MAP;
    const int old_slots = ctx->n_slots;
    for (int l = 0; l < L; ++l) ctx->share_map[l] = share_map[l];
    resolve_map(ctx);
    // A pool bound for fewer slots than the new strategy needs can no longer be used.
    if (ctx->bound && ctx->n_slots > old_slots) {
        ctx->bound = false;
        ctx->pool = nullptr;
        ctx->ws = nullptr;
    }
    return KVS_OK;
}

kvs_status kvs_set_cache_format(kvs_ctx* ctx, int32_t format) {
    if (!ctx || (format != KVS_CACHE_PLAIN && format != KVS_CACHE_4BIT)) return KVS_ERR_INVALID_ARG;
    for (int s = 0; s < ctx->n_slots; ++s)
        if (ctx->slot_len[s] != 0) return KVS_ERR_STATE;
    if (format == ctx->format) return KVS_OK;
    ctx->format = format;
    layout_workspace(ctx);
    ctx->bound = false;        // pool and workspace have other sizes now
    ctx->pool = nullptr;
    ctx->ws = nullptr;
    return KVS_OK;
}

kvs_status kvs_required_bytes(const kvs_ctx* ctx, size_t* pool_bytes, size_t* workspace_bytes) {
    if (!ctx || !pool_bytes || !workspace_bytes) return KVS_ERR_INVALID_ARG;
    *pool_bytes = (size_t)ctx->n_slots * 2 * ctx->plane_bytes;
    *workspace_bytes = ctx->ws_bytes;
    return KVS_OK;
}

kvs_status kvs_bind_memory(kvs_ctx* ctx, void* pool, size_t pool_bytes, void* workspace, size_t workspace_bytes) {
    if (!ctx || !pool || !workspace) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)pool % kAlign) != 0 || ((uintptr_t)workspace % kAlign) != 0) return KVS_ERR_INVALID_ARG;
    const size_t need_pool = (size_t)ctx->n_slots * 2 * ctx->plane_bytes;
    if (pool_bytes < need_pool || workspace_bytes < ctx->ws_bytes) return KVS_ERR_OOM;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    if (init_device_once(ctx->cfg.device) != cudaSuccess) return KVS_ERR_CUDA;
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, ctx->cfg.device) != cudaSuccess) return KVS_ERR_CUDA;
    if (cudaMemsetAsync(pool, 0, need_pool, 0) != cudaSuccess) return KVS_ERR_CUDA;
    if (cudaMemsetAsync(workspace, 0, ctx->ws_bytes, 0) != cudaSuccess) return KVS_ERR_CUDA;
    if (cudaStreamSynchronize(0) != cudaSuccess) return KVS_ERR_CUDA;
    ctx->have_tensor_map = false;
    if (ctx->cfg.dtype == KVS_BF16 && ctx->format == KVS_CACHE_4BIT) {
        const long long rows = (long long)(ctx->plain_bytes / ((size_t)ctx->cfg.head_dim * ctx->elem));
        if (rows >= (1ll << 31)) return KVS_ERR_INVALID_ARG;
        if (kvs::make_pool_tensor_map(ctx->plain_map, static_cast<char*>(workspace) + ctx->off_plain, rows, ctx->cfg.head_dim, false) != cudaSuccess)
            return KVS_ERR_CUDA;
    } else if (ctx->cfg.dtype == KVS_BF16) {
        const long long total_rows = (long long)(need_pool / ctx->row_bytes);
        if (total_rows >= (1ll << 31)) return KVS_ERR_INVALID_ARG;
        if (kvs::make_pool_tensor_map(ctx->tensor_map, pool, total_rows, ctx->cfg.head_dim, false) != cudaSuccess ||
            kvs::make_pool_tensor_map(ctx->tensor_map_tail, pool, total_rows, ctx->cfg.head_dim, true) != cudaSuccess)
            return KVS_ERR_CUDA;
        ctx->have_tensor_map = true;
    }
    ctx->sm_count = sms;
    {
        int l2 = 0;
        if (cudaDeviceGetAttribute(&l2, cudaDevAttrL2CacheSize, ctx->cfg.device) == cudaSuccess && l2 > 0) ctx->l2_bytes = l2;
    }
    ctx->pool = static_cast<char*>(pool);
    ctx->ws = static_cast<char*>(workspace);
    ctx->bound = true;
    for (auto& x : ctx->slot_len) x = 0;
    for (auto& x : ctx->ragged) x = 0;
    ctx->cur_batch = 0;
    // the device was idle a moment ago: nothing of this context is in flight
    for (auto& x : ctx->app_seq_latest) x = 0;
    for (auto& x : ctx->app_seq_prev) x = 0;
    ctx->last_splitk_seq = 0;
    return KVS_OK;
}

kvs_status kvs_reset(kvs_ctx* ctx) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    for (auto& x : ctx->ragged) x = 0;
    for (auto& x : ctx->slot_len) x = 0;
    ctx->cur_batch = 0;
    return KVS_OK;
}

kvs_status kvs_truncate(kvs_ctx* ctx, int32_t n_tokens) {
    if (!ctx || n_tokens < 0) return KVS_ERR_INVALID_ARG;
    // a slot rows were evicted from has per-unit lengths on the device as well: refused, not half-updated
    for (int s = 0; s < ctx->n_slots; ++s)
        if (ctx->slot_len[s] > n_tokens && ctx->ragged[s]) return KVS_ERR_STATE;
    for (int s = 0; s < ctx->n_slots; ++s) {
        if (ctx->slot_len[s] <= n_tokens) continue;
        ctx->slot_len[s] = n_tokens;
        // Rows from n_tokens on will be written again.  Kernels of earlier calls may still be reading
        // them, but every writer stores only after its wait for its predecessor; and what a later
        // launch may fetch before its own wait must lie below the old and the new writes alike.
        ctx->app_start_latest[s] = std::min(ctx->app_start_latest[s], n_tokens);
    }
    if (n_tokens == 0) ctx->cur_batch = 0;
    return KVS_OK;
}

kvs_status kvs_append(kvs_ctx* ctx, int32_t layer, const void* k, const void* v, int32_t batch, int32_t n_new,
                      void* stream) {
    bool sharing = false;
    kvs_status s = check_append(ctx, layer, k, v, batch, n_new, &sharing);
    if (s != KVS_OK) return s;
    if (sharing) {
        ctx->stats.append_skipped += 1;
        return KVS_OK;
    }
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    return do_append(ctx, layer, k, v, batch, n_new, static_cast<cudaStream_t>(stream));
}

kvs_status kvs_decode_attention(kvs_ctx* ctx, int32_t layer, const void* q, float* out, int32_t batch, void* stream) {
    kvs_status s = check_attention(ctx, layer, q, out, batch);
    if (s != KVS_OK) return s;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    return do_attention(ctx, layer, q, out, batch, static_cast<cudaStream_t>(stream));
}

kvs_status kvs_decode_step(kvs_ctx* ctx, int32_t layer, const void* q, const void* k, const void* v, float* out,
                           int32_t batch, void* stream) {
    bool sharing = false;
    kvs_status s = check_append(ctx, layer, k, v, batch, 1, &sharing);
    if (s != KVS_OK) return s;
    if (!q || !out) return KVS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (sharing) {
        s = check_attention(ctx, layer, q, out, batch);
        if (s != KVS_OK) return s;
        DeviceGuard guard(ctx->cfg.device);
        if (!guard.ok) return KVS_ERR_CUDA;
        ctx->stats.append_skipped += 1;
        return do_attention(ctx, layer, q, out, batch, st);
    }
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    const int slot = ctx->slot_of_layer[layer];
    if (((uintptr_t)q % 16) != 0 || ((uintptr_t)out % 4) != 0) return KVS_ERR_INVALID_ARG;
    if (can_fuse_append(ctx, slot)) return do_fused_step(ctx, layer, q, k, v, out, batch, st);
    s = do_append(ctx, layer, k, v, batch, 1, st);
    if (s != KVS_OK) return s;
    return do_attention(ctx, layer, q, out, batch, st);
}

kvs_status kvs_prefill_attention(kvs_ctx* ctx, int32_t layer, const void* q, float* out, int32_t batch, int32_t n_q,
                                 void* stream) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    if (layer < 0 || layer >= ctx->cfg.n_layers || !q || !out) return KVS_ERR_INVALID_ARG;
    if (batch < 1 || batch > ctx->cfg.max_batch || n_q < 1) return KVS_ERR_INVALID_ARG;
    const bool packed = ctx->format == KVS_CACHE_4BIT;
    if (ctx->cfg.dtype == KVS_BF16 && !packed && !ctx->have_tensor_map) return KVS_ERR_STATE;
    if (((uintptr_t)q % 16) != 0 || ((uintptr_t)out % 16) != 0) return KVS_ERR_INVALID_ARG;
    const int slot = ctx->slot_of_layer[layer];
    const int n = ctx->slot_len[slot];
    if (n == 0 || ctx->ragged[slot]) return KVS_ERR_STATE;   // positions are undefined once rows were evicted
    if (batch > ctx->cur_batch || n_q > n) return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    if (packed) {
        // Sequences at a time: their rows in the storage type into the scratch, then the kernel a plain cache gets.  The rows
        // take 2 (D + 32 + 2 D e) bytes a token and head, the attention reads them n_q / 128 times.
        const kvs_config& f = ctx->cfg;
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        const int stride = (int)align_up(n, kRowStrideQuantum), step = plain_seqs(ctx, batch, stride);
        for (int b0 = 0; b0 < batch; b0 += step) {
            const int seqs = std::min(step, batch - b0);
            if (plain_rows(ctx, slot, b0, seqs, n, stride, st) != cudaSuccess) return KVS_ERR_CUDA;
            const size_t heads0 = (size_t)b0 * n_q * f.n_q_heads * f.head_dim;
            const char* qb = static_cast<const char*>(q) + heads0 * ctx->elem;
            const long long rows = (long long)seqs * f.n_kv_heads * stride;      // of one of the two planes
            const char* kp = ctx->ws + ctx->off_plain;
            const cudaError_t e =
                f.dtype == KVS_F32
                    ? kvs::launch_prefill_f32(qb, out + heads0, kp, kp + (size_t)rows * f.head_dim * ctx->elem, seqs, n_q, f.n_q_heads, ctx->G,
                                              f.head_dim, n, stride, ctx->scale * 1.4426950408889634f, st)
                    : kvs::launch_prefill(qb, out + heads0, reinterpret_cast<int*>(ctx->ws + ctx->off_status),
                                          reinterpret_cast<int*>(ctx->ws + ctx->off_status + 64), ctx->plain_map, seqs, n_q, f.n_q_heads, ctx->G,
                                          f.head_dim, n, stride, 0, rows, rows, ctx->scale * 1.4426950408889634f, ctx->sm_count, ctx->l2_bytes, st);
            if (e != cudaSuccess) return KVS_ERR_CUDA;
            ctx->seq += 2;
            ctx->last_splitk_seq = ctx->seq;     // the attention is a plain launch
            ctx->counter_written = false;
        }
        ctx->stats.prefill_launches += 1;
        return KVS_OK;
    }
    if (ctx->cfg.dtype == KVS_F32) {
        // fp32 storage: the plain fp32 kernel (a plain launch, like the tensor-core one)
        const char* kp = ctx->pool + (size_t)(2 * slot) * ctx->plane_bytes;
        if (kvs::launch_prefill_f32(q, out, kp, kp + ctx->plane_bytes, batch, n_q, ctx->cfg.n_q_heads, ctx->G,
                                    ctx->cfg.head_dim, n, ctx->row_stride, ctx->scale * 1.4426950408889634f,
                                    static_cast<cudaStream_t>(stream)) != cudaSuccess)
            return KVS_ERR_CUDA;
        ctx->seq += 1;
        ctx->last_splitk_seq = ctx->seq;
        ctx->stats.prefill_launches += 1;
        ctx->counter_written = false;
        return KVS_OK;
    }
    const long long plane_rows = (long long)ctx->cfg.max_batch * ctx->cfg.n_kv_heads * ctx->row_stride;
    // the prefill kernel's work counter lives in the status block, 64 bytes after the status word
    if (kvs::launch_prefill(q, out, reinterpret_cast<int*>(ctx->ws + ctx->off_status),
                            reinterpret_cast<int*>(ctx->ws + ctx->off_status + 64), ctx->tensor_map, batch, n_q,
                            ctx->cfg.n_q_heads, ctx->G, ctx->cfg.head_dim, n, ctx->row_stride, plane_rows * (2 * slot),
                            plane_rows * (2 * slot + 1), plane_rows, ctx->scale * 1.4426950408889634f, ctx->sm_count, ctx->l2_bytes,
                            static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return KVS_ERR_CUDA;
    // a plain launch: it starts only after everything before it on the stream has finished
    ctx->seq += 1;
    ctx->last_splitk_seq = ctx->seq;
    ctx->stats.prefill_launches += 1;
    ctx->counter_written = false;   // a plain launch: full dependency on everything before it
    ctx->stats.kv_bytes_read += 0;  // prefill is compute-bound; its K/V reads are not counted as decode traffic
    return KVS_OK;
}

kvs_status kvs_evict(kvs_ctx* ctx, int32_t layer, const int32_t* keep, const int32_t* n_keep, int32_t keep_stride,
                     int32_t batch, void* stream) {
    if (!ctx || !keep || !n_keep) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    if (layer < 0 || layer >= ctx->cfg.n_layers || keep_stride < 1) return KVS_ERR_INVALID_ARG;
    if (ctx->share_map[layer] != layer) return KVS_ERR_INVALID_ARG;   // a sharing layer has no cache of its own
    const int slot = ctx->slot_of_layer[layer];
    if (ctx->slot_len[slot] == 0) return KVS_ERR_STATE;
    if (batch < 1 || batch != ctx->cur_batch) return KVS_ERR_INVALID_ARG;
    const int units = batch * ctx->cfg.n_kv_heads;
    int longest = 0;
    for (int u = 0; u < units; ++u) {
        const int have = ctx->ragged[slot] ? ctx->unit_len_host[slot][u] : ctx->slot_len[slot];
        if (n_keep[u] < 1 || n_keep[u] > have || n_keep[u] > keep_stride) return KVS_ERR_INVALID_ARG;
        longest = n_keep[u] > longest ? n_keep[u] : longest;
    }
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int* counts = reinterpret_cast<int*>(ctx->ws + ctx->off_counts);
    int* lens = unit_len_dev(ctx, slot);
    if (kvs::launch_put_counts(counts, n_keep, units, st) != cudaSuccess) return KVS_ERR_CUDA;
    char* kp = ctx->pool + (size_t)(2 * slot) * ctx->plane_bytes;
    const bool pdl = ctx->opt_pdl != 0;
    if (kvs::launch_evict(kp, kp + ctx->plane_bytes, keep, counts, ctx->ragged[slot] ? lens : nullptr,
                          ctx->slot_len[slot], units, keep_stride, ctx->row_bytes, ctx->row_stride,
                          reinterpret_cast<int*>(ctx->ws + ctx->off_status), false, st) != cudaSuccess ||
        kvs::launch_set_len(lens, counts, units, pdl, st) != cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->unit_len_host[slot].assign((size_t)ctx->cfg.max_batch * ctx->cfg.n_kv_heads, 0);
    for (int u = 0; u < units; ++u) ctx->unit_len_host[slot][u] = n_keep[u];
    ctx->ragged[slot] = 1;
    ctx->slot_len[slot] = longest;
    // every row of the slot may just have moved: nothing of it may be fetched early
    ctx->seq += 2;
    rows_moved(ctx, slot);
    ctx->stats.evict_launches += 1;
    ctx->counter_written = false;   // a plain launch: full dependency on everything before it
    return KVS_OK;
}

kvs_status kvs_append_rotary(kvs_ctx* ctx, int32_t layer, const kvs_rotary* rot, const void* q, int64_t q_stride,
                             const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                             const void* q_weight, const void* k_weight, void* q_out, int32_t batch, int32_t n_new,
                             void* stream) {
    bool sharing = false;
    kvs_status s = check_append(ctx, layer, k, v, batch, n_new, &sharing);
    if (s != KVS_OK) return s;
    const kvs_config& f = ctx->cfg;
    if (!rot || !q || !q_out) return KVS_ERR_INVALID_ARG;
    if (rot->rotary_dim < 0 || rot->rotary_dim > f.head_dim || rot->rotary_dim % 16 != 0) return KVS_ERR_INVALID_ARG;
    if (rot->interleaved != 0 && rot->interleaved != 1) return KVS_ERR_INVALID_ARG;
    if (rot->rotary_dim > 0 && (!rot->inv_freq || !positions)) return KVS_ERR_INVALID_ARG;
    for (int i = 0; i < rot->rotary_dim / 2; ++i)
        if (!std::isfinite(rot->inv_freq[i])) return KVS_ERR_INVALID_ARG;
    if (!(rot->eps >= 0.f) || std::isinf(rot->eps)) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)q % 16) != 0 || ((uintptr_t)q_out % 16) != 0 || ((uintptr_t)positions % 4) != 0 ||
        ((uintptr_t)q_weight % 16) != 0 || ((uintptr_t)k_weight % 16) != 0)
        return KVS_ERR_INVALID_ARG;
    // token strides: 16-byte vector loads, and no two tokens overlap
    const int per = 16 / ctx->elem;
    const long long q_row = (long long)f.n_q_heads * f.head_dim, kv_row = (long long)f.n_kv_heads * f.head_dim;
    if (q_stride < q_row || q_stride % per != 0) return KVS_ERR_INVALID_ARG;
    if (!sharing && (k_stride < kv_row || k_stride % per != 0 || v_stride < kv_row || v_stride % per != 0))
        return KVS_ERR_INVALID_ARG;
    if ((long long)batch * n_new > 0x7fffffffll) return KVS_ERR_INVALID_ARG;
    if (q == q_out && q_stride != q_row && (long long)batch * n_new > 1) return KVS_ERR_INVALID_ARG;   // in place: packed rows only
    DeviceGuard guard(f.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    const int slot = ctx->slot_of_layer[layer];
    kvs::RotaryArgs r = {};
    r.q = q;
    r.q_stride = q_stride;
    r.positions = positions;
    r.q_weight = q_weight;
    r.q_out = q_out;
    r.batch = batch;
    r.n_new = n_new;
    r.Hq = f.n_q_heads;
    r.D = f.head_dim;
    r.dtype = f.dtype;
    r.inv_freq = rot->inv_freq;
    r.rotary_dim = rot->rotary_dim;
    r.interleaved = rot->interleaved != 0;
    r.eps = rot->eps;
    r.sm_count = ctx->sm_count;
    r.status = reinterpret_cast<int*>(ctx->ws + ctx->off_status);
    if (!sharing) {
        r.k = k;
        r.k_stride = k_stride;
        r.v = v;
        r.v_stride = v_stride;
        r.k_weight = k_weight;
        r.Hkv = f.n_kv_heads;
        r.kplane = ctx->pool + (size_t)(2 * slot) * ctx->plane_bytes;
        r.vplane = ctx->pool + (size_t)(2 * slot + 1) * ctx->plane_bytes;
        r.row_stride = ctx->row_stride;
        r.len0 = ctx->slot_len[slot];
        r.capacity = f.max_seq;
        r.unit_len = ctx->ragged[slot] ? unit_len_dev(ctx, slot) : nullptr;
        r.n_extra = replay_counter(ctx);
        r.plane_bytes = (long long)ctx->plane_bytes;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!sharing && ctx->format == KVS_CACHE_4BIT) {
        // sequences at a time: finished keys and values into the scratch, from there into the 4-bit rows
        const long long head = (long long)n_new * f.head_dim, seq = f.n_kv_heads * head;
        const int step = plain_seqs(ctx, batch, n_new);
        r.row_stride = r.capacity = n_new;
        r.len0 = 0;
        r.unit_len = nullptr;
        r.n_extra = nullptr;
        for (int b0 = 0; b0 < batch; b0 += step) {
            const long long tok0 = (long long)b0 * n_new;
            r.batch = std::min(step, batch - b0);
            r.q = static_cast<const char*>(q) + tok0 * q_stride * ctx->elem;
            r.k = static_cast<const char*>(k) + tok0 * k_stride * ctx->elem;
            r.v = static_cast<const char*>(v) + tok0 * v_stride * ctx->elem;
            r.positions = positions ? positions + tok0 : nullptr;
            r.q_out = static_cast<char*>(q_out) + tok0 * q_row * ctx->elem;
            r.kplane = ctx->ws + ctx->off_plain;
            r.vplane = ctx->ws + ctx->off_plain + (size_t)r.batch * seq * ctx->elem;
            r.plane_bytes = (long long)r.batch * seq * ctx->elem;
            r.programmatic = take_early_start(ctx);
            if (kvs::launch_append_rotary(r, st) != cudaSuccess ||
                store_packed(ctx, slot, r.kplane, r.vplane, seq, f.head_dim, head, b0, r.batch, n_new, st) != cudaSuccess)
                return KVS_ERR_CUDA;
            ctx->seq += 2;
        }
        return appended(ctx, slot, batch, n_new, st);
    }
    r.programmatic = take_early_start(ctx);
    if (kvs::launch_append_rotary(r, st) != cudaSuccess) return KVS_ERR_CUDA;
    if (!sharing) return appended(ctx, slot, batch, n_new, st);
    ctx->seq += 1;
    ctx->stats.append_skipped += 1;
    return KVS_OK;
}

kvs_status kvs_tree_attention(kvs_ctx* ctx, int32_t layer, const void* q, void* out, const uint64_t* mask, int32_t batch,
                              int32_t n_t, void* stream) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || ctx->opt_replay || ctx->format == KVS_CACHE_4BIT) return KVS_ERR_STATE;
    if (ctx->cfg.dtype == KVS_BF16 && !ctx->have_tensor_map) return KVS_ERR_STATE;
    if (layer < 0 || layer >= ctx->cfg.n_layers || !q || !out) return KVS_ERR_INVALID_ARG;
    if (batch < 1 || batch > ctx->cfg.max_batch || n_t < 1 || n_t > kvs::kTreeMaxTokens) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)q % 16) != 0 || ((uintptr_t)out % 16) != 0 || ((uintptr_t)mask % 8) != 0) return KVS_ERR_INVALID_ARG;
    if (q == out) return KVS_ERR_INVALID_ARG;   // one block's result would overwrite another's queries
    const int slot = ctx->slot_of_layer[layer];
    if (ctx->slot_len[slot] == 0) return KVS_ERR_STATE;
    if (batch > ctx->cur_batch || !holds_rows(ctx, slot, batch, n_t)) return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    kvs::TreeArgs a;
    a.q = q;
    a.out = out;
    a.mask = reinterpret_cast<const unsigned long long*>(mask);
    a.kplane = ctx->pool + (size_t)(2 * slot) * ctx->plane_bytes;
    a.vplane = ctx->pool + (size_t)(2 * slot + 1) * ctx->plane_bytes;
    a.part_o = reinterpret_cast<float*>(ctx->ws + ctx->off_tree_o);
    a.part_ml = reinterpret_cast<float*>(ctx->ws + ctx->off_tree_ml);
    a.status = reinterpret_cast<int*>(ctx->ws + ctx->off_status);
    a.n = ctx->slot_len[slot];
    a.unit_len = ctx->ragged[slot] ? unit_len_dev(ctx, slot) : nullptr;
    a.n_t = n_t;
    a.units = batch * ctx->cfg.n_kv_heads;
    a.B = batch;
    a.Hq = ctx->cfg.n_q_heads;
    a.Hkv = ctx->cfg.n_kv_heads;
    a.G = ctx->G;
    a.D = ctx->cfg.head_dim;
    a.dtype = ctx->cfg.dtype;
    a.row_stride = ctx->row_stride;
    a.capacity = ctx->cfg.max_seq;
    a.plane_bytes = (long long)ctx->plane_bytes;
    a.scale_log2 = ctx->scale * 1.4426950408889634f;
    a.wait_ns = 1000ull * (unsigned long long)ctx->opt_wait_us;
    a.programmatic = take_early_start(ctx);
    a.pool_map = ctx->tensor_map;
    a.pool_map_tail = ctx->tensor_map_tail;
    const long long plane_rows = (long long)ctx->cfg.max_batch * ctx->cfg.n_kv_heads * ctx->row_stride;
    a.krow0 = plane_rows * (2 * slot);
    a.vrow0 = plane_rows * (2 * slot + 1);
    int launches = 0;
    if (kvs::launch_tree(a, ctx->sm_count, ctx->opt_max_ctas, &launches, static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return KVS_ERR_CUDA;
    // like a split-K kernel, the attention kernel lets its successor start only after its own wait
    ctx->last_splitk_seq = ctx->seq + 1;
    ctx->seq += launches;
    ctx->stats.prefill_launches += 1;
    return KVS_OK;
}

kvs_status kvs_accept_draft(kvs_ctx* ctx, const int32_t* path, int32_t path_stride, const int32_t* n_accept, int32_t n_draft,
                            int32_t batch, void* stream) {
    if (!ctx || !path || !n_accept) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || ctx->opt_replay) return KVS_ERR_STATE;
    if (n_draft < 1 || n_draft > kvs::kTreeMaxTokens || path_stride < 1) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)path % 4) != 0) return KVS_ERR_INVALID_ARG;
    if (ctx->cur_batch == 0) return KVS_ERR_STATE;
    if (batch != ctx->cur_batch) return KVS_ERR_INVALID_ARG;
    bool same = true;
    for (int b = 0; b < batch; ++b) {
        if (n_accept[b] < 0 || n_accept[b] > n_draft || n_accept[b] > path_stride) return KVS_ERR_INVALID_ARG;
        same = same && n_accept[b] == n_accept[0];
    }
    const int Hkv = ctx->cfg.n_kv_heads, units = batch * Hkv;
    for (int s = 0; s < ctx->n_slots; ++s) {
        if (!holds_rows(ctx, s, batch, n_draft)) return KVS_ERR_STATE;
        // a slot whose units differ in length has none that is empty
        if (!same || ctx->ragged[s])
            for (int u = 0; u < units; ++u)
                if (unit_rows(ctx, s, u) - n_draft + n_accept[u / Hkv] < 1) return KVS_ERR_INVALID_ARG;
    }
    // the lengths of the slots whose units will differ, before anything is launched
    std::vector<std::vector<int32_t>> lens;
    try {
        lens.resize(ctx->n_slots);
        for (int s = 0; s < ctx->n_slots; ++s) {
            if (same && !ctx->ragged[s]) continue;
            lens[s].assign((size_t)ctx->cfg.max_batch * Hkv, 0);
            for (int u = 0; u < units; ++u) lens[s][u] = unit_rows(ctx, s, u) - n_draft + n_accept[u / Hkv];
        }
    } catch (const std::bad_alloc&) {
        return KVS_ERR_OOM;
    }
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    bool empty = true;
    for (int s = 0; s < ctx->n_slots; ++s) {
        const bool was = ctx->ragged[s] != 0, becomes = !lens[s].empty();
        char* kp = ctx->pool + (size_t)(2 * s) * ctx->plane_bytes;
        for (int b0 = 0; b0 < batch; b0 += kvs::AcceptCounts::kMax) {
            const int seqs = std::min(batch - b0, (int)kvs::AcceptCounts::kMax);
            kvs::AcceptCounts counts;
            for (int i = 0; i < seqs; ++i) counts.n[i] = (unsigned char)n_accept[b0 + i];
            if (kvs::launch_accept(kp, kp + ctx->plane_bytes, path, path_stride, counts, b0, seqs, Hkv, n_draft,
                                   was ? -1 : ctx->slot_len[s], becomes ? unit_len_dev(ctx, s) : nullptr, becomes, ctx->row_bytes,
                                   ctx->row_stride, reinterpret_cast<int*>(ctx->ws + ctx->off_status),
                                   (long long)ctx->plane_bytes, take_early_start(ctx), static_cast<cudaStream_t>(stream)) != cudaSuccess)
                return KVS_ERR_CUDA;
            ctx->seq += 1;
        }
        if (becomes) {
            ctx->unit_len_host[s].swap(lens[s]);
            ctx->ragged[s] = 1;
            ctx->slot_len[s] = *std::max_element(ctx->unit_len_host[s].begin(), ctx->unit_len_host[s].begin() + units);
        } else {
            ctx->slot_len[s] += n_accept[0] - n_draft;
        }
        empty = empty && ctx->slot_len[s] == 0;
        rows_moved(ctx, s);
    }
    if (empty) ctx->cur_batch = 0;
    ctx->stats.evict_launches += 1;
    return KVS_OK;
}

kvs_status kvs_decode_attention_weights(kvs_ctx* ctx, int32_t layer, const void* q, float* out, const float* total_in,
                                        float* total_out, int32_t total_stride, int32_t batch, void* stream) {
    kvs_status s = check_attention(ctx, layer, q, out, batch);
    if (s != KVS_OK) return s;
    if (ctx->format == KVS_CACHE_4BIT) return KVS_ERR_STATE;
    if (!total_out || ((uintptr_t)total_in % 4) != 0 || ((uintptr_t)total_out % 4) != 0) return KVS_ERR_INVALID_ARG;
    // a recorded launch grows on the device: its totals need room for every row the slot can hold
    if (total_stride < (ctx->opt_replay ? ctx->cfg.max_seq : ctx->slot_len[ctx->slot_of_layer[layer]])) return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    WeightTotals totals = {total_in, total_out, total_stride, 0};
    return do_attention(ctx, layer, q, out, batch, static_cast<cudaStream_t>(stream), &totals);
}

kvs_status kvs_select_rows(kvs_ctx* ctx, int32_t layer, const float* total, int32_t total_stride, const int32_t* n_keep,
                           int32_t n_recent, int32_t* keep, float* kept_total, int32_t keep_stride, int32_t batch, void* stream) {
    if (!ctx || !total || !n_keep || !keep) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || ctx->opt_replay) return KVS_ERR_STATE;
    if (layer < 0 || layer >= ctx->cfg.n_layers || n_recent < 0 || keep_stride < 1) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)total % 4) != 0 || ((uintptr_t)keep % 4) != 0 || ((uintptr_t)kept_total % 4) != 0) return KVS_ERR_INVALID_ARG;
    const int slot = ctx->slot_of_layer[layer];
    if (ctx->slot_len[slot] == 0) return KVS_ERR_STATE;
    if (batch < 1 || batch > ctx->cur_batch || total_stride < ctx->slot_len[slot]) return KVS_ERR_INVALID_ARG;
    const int units = batch * ctx->cfg.n_kv_heads;
    for (int u = 0; u < units; ++u)
        if (n_keep[u] < 1 || n_keep[u] > unit_rows(ctx, slot, u) || n_keep[u] < n_recent || n_keep[u] > keep_stride)
            return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    kvs::SelectArgs a;
    a.total = total;
    a.keep = keep;
    a.kept = kept_total;
    a.total_stride = total_stride;
    a.keep_stride = keep_stride;
    a.n = ctx->slot_len[slot];
    a.unit_len = ctx->ragged[slot] ? unit_len_dev(ctx, slot) : nullptr;
    a.n_recent = n_recent;
    a.sm_count = ctx->sm_count;
    a.status = reinterpret_cast<int*>(ctx->ws + ctx->off_status);
    for (int u0 = 0; u0 < units; u0 += kvs::SelectCounts::kMax) {
        a.unit0 = u0;
        a.units = std::min(units - u0, (int)kvs::SelectCounts::kMax);
        kvs::SelectCounts counts;
        for (int i = 0; i < a.units; ++i) counts.n[i] = n_keep[u0 + i];
        if (kvs::launch_select(a, counts, static_cast<cudaStream_t>(stream)) != cudaSuccess) return KVS_ERR_CUDA;
        ctx->seq += 1;
    }
    ctx->last_splitk_seq = ctx->seq;   // plain launches: everything before them has finished when they run
    ctx->counter_written = false;
    return KVS_OK;
}

kvs_status kvs_read_rows(kvs_ctx* ctx, int32_t layer, int32_t first, int32_t n_rows, void* k_out, void* v_out, int32_t batch, void* stream) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    if (layer < 0 || layer >= ctx->cfg.n_layers || !k_out || !v_out || first < 0 || n_rows < 1) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)k_out % 16) != 0 || ((uintptr_t)v_out % 16) != 0) return KVS_ERR_INVALID_ARG;
    const int slot = ctx->slot_of_layer[layer];
    if (ctx->slot_len[slot] == 0) return KVS_ERR_STATE;
    if (batch < 1 || batch > ctx->cur_batch || (long long)first + n_rows > ctx->slot_len[slot]) return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    const long long D = ctx->cfg.head_dim, token = ctx->cfg.n_kv_heads * D;
    kvs::ReadArgs r = {};
    r.kplane = ctx->pool + (size_t)(2 * slot) * ctx->plane_bytes;
    r.vplane = static_cast<const char*>(r.kplane) + ctx->plane_bytes;
    r.packed = ctx->format == KVS_CACHE_4BIT;
    r.row_stride = ctx->row_stride;
    r.first = first;
    r.n = n_rows;
    r.unit_len = ctx->ragged[slot] ? unit_len_dev(ctx, slot) : nullptr;
    r.k_out = k_out;
    r.v_out = v_out;
    r.dst_b = n_rows * token;
    r.dst_t = token;
    r.dst_h = D;
    r.batch = batch;
    r.Hkv = ctx->cfg.n_kv_heads;
    r.D = ctx->cfg.head_dim;
    r.dtype = ctx->cfg.dtype;
    r.status = reinterpret_cast<int*>(ctx->ws + ctx->off_status);
    r.plane_bytes = (long long)ctx->plane_bytes;
    r.sm_count = ctx->sm_count;
    r.programmatic = take_early_start(ctx);
    if (kvs::launch_read_rows(r, static_cast<cudaStream_t>(stream)) != cudaSuccess) return KVS_ERR_CUDA;
    ctx->seq += 1;
    return KVS_OK;
}

kvs_status kvs_beam_select(kvs_ctx* ctx, const void* logits, int32_t logits_dtype, int64_t logits_stride, int32_t vocab, const float* scores,
                           int32_t n_requests, int32_t n_beams, int32_t n_out, float* out_scores, int32_t* out_tokens,
                           int32_t* out_parents, void* stream) {
    if (!ctx || !logits || !scores || !out_scores || !out_tokens || !out_parents) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    if (logits_dtype != KVS_BF16 && logits_dtype != KVS_F32) return KVS_ERR_INVALID_ARG;
    if (vocab < 1 || logits_stride < vocab || n_requests < 1 || n_beams < 1 || n_beams > kvs::kBeamMaxBeams || n_out < 1 ||
        n_out > kvs::kBeamMaxOut)
        return KVS_ERR_INVALID_ARG;
    if ((long long)n_requests * n_beams > ctx->cfg.max_batch || (long long)n_beams * vocab > 0x7fffffffll) return KVS_ERR_INVALID_ARG;
    if (n_requests * n_beams > 65535) return KVS_ERR_INVALID_ARG;      // a grid dimension
    if (((uintptr_t)logits % (logits_dtype == KVS_BF16 ? 2 : 4)) != 0 || ((uintptr_t)scores % 4) != 0 || ((uintptr_t)out_scores % 4) != 0 ||
        ((uintptr_t)out_tokens % 4) != 0 || ((uintptr_t)out_parents % 4) != 0)
        return KVS_ERR_INVALID_ARG;
    if (scores == out_scores) return KVS_ERR_INVALID_ARG;      // one request's result would overwrite another's scores
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    kvs::BeamArgs b = {};
    b.logits = logits;
    b.stride = logits_stride;
    b.vocab = vocab;
    b.dtype = logits_dtype;
    b.scores = scores;
    b.requests = n_requests;
    b.beams = n_beams;
    b.n_out = n_out;
    b.out_scores = out_scores;
    b.out_tokens = out_tokens;
    b.out_parents = out_parents;
    b.scratch = ctx->ws + ctx->off_search;
    b.status = reinterpret_cast<int*>(ctx->ws + ctx->off_status);
    b.sm_count = ctx->sm_count;
    b.programmatic = take_early_start(ctx);
    if (kvs::launch_beam_select(b, static_cast<cudaStream_t>(stream)) != cudaSuccess) return KVS_ERR_CUDA;
    ctx->seq += 2;
    return KVS_OK;
}

kvs_status kvs_reorder(kvs_ctx* ctx, const int32_t* parent, int32_t first_row, int32_t batch, void* stream) {
    if (!ctx || !parent) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    if (batch < 1 || batch > ctx->cfg.max_batch || first_row < 0 || ((uintptr_t)parent % 4) != 0) return KVS_ERR_INVALID_ARG;
    if (ctx->cur_batch == 0) return KVS_ERR_STATE;
    // a recorded step keeps its batch; sequences the batch gains have no rows before first_row yet
    if (batch != ctx->cur_batch && ctx->opt_replay) return KVS_ERR_STATE;
    if (batch > ctx->cur_batch && first_row != 0) return KVS_ERR_INVALID_ARG;
    if (batch > kvs::kReorderMaxBatch || ctx->cur_batch > kvs::kReorderMaxBatch) return KVS_ERR_INVALID_ARG;
    for (int s = 0; s < ctx->n_slots; ++s)
        if (ctx->ragged[s]) return KVS_ERR_STATE;      // whose lengths go with which sequence only the device knows
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    kvs::ReorderArgs r = {};
    r.parent = parent;
    r.plane_bytes = (long long)ctx->plane_bytes;
    r.Hkv = ctx->cfg.n_kv_heads;
    r.row_bytes = ctx->row_bytes;
    r.row_stride = ctx->row_stride;
    r.first = first_row;
    r.capacity = ctx->cfg.max_seq;
    r.old_batch = ctx->cur_batch;
    r.new_batch = batch;
    r.n_extra = replay_counter(ctx);
    r.status = reinterpret_cast<int*>(ctx->ws + ctx->off_status);
    r.wait_ns = 1000ull * (unsigned long long)ctx->opt_wait_us;
    r.sm_count = ctx->sm_count;
    for (int s0 = 0; s0 < ctx->n_slots; s0 += kvs::ReorderRows::kMax) {
        r.pool = ctx->pool + (size_t)(2 * s0) * ctx->plane_bytes;
        r.slots = std::min(ctx->n_slots - s0, (int)kvs::ReorderRows::kMax);
        r.programmatic = take_early_start(ctx);
        kvs::ReorderRows rows = {};
        for (int s = 0; s < r.slots; ++s) rows.n[s] = ctx->slot_len[s0 + s];
        if (kvs::launch_reorder(r, rows, static_cast<cudaStream_t>(stream)) != cudaSuccess) return KVS_ERR_CUDA;
        ctx->seq += 1;
    }
    for (int s = 0; s < ctx->n_slots; ++s) rows_moved(ctx, s);
    ctx->cur_batch = batch;
    return KVS_OK;
}

kvs_status kvs_unit_len(const kvs_ctx* ctx, int32_t layer, int32_t b, int32_t h, int32_t* len) {
    if (!ctx || !len || layer < 0 || layer >= ctx->cfg.n_layers) return KVS_ERR_INVALID_ARG;
    if (b < 0 || b >= ctx->cfg.max_batch || h < 0 || h >= ctx->cfg.n_kv_heads) return KVS_ERR_INVALID_ARG;
    const int slot = ctx->slot_of_layer[layer];
    *len = ctx->ragged[slot] ? ctx->unit_len_host[slot][(size_t)b * ctx->cfg.n_kv_heads + h]
                             : (b < ctx->cur_batch ? ctx->slot_len[slot] : 0);
    return KVS_OK;
}

kvs_status kvs_layer_distances(kvs_ctx* ctx, int32_t batch, float* dist, void* stream) {
    if (!ctx || !dist) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || ctx->format == KVS_CACHE_4BIT) return KVS_ERR_STATE;
    if (ctx->cfg.n_layers > kvs::kMaxLayersSearch) return KVS_ERR_INVALID_ARG;
    if (batch < 1 || batch > ctx->cur_batch) return ctx->cur_batch == 0 ? KVS_ERR_STATE : KVS_ERR_INVALID_ARG;
    const int n = ctx->slot_len[0];
    if (n == 0) return KVS_ERR_STATE;
    for (int s = 0; s < ctx->n_slots; ++s)
        if (ctx->slot_len[s] != n || ctx->ragged[s]) return KVS_ERR_STATE;   // equally long, un-evicted caches only
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    {
        // not recorded into graphs: the launch pattern (programmatic dependents between plain launches) is
        // only exercised on a live stream
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(static_cast<cudaStream_t>(stream), &cap) != cudaSuccess) return KVS_ERR_CUDA;
        if (cap != cudaStreamCaptureStatusNone) return KVS_ERR_STATE;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int launches = 0;
    if (kvs::launch_layer_distances(ctx->pool, (long long)ctx->plane_bytes, ctx->slot_of_layer.data(), ctx->cfg.n_layers,
                                    ctx->n_slots, batch, ctx->cfg.n_kv_heads, n, ctx->row_stride, ctx->cfg.head_dim,
                                    ctx->cfg.dtype, reinterpret_cast<float*>(ctx->ws + ctx->off_search), ctx->search_bytes,
                                    dist, ctx->sm_count, &launches, st) != cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->seq += launches;
    ctx->last_splitk_seq = ctx->seq;     // the first and the last launches are plain: everything before them has finished
    ctx->stats.search_launches += launches;
    ctx->counter_written = false;   // a plain launch: full dependency on everything before it
    return KVS_OK;
}

kvs_status kvs_mean_cosine(kvs_ctx* ctx, const void* a, const void* b, int32_t n_samples, int64_t dim, float* out,
                           void* stream) {
    if (!ctx || !a || !b || !out) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    if (n_samples < 1 || dim < 2 || (dim & 1) != 0) return KVS_ERR_INVALID_ARG;
    if (((uintptr_t)a % 8) != 0 || ((uintptr_t)b % 8) != 0) return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    if (kvs::launch_mean_cosine(a, b, n_samples, dim, ctx->cfg.dtype, reinterpret_cast<double*>(ctx->ws + ctx->off_search),
                                out, ctx->sm_count, static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->seq += 2;
    ctx->last_splitk_seq = ctx->seq;
    ctx->stats.search_launches += 2;
    ctx->counter_written = false;   // a plain launch: full dependency on everything before it
    return KVS_OK;
}

kvs_status kvs_replay_advance(kvs_ctx* ctx, void* stream) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || !ctx->opt_replay) return KVS_ERR_STATE;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    // Outside stream capture the host lengths already advance with every call, so there is nothing
    // to count: the same step function can be run eagerly and recorded.
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(static_cast<cudaStream_t>(stream), &cap) != cudaSuccess) return KVS_ERR_CUDA;
    if (cap != cudaStreamCaptureStatusActive) return KVS_OK;
    if (kvs::launch_replay_advance(reinterpret_cast<int*>(ctx->ws + ctx->off_replay), ctx->opt_pdl != 0,
                                   static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->seq += 1;
    ctx->counter_written = true;
    return KVS_OK;
}

kvs_status kvs_replay_commit(kvs_ctx* ctx, int32_t times_run, void* stream) {
    if (!ctx || times_run < 1) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || !ctx->opt_replay) return KVS_ERR_STATE;
    const int extra = times_run - 1;     // the recording itself was already counted once
    for (int s = 0; s < ctx->n_slots; ++s)
        if (ctx->slot_len[s] > 0 && (long long)ctx->slot_len[s] + extra > ctx->cfg.max_seq) return KVS_ERR_CAPACITY;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    if (cudaMemsetAsync(ctx->ws + ctx->off_replay, 0, sizeof(int), static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->counter_written = true;
    for (int s = 0; s < ctx->n_slots; ++s) {
        if (ctx->slot_len[s] == 0) continue;
        ctx->slot_len[s] += extra;
        if (ctx->ragged[s])
            for (int u = 0; u < ctx->cur_batch * ctx->cfg.n_kv_heads; ++u) ctx->unit_len_host[s][u] += extra;
    }
    return KVS_OK;
}

kvs_status kvs_step_host(kvs_ctx* ctx, const void* q_host, const void* k_host, const void* v_host, float* out_host,
                         int32_t batch, void* stream, uint64_t* h2d_bytes, uint64_t* d2h_bytes) {
    if (!ctx || !q_host || !k_host || !v_host || !out_host) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    const kvs_config& f = ctx->cfg;
    if (batch < 1 || batch > f.max_batch) return KVS_ERR_INVALID_ARG;
    if (ctx->cur_batch != 0 && batch != ctx->cur_batch) return KVS_ERR_INVALID_ARG;
    // every own-cache slot grows by one token; check all capacities before any work
    for (int sl = 0; sl < ctx->n_slots; ++sl)
        if (ctx->slot_len[sl] + 1 > f.max_seq) return KVS_ERR_CAPACITY;
    DeviceGuard guard(f.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t q_layer = (size_t)batch * f.n_q_heads * f.head_dim * ctx->elem;
    const size_t kv_layer = (size_t)batch * f.n_kv_heads * f.head_dim * ctx->elem;
    const size_t out_layer = (size_t)batch * f.n_q_heads * f.head_dim * sizeof(float);
    char* dq = ctx->ws + ctx->off_stage_q;
    char* dk = ctx->ws + ctx->off_stage_k;
    char* dv = ctx->ws + ctx->off_stage_v;
    char* dout = ctx->ws + ctx->off_stage_out;
    uint64_t h2d = 0;
    // The layers are cut into chunks; one extra stream copies chunk c+1's inputs in and another copies
    // chunk c-1's outputs out while chunk c computes, so only the first input copy and the last
    // output copy are exposed.  Chunk c+1's copies are queued before chunk c's kernels so that the
    // host never stands between the device and its next piece of work.
    if (!ctx->copy_ready) {
        if (cudaStreamCreateWithFlags(&ctx->copy_stream, cudaStreamNonBlocking) != cudaSuccess ||
            cudaStreamCreateWithFlags(&ctx->out_stream, cudaStreamNonBlocking) != cudaSuccess)
            return KVS_ERR_CUDA;
        for (int i = 0; i < kvs_ctx::kChunks; ++i)
            if (cudaEventCreateWithFlags(&ctx->ev_in[i], cudaEventDisableTiming) != cudaSuccess ||
                cudaEventCreateWithFlags(&ctx->ev_done[i], cudaEventDisableTiming) != cudaSuccess)
                return KVS_ERR_CUDA;
        if (cudaEventCreateWithFlags(&ctx->ev_start, cudaEventDisableTiming) != cudaSuccess) return KVS_ERR_CUDA;
        ctx->copy_ready = true;
    }
    cudaStream_t cs = ctx->copy_stream, os = ctx->out_stream;
    const int L = f.n_layers;
    const int chunks = L < ctx->opt_host_chunks ? L : ctx->opt_host_chunks;
    // the copy streams start after whatever the caller already queued on `st`
    if (cudaEventRecord(ctx->ev_start, st) != cudaSuccess || cudaStreamWaitEvent(cs, ctx->ev_start, 0) != cudaSuccess ||
        cudaStreamWaitEvent(os, ctx->ev_start, 0) != cudaSuccess)
        return KVS_ERR_CUDA;
    // Chunk c covers layers [edge(c), edge(c+1)).  With three or more chunks the first and the last are
    // a single layer, so that the input copy nothing can hide and the output copy nothing can hide
    // are as small as they can be; the layers between are cut evenly.
    auto edge = [&](int c) -> int {
        if (chunks < 3 || L < chunks + 2) return (int)((long long)c * L / chunks);
        if (c == 0) return 0;
        if (c == chunks) return L;
        return 1 + (int)((long long)(c - 1) * (L - 2) / (chunks - 2));
    };
    auto copy_in = [&](int c) -> bool {
        const int l0 = edge(c), l1 = edge(c + 1);
        if (cudaMemcpyAsync(dq + q_layer * l0, (const char*)q_host + q_layer * l0, q_layer * (l1 - l0),
                            cudaMemcpyHostToDevice, cs) != cudaSuccess)
            return false;
        h2d += q_layer * (l1 - l0);
        // K/V of own-cache layers only; consecutive own-cache layers go in one copy
        for (int l = l0; l < l1;) {
            if (ctx->share_map[l] != l) { ++l; continue; }
            int e = l;
            while (e + 1 < l1 && ctx->share_map[e + 1] == e + 1) ++e;
            const size_t off = kv_layer * l, len = kv_layer * (e - l + 1);
            if (cudaMemcpyAsync(dk + off, (const char*)k_host + off, len, cudaMemcpyHostToDevice, cs) != cudaSuccess ||
                cudaMemcpyAsync(dv + off, (const char*)v_host + off, len, cudaMemcpyHostToDevice, cs) != cudaSuccess)
                return false;
            h2d += 2 * len;
            l = e + 1;
        }
        return cudaEventRecord(ctx->ev_in[c], cs) == cudaSuccess;
    };
    if (!copy_in(0)) return KVS_ERR_CUDA;
    for (int c = 0; c < chunks; ++c) {
        const int l0 = edge(c), l1 = edge(c + 1);
        if (c + 1 < chunks && !copy_in(c + 1)) return KVS_ERR_CUDA;
        if (cudaStreamWaitEvent(st, ctx->ev_in[c], 0) != cudaSuccess) return KVS_ERR_CUDA;
        for (int l = l0; l < l1; ++l) {
            float* o = reinterpret_cast<float*>(dout + out_layer * l);
            kvs_status s;
            if (ctx->share_map[l] == l && can_fuse_append(ctx, ctx->slot_of_layer[l])) {
                // the append rides in the split-K kernel (the staging rows are 16-byte aligned)
                s = do_fused_step(ctx, l, dq + q_layer * l, dk + kv_layer * l, dv + kv_layer * l, o, batch, st);
            } else {
                if (ctx->share_map[l] == l) {
                    s = do_append(ctx, l, dk + kv_layer * l, dv + kv_layer * l, batch, 1, st);
                    if (s != KVS_OK) return s;
                } else {
                    ctx->stats.append_skipped += 1;
                }
                s = do_attention(ctx, l, dq + q_layer * l, o, batch, st);
            }
            if (s != KVS_OK) return s;
        }
        if (cudaEventRecord(ctx->ev_done[c], st) != cudaSuccess || cudaStreamWaitEvent(os, ctx->ev_done[c], 0) != cudaSuccess)
            return KVS_ERR_CUDA;
        if (cudaMemcpyAsync((char*)out_host + out_layer * l0, dout + out_layer * l0, out_layer * (l1 - l0),
                            cudaMemcpyDeviceToHost, os) != cudaSuccess)
            return KVS_ERR_CUDA;
    }
    if (cudaStreamSynchronize(os) != cudaSuccess || cudaStreamSynchronize(cs) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return KVS_ERR_CUDA;
    if (h2d_bytes) *h2d_bytes = h2d;
    if (d2h_bytes) *d2h_bytes = out_layer * f.n_layers;
    return KVS_OK;
}

kvs_status kvs_num_slots(const kvs_ctx* ctx, int32_t* n_slots) {
    if (!ctx || !n_slots) return KVS_ERR_INVALID_ARG;
    *n_slots = ctx->n_slots;
    return KVS_OK;
}

kvs_status kvs_slot_of_layer(const kvs_ctx* ctx, int32_t layer, int32_t* slot) {
    if (!ctx || !slot || layer < 0 || layer >= ctx->cfg.n_layers) return KVS_ERR_INVALID_ARG;
    *slot = ctx->slot_of_layer[layer];
    return KVS_OK;
}

kvs_status kvs_seq_len(const kvs_ctx* ctx, int32_t layer, int32_t* len) {
    if (!ctx || !len || layer < 0 || layer >= ctx->cfg.n_layers) return KVS_ERR_INVALID_ARG;
    *len = ctx->slot_len[ctx->slot_of_layer[layer]];
    return KVS_OK;
}

kvs_status kvs_cached_batch(const kvs_ctx* ctx, int32_t* batch) {
    if (!ctx || !batch) return KVS_ERR_INVALID_ARG;
    *batch = ctx->cur_batch;
    return KVS_OK;
}

kvs_status kvs_row_stride(const kvs_ctx* ctx, int32_t* rows) {
    if (!ctx || !rows) return KVS_ERR_INVALID_ARG;
    *rows = ctx->row_stride;
    return KVS_OK;
}

kvs_status kvs_plane_offset(const kvs_ctx* ctx, int32_t slot, int32_t kv, size_t* offset) {
    if (!ctx || !offset || slot < 0 || slot >= ctx->n_slots || (kv != 0 && kv != 1)) return KVS_ERR_INVALID_ARG;
    *offset = (size_t)(2 * slot + kv) * ctx->plane_bytes;
    return KVS_OK;
}

kvs_status kvs_stats(const kvs_ctx* ctx, kvs_stats_t* stats) {
    if (!ctx || !stats) return KVS_ERR_INVALID_ARG;
    *stats = ctx->stats;
    return KVS_OK;
}

kvs_status kvs_last_device_status(kvs_ctx* ctx, int32_t* device_status) {
    if (!ctx || !device_status) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    int v = 0;
    if (cudaMemcpy(&v, ctx->ws + ctx->off_status, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess)
        return KVS_ERR_CUDA;
    *device_status = v;
    return KVS_OK;
}

kvs_status kvs_clear_device_status(kvs_ctx* ctx, void* stream) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // a launch that gave up may have left hand-over flags raised: they go back to zero with the status word
    if (cudaMemsetAsync(ctx->ws + ctx->off_status, 0, sizeof(int), st) != cudaSuccess ||
        cudaMemsetAsync(ctx->ws + ctx->off_flags, 0, sizeof(int32_t) * ctx->cfg.max_batch * ctx->cfg.n_kv_heads, st) !=
            cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->counter_written = true;   // the next launch takes a full dependency: it starts with the clears done
    return KVS_OK;
}

kvs_status kvs_selftest_stalled_copy(kvs_ctx* ctx, int32_t layer, const void* q, float* out, int32_t batch, void* stream) {
    kvs_status s = check_attention(ctx, layer, q, out, batch);
    if (s != KVS_OK) return s;
    if (ctx->format == KVS_CACHE_4BIT && ctx->cfg.dtype == KVS_F32) return KVS_ERR_STATE;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    const int slot = ctx->slot_of_layer[layer];
    kvs::DecodePlan plan;
    choose_plan(ctx, batch * ctx->cfg.n_kv_heads, ctx->slot_len[slot], &plan);
    ctx->stall_tile = plan.T / 2;          // a tile in the middle of the line
    ctx->counter_written = true;           // a plain launch, and so is whatever follows it
    s = do_attention(ctx, layer, q, out, batch, static_cast<cudaStream_t>(stream));
    ctx->stall_tile = -1;
    ctx->counter_written = true;
    return s;
}

kvs_status kvs_selftest_wait_timeout(kvs_ctx* ctx, uint32_t limit_us, uint64_t* waited_ns, void* stream) {
    if (!ctx || limit_us < 1 || limit_us > 1000000u) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound) return KVS_ERR_STATE;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // the measured wait goes to a spare word of the status block (128 bytes after the status word)
    unsigned long long* waited_dev = reinterpret_cast<unsigned long long*>(ctx->ws + ctx->off_status + 128);
    if (kvs::launch_wait_timeout_selftest(reinterpret_cast<int*>(ctx->ws + ctx->off_status), 1000ull * limit_us, waited_dev,
                                          st) != cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->seq += 1;
    ctx->last_splitk_seq = ctx->seq;   // a plain launch: everything before it has finished when it runs
    ctx->counter_written = false;
    unsigned long long w = 0;
    if (cudaMemcpyAsync(&w, waited_dev, sizeof(w), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return KVS_ERR_CUDA;
    if (waited_ns) *waited_ns = w;
    return KVS_OK;
}

kvs_status kvs_trace_begin(kvs_ctx* ctx, void* buffer, size_t bytes) {
    if (!ctx || !buffer || ((uintptr_t)buffer % 8) != 0) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || !kvs::is_tracing_build()) return KVS_ERR_STATE;
    const size_t per_launch = (size_t)kvs::kTraceLaunchWords * sizeof(unsigned long long);
    if (bytes < per_launch) return KVS_ERR_INVALID_ARG;
    ctx->trace_buf = static_cast<unsigned long long*>(buffer);
    ctx->trace_capacity = (int)std::min<size_t>(bytes / per_launch, 1 << 20);
    ctx->trace_launch = 0;
    return KVS_OK;
}

kvs_status kvs_trace_end(kvs_ctx* ctx, int32_t* launches_recorded) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (launches_recorded) *launches_recorded = ctx->trace_launch;
    ctx->trace_buf = nullptr;
    ctx->trace_capacity = ctx->trace_launch = 0;
    return KVS_OK;
}

kvs_status kvs_selftest_bounds(kvs_ctx* ctx, void* stream) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    if (!ctx->bound || !kvs::is_bounds_checking_build()) return KVS_ERR_STATE;
    DeviceGuard guard(ctx->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    if (kvs::launch_bounds_selftest(reinterpret_cast<int*>(ctx->ws + ctx->off_status), static_cast<cudaStream_t>(stream)) !=
        cudaSuccess)
        return KVS_ERR_CUDA;
    ctx->seq += 1;
    ctx->last_splitk_seq = ctx->seq;   // a plain launch: everything before it has finished when it runs
    ctx->counter_written = false;
    return KVS_OK;
}

kvs_status kvs_set_option(kvs_ctx* ctx, int32_t option, int32_t value) {
    if (!ctx) return KVS_ERR_INVALID_ARG;
    switch (option) {
        case KVS_OPT_MAX_CTAS:
            if (value < 0 || value > kvs::kMaxCtas) return KVS_ERR_INVALID_ARG;
            ctx->opt_max_ctas = value;
            return KVS_OK;
        case KVS_OPT_EARLY_START:
            if (value != 0 && value != 1) return KVS_ERR_INVALID_ARG;
            ctx->opt_pdl = value;
            return KVS_OK;
        case KVS_OPT_REPLAY:
            if (value != 0 && value != 1) return KVS_ERR_INVALID_ARG;
            ctx->opt_replay = value;
            return KVS_OK;
        case KVS_OPT_HOST_CHUNKS:
            if (value < 1 || value > kvs_ctx::kChunks) return KVS_ERR_INVALID_ARG;
            ctx->opt_host_chunks = value;
            return KVS_OK;
        case KVS_OPT_WAIT_LIMIT_US:
            if (value < 100 || value > 10000000) return KVS_ERR_INVALID_ARG;
            ctx->opt_wait_us = value;
            return KVS_OK;
        case KVS_OPT_FINISH_IN_KERNEL:
            if (value != 0 && value != 1) return KVS_ERR_INVALID_ARG;
            ctx->opt_finish = value;
            return KVS_OK;
        case KVS_OPT_KERNEL:
            if (value < 0 || value > 2) return KVS_ERR_INVALID_ARG;
            if (value == 2 && ctx->cfg.dtype != KVS_BF16) return KVS_ERR_INVALID_ARG;  // tensor-core path is bf16 only
            if (value == 1 && ctx->G != 1 && ctx->G != 2 && ctx->G != 4 && ctx->G != 8)
                return KVS_ERR_INVALID_ARG;                                          // scalar path: groups of 1, 2, 4, 8
            ctx->opt_kernel = value;
            return KVS_OK;
        default:
            return KVS_ERR_INVALID_ARG;
    }
}

kvs_status kvs_last_launch(const kvs_ctx* ctx, int32_t* ctas, int32_t* tile_rows, int32_t* kernel) {
    if (!ctx || !ctas || !tile_rows || !kernel) return KVS_ERR_INVALID_ARG;
    *ctas = ctx->last_plan.NC;
    *tile_rows = ctx->last_plan.tile_rows;
    *kernel = ctx->last_plan.kernel;
    return KVS_OK;
}

const char* kvs_status_string(kvs_status s) {
    switch (s) {
        case KVS_OK: return "ok";
        case KVS_ERR_INVALID_ARG: return "invalid argument";
        case KVS_ERR_BAD_SHARE_MAP: return "bad share map";
        case KVS_ERR_STATE: return "call made in the wrong state";
        case KVS_ERR_CAPACITY: return "slot capacity exceeded";
        case KVS_ERR_OOM: return "bound buffer too small";
        case KVS_ERR_CUDA: return "CUDA call failed";
        case KVS_ERR_TIMEOUT: return "device-side wait timed out";
        case KVS_ERR_SCRATCH_LIMIT: return "call needs more scratch than the built-in scratch array holds";
        case KVS_ERR_BOUNDS: return "a bounds-checking build found an offset outside its buffer";
    }
    return "unknown status";
}

kvs_status kvs_read_roof(const void* src, size_t bytes, uint64_t* checksum, int32_t device, void* stream) {
    if (!src || !checksum || bytes == 0 || bytes % 32768 != 0 || device < 0 || device >= 64) return KVS_ERR_INVALID_ARG;
    DeviceGuard guard(device);
    if (!guard.ok) return KVS_ERR_CUDA;
    if (init_device_once(device) != cudaSuccess) return KVS_ERR_CUDA;
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return KVS_ERR_CUDA;
    if (kvs::launch_read_roof(src, bytes, reinterpret_cast<unsigned long long*>(checksum), sms,
                              static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return KVS_ERR_CUDA;
    return KVS_OK;
}

kvs_status kvs_decode_attention_static(kvs_ctx* ctx, int32_t layer, const void* q, float* out, int32_t batch,
                                       void* stream, int32_t* device_status) {
    kvs_status s = check_attention(ctx, layer, q, out, batch);
    if (s != KVS_OK) return s;
    if (((uintptr_t)device_status % 4) != 0) return KVS_ERR_INVALID_ARG;   // the kernels update it atomically
    kvs_ctx* c = ctx;
    const int slot = c->slot_of_layer[layer];
    const int units = batch * c->cfg.n_kv_heads;
    const int D = c->cfg.head_dim;
    kvs::DecodePlan plan;
    const bool use_mma = choose_plan(c, units, c->slot_len[slot], &plan);
    // one partial (o[D], m, l) per (piece, q-head); pieces are indexed unit + block
    const size_t pieces = (size_t)units + plan.NC;
    const size_t part_o_bytes = align_up(pieces * c->G * D * sizeof(float), kAlign);
    const size_t part_ml_bytes = align_up(pieces * c->G * 2 * sizeof(float), kAlign);
    const size_t flag_bytes = kStaticFlagBytes;
    if ((size_t)units * sizeof(int32_t) > kStaticFlagBytes ||
        kStaticStatusBytes + part_o_bytes + part_ml_bytes + flag_bytes > kStaticScratchBytes)
        return KVS_ERR_SCRATCH_LIMIT;

    DeviceGuard guard(c->cfg.device);
    if (!guard.ok) return KVS_ERR_CUDA;
    // the address was looked up when the context's memory was bound (per-device set-up): no
    // runtime query here
    unsigned char* base = g_static_ptr[c->cfg.device];
    if (g_static_err[c->cfg.device] != cudaSuccess || base == nullptr) return KVS_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int* status_word = device_status ? device_status : reinterpret_cast<int*>(base);
    // the array keeps whatever the previous call left; only the status word must start at zero
    if (cudaMemsetAsync(status_word, 0, sizeof(int), st) != cudaSuccess) return KVS_ERR_CUDA;
    // Plain launches: the kernels start after everything before them on `stream`.  The call may be
    // on another stream than the context's other calls, so it stays out of the bookkeeping that
    // decides what those calls may fetch early (untracked), and it leaves the "growth counter was
    // just written" mark for the next call of the chain.
    // layout: status word, flags (fixed size), partial outputs, partial (max, sum) pairs
    const AttentionScratch scratch = {reinterpret_cast<float*>(base + kStaticStatusBytes + flag_bytes),
                                      reinterpret_cast<float*>(base + kStaticStatusBytes + flag_bytes + part_o_bytes),
                                      reinterpret_cast<int*>(base + kStaticStatusBytes), status_word, false, false};
    return run_attention(c, slot, q, out, 0, batch * c->cfg.n_kv_heads, plan, use_mma, scratch, st);
}

}  // extern "C"
