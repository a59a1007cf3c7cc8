// Host side of the C ABI: context, validation, layout tables, launches.  No arithmetic of the
// method happens here; every step runs in the gfx950 kernels.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <mutex>
#include <new>
#include <vector>

#include "qgx_internal.h"
#include "qgx_plan.h"

using namespace qgx;

// Scratch of qgx_eg_step_static, the variant of qgx_eg_step for callers that may not allocate: the
// partial sums (two per chunk) of the step-size accumulator S, which qgx_eg_step keeps in memory that
// qgx_create allocated.  Every GPU the library runs on holds its own copy of the array, at its own
// address, until the process ends.  The name below is a host-side stand-in for it, not a device
// address: host code uses the address hipGetSymbolAddress gave for the device (static_scratch_of).
static __device__ __align__(256) double scratch[2 * QGX_STATIC_MAX_CHUNKS];

namespace {
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
double* g_scratch_ptr[kMaxDevices] = {nullptr};

// Address of `scratch` on `device`, which must be the current device; asked for once per device.
hipError_t static_scratch_of(int device, double** out)
{
    if (device < 0 || device >= kMaxDevices) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[device]) {
        void* p = nullptr;
        hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        if (!p) return hipErrorInvalidSymbol;
        g_scratch_ptr[device] = static_cast<double*>(p);
    }
    *out = g_scratch_ptr[device];
    return hipSuccess;
}
}  // namespace

// What the host knows of one of the context's level tables (the table itself lives on the device).
struct TableState {
    uint32_t n_sym = 0;
    uint32_t max_code_len = 0;      // longest code word of the code in use (without the sign bit)
    bool levels_set = false, code_set = false;
    bool wide = false;              // 11 bits identify every code word: the decoders may use the 8-byte table
    bool crowded = false;           // levels too close for the encoder's cells, as far as the host knows (not of fitted ones)
};

struct qgx_ctx {
    qgx_config cfg{};
    std::vector<uint64_t> seg;
    int device = 0;
    uint32_t rows = 0;               // of the longest bucket's last chunk, or with shared chunks of a bucket (columns_pay)
    uint32_t n_simd = 1024;          // SIMDs of the device (four per compute unit)
    int ksplit_forced = -1;          // qgx_debug_set_waves_per_position: 1, 2 or 4, else -1: by the rule
    Layout lay{};
    uint32_t* d_layout = nullptr;
    Tables* d_tabs = nullptr;        // [QGX_TABLES]
    TableState ts[QGX_TABLES];
    uint32_t sel = 0, sel_prev = 0;  // qgx_select_table
    Scalars* d_sc = nullptr;
    float* d_Y = nullptr;
    float* d_anchor = nullptr;
    unsigned long long* d_scan = nullptr;
    unsigned long long* d_xch = nullptr;   // partial norms of buckets shared by several workgroups
    uint32_t parts = 1;                    // workgroups per bucket in the encoder
    unsigned long long* d_tickets = nullptr;
    double* d_spartial = nullptr;
    double* d_static_scratch = nullptr;   // this device's copy of the file-scope scratch array (not owned)
    double* d_hpartial = nullptr;
    double* d_hist = nullptr;
    FitCodeResult* h_fit = nullptr;    // what the last qgx_fit_code left for the host: pinned memory, which the kernel writes (QGX_CODE_TABLE)
    FitCodeResult* d_fit = nullptr;    // the same as the device sees it
    double* d_norm = nullptr;       // [2 kNormBlocks + 2] partial sums and results of qgx_norm2 and qgx_game_gap
    double* d_metrics = nullptr;    // [K][3][kMetricBlocks] partial sums, then [K][3] results of qgx_quantization_metrics
    double* d_xsum = nullptr;       // [d] sum of the X_{t+1/2} since qgx_average_reset (allocated there)
    bool xsum_on = false;
    uint32_t hist_bins = 0;         // bins of the histogram d_hist holds (0: none yet)
    uint32_t h_groups = 0;
    bool state_ready = false, has_anchor = false;
    uint64_t worst_words = 0;
    char err[256] = "";
};

namespace {

qgx_status fail(qgx_ctx* ctx, qgx_status st, const char* fmt, ...)
{
    if (ctx) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
        va_end(ap);
    }
    return st;
}

#define QGX_HIP(ctx, call)                                                                             \
    do {                                                                                               \
        hipError_t e_ = (call);                                                                        \
        if (e_ != hipSuccess) return fail((ctx), QGX_ERR_HIP, "%s: %s", #call, hipGetErrorString(e_)); \
    } while (0)

// The same after an asynchronous copy into a local variable has been queued on `st`: the function may
// not return, and so end the variable's life, before the queue has drained.
#define QGX_HIP_DRAIN(ctx, st, call)                                                                   \
    do {                                                                                               \
        hipError_t e_ = (call);                                                                        \
        if (e_ != hipSuccess) {                                                                        \
            (void)hipStreamSynchronize(st);                                                            \
            return fail((ctx), QGX_ERR_HIP, "%s: %s", #call, hipGetErrorString(e_));                   \
        }                                                                                              \
    } while (0)

// Length of Elias' recursive (omega) code of N >= 1: one terminating bit plus every prefixed group.
uint32_t omega_length(uint32_t N)
{
    uint32_t len = 1;
    while (N > 1) {
        uint32_t nb = 0;
        for (uint32_t x = N; x; x >>= 1) ++nb;
        len += nb;
        N = nb - 1;
    }
    return len;
}

TableState& T(qgx_ctx* ctx) { return ctx->ts[ctx->sel]; }
const TableState& T(const qgx_ctx* ctx) { return ctx->ts[ctx->sel]; }
Tables* tab_of(const qgx_ctx* ctx) { return ctx->d_tabs + ctx->sel; }

// Do the first kWideBits bits of a code word always tell which one it is?  packed[j] = bits | length << 16,
// first-written bit in bit 0.  In a prefix-free code only two words that are both longer can agree there.
bool wide_table_ok(const uint32_t* packed, uint32_t n_sym)
{
    const uint32_t mask = (1u << kWideBits) - 1u;
    for (uint32_t i = 0; i < n_sym; ++i)
        for (uint32_t j = i + 1; j < n_sym; ++j)
            if ((packed[i] >> 16) > (uint32_t)kWideBits && (packed[j] >> 16) > (uint32_t)kWideBits &&
                ((packed[i] ^ packed[j]) & mask) == 0u)
                return false;
    return true;
}

// A kernel on the context's device may write doubles there.
bool writable_here(const qgx_ctx* ctx, const double* p)
{
    hipPointerAttribute_t at{};
    if ((reinterpret_cast<uintptr_t>(p) & 7u) != 0) return false;
    if (hipPointerGetAttributes(&at, p) != hipSuccess) { (void)hipGetLastError(); return false; }
    return at.type == hipMemoryTypeDevice && at.device == ctx->device;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

qgx_status check_stream(qgx_ctx* ctx, const qgx_stream* s, const char* what)
{
    if (!s || !s->norms || !s->chunk_off || !s->sub_end || !s->payload)
        return fail(ctx, QGX_ERR_ARG, "%s: null stream pointer", what);
    if (!aligned16(s->norms) || !aligned16(s->chunk_off) || !aligned16(s->sub_end) || !aligned16(s->payload))
        return fail(ctx, QGX_ERR_ARG, "%s: stream buffers must be 16-byte aligned", what);
    if (s->payload_words_per_worker == 0 || (s->payload_words_per_worker & 3u) ||
        s->payload_words_per_worker > 0xFFFFFFFFull)
        return fail(ctx, QGX_ERR_ARG, "%s: payload_words_per_worker must be a non-zero multiple of 4 below 2^32", what);
    if (s->slot_words & 3u) return fail(ctx, QGX_ERR_ARG, "%s: slot_words must be a multiple of 4", what);
    return QGX_OK;
}

// longest code word over the context's tables, so that streams of either share a slot size
uint32_t longest_code(const qgx_ctx* ctx)
{
    uint32_t m = 0;
    for (const TableState& t : ctx->ts) m = t.levels_set && t.max_code_len > m ? t.max_code_len : m;
    return m;
}

// most words a full chunk can take with the codes in use, multiple of 4
uint32_t chunk_slot_words(const qgx_ctx* ctx)
{
    const uint32_t words = (kChunk * (longest_code(ctx) + 1) + 31) / 32;
    return (words + 3) / 4 * 4;
}

qgx_status need_levels(qgx_ctx* ctx, uint32_t which)
{
    const TableState& t = ctx->ts[which];
    if (!t.levels_set) return fail(ctx, QGX_ERR_STATE, "level table %u not set", which);
    if (ctx->cfg.code == QGX_CODE_TABLE && !t.code_set) return fail(ctx, QGX_ERR_STATE, "code table %u not set", which);
    return QGX_OK;
}

qgx_status need_levels(qgx_ctx* ctx) { return need_levels(ctx, ctx->sel); }

void free_all(qgx_ctx* c)
{
    void* all[] = {c->d_layout, c->d_tabs, c->d_sc, c->d_Y, c->d_anchor, c->d_scan, c->d_xch, c->d_tickets, c->d_spartial, c->d_hpartial, c->d_hist, c->d_norm, c->d_metrics, c->d_xsum};
    for (void* p : all) (void)hipFree(p);
    if (c->h_fit) (void)hipHostFree(c->h_fit);
}

}  // namespace

extern "C" {

qgx_status qgx_create(qgx_ctx** out, const qgx_config* cfg)
{
    if (!out || !cfg) return QGX_ERR_ARG;
    *out = nullptr;
    if (cfg->d == 0 || cfg->d >= (1ull << 31) || cfg->K == 0 || cfg->K > 65535u) return QGX_ERR_ARG;
    if (cfg->bucket == 0 || (cfg->bucket & 3u) || cfg->bucket > QGX_MAX_BUCKET) return QGX_ERR_ARG;
    if (cfg->norm < 0 || cfg->norm > QGX_MAX_NORM_Q) return QGX_ERR_ARG;
    if (cfg->code != QGX_CODE_ELIAS_OMEGA && cfg->code != QGX_CODE_TABLE) return QGX_ERR_ARG;
    qgx_ctx* c = new (std::nothrow) qgx_ctx;
    if (!c) return QGX_ERR_ARG;
    c->cfg = *cfg;
    if (cfg->n_segments > 1) {
        if (!cfg->segment_len) { delete c; return QGX_ERR_ARG; }
        c->seg.assign(cfg->segment_len, cfg->segment_len + cfg->n_segments);
    } else {
        c->seg.assign(1, cfg->n_segments == 1 && cfg->segment_len ? cfg->segment_len[0] : cfg->d);
    }
    c->cfg.segment_len = nullptr;
    uint64_t sum = 0;
    for (size_t s = 0; s < c->seg.size(); ++s) {
        if (c->seg[s] == 0 || (s + 1 < c->seg.size() && (c->seg[s] & 3u))) { delete c; return QGX_ERR_ARG; }
        sum += c->seg[s];
    }
    if (sum != cfg->d) { delete c; return QGX_ERR_ARG; }

    // buckets and chunks of one worker
    std::vector<uint32_t> bstart, bchunk0, cstart, cbucket, tasks, ragged;
    uint64_t pos = 0, worst = 0;
    const bool shared = shares_chunks(cfg->bucket);
    auto add_chunk = [&](uint64_t start, uint64_t cl, uint32_t first_bucket) {
        const uint32_t first_half = 2u * (uint32_t)cstart.size();
        (cl >= (uint64_t)kChunk / 2 ? tasks : ragged).push_back(first_half);
        if (cl > (uint64_t)kChunk / 2) (cl == (uint64_t)kChunk ? tasks : ragged).push_back(first_half + 1u);
        cstart.push_back((uint32_t)start);
        cbucket.push_back(first_bucket);
        const uint64_t wds = (cl * kMaxSymBits + 31) / 32;
        worst += (wds + kAlignWords - 1) / kAlignWords * kAlignWords;
    };
    for (uint64_t len_s : c->seg) {
        uint64_t left = len_s;
        if (shared) {                                   // chunks are runs of the segment, each holding whole buckets
            for (uint64_t o = 0; o < len_s; o += kChunk)
                add_chunk(pos + o, (len_s - o) < (uint64_t)kChunk ? (len_s - o) : (uint64_t)kChunk,
                          (uint32_t)(bstart.size() + o / cfg->bucket));
        }
        while (left) {
            const uint64_t len = left < cfg->bucket ? left : cfg->bucket;
            bstart.push_back((uint32_t)pos);
            bchunk0.push_back((uint32_t)cstart.size());     // (not meaningful with shared chunks)
            if (!shared) {
                for (uint64_t o = 0; o < len; o += kChunk)
                    add_chunk(pos + o, (len - o) < (uint64_t)kChunk ? (len - o) : (uint64_t)kChunk,
                              (uint32_t)(bstart.size() - 1));
            }
            pos += len;
            left -= len;
        }
    }
    bstart.push_back((uint32_t)pos);
    bchunk0.push_back((uint32_t)cstart.size());
    cstart.push_back((uint32_t)pos);
    const uint32_t NB = (uint32_t)bstart.size() - 1, NC = (uint32_t)cbucket.size();
    if ((uint64_t)NB * cfg->K >= (1ull << 31) || (uint64_t)NC * cfg->K >= (1ull << 31)) { delete c; return QGX_ERR_ARG; }
    c->worst_words = worst;

    if (hipGetDevice(&c->device) != hipSuccess) { delete c; return QGX_ERR_HIP; }
    if (static_scratch_of(c->device, &c->d_static_scratch) != hipSuccess) { delete c; return QGX_ERR_HIP; }
    {
        int cus = 0;
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, c->device) == hipSuccess && cus > 0)
            c->n_simd = 4u * (uint32_t)cus;
    }
    const bool all_full = tasks.size() == 2 * (size_t)NC;      // then task t is half t & 1 of chunk t >> 1
    tasks.insert(tasks.end(), ragged.begin(), ragged.end());
    const size_t n_lay = (size_t)(NB + 1) * 2 + (NC + 1) + NC + (all_full ? 0 : tasks.size()) + 1;
    std::vector<uint32_t> flat;
    flat.reserve(n_lay);
    flat.insert(flat.end(), bstart.begin(), bstart.end());
    flat.insert(flat.end(), bchunk0.begin(), bchunk0.end());
    flat.insert(flat.end(), cstart.begin(), cstart.end());
    flat.insert(flat.end(), cbucket.begin(), cbucket.end());
    if (!all_full) flat.insert(flat.end(), tasks.begin(), tasks.end());
    flat.push_back(0u);

    c->lay.NB = NB; c->lay.NC = NC; c->lay.K = cfg->K; c->lay.d = (uint32_t)cfg->d;
    c->lay.n_tasks = (uint32_t)tasks.size();
    uint32_t max_len = 0;
    for (uint32_t b = 0; b < NB; ++b) max_len = bstart[b + 1] - bstart[b] > max_len ? bstart[b + 1] - bstart[b] : max_len;
    c->lay.waves_per_bucket = (max_len + kChunk - 1) / kChunk;
    c->rows = shared ? cfg->bucket / 256u : ((max_len - 1u) % (uint32_t)kChunk) / 256u + 1u;
    c->lay.uniform_bucket = (c->seg.size() == 1 && !shared) ? cfg->bucket : 0u;
    c->lay.shared_chunks = shared ? 1u : 0u;
    c->lay.bucket_shift = 31u;
    if (shared)
        for (c->lay.bucket_shift = 0; (1u << c->lay.bucket_shift) < cfg->bucket;) ++c->lay.bucket_shift;
    c->h_groups = histogram_groups(c->lay);

    bool ok = true;
    ok = ok && hipMalloc(&c->d_layout, n_lay * sizeof(uint32_t)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_tabs, QGX_TABLES * sizeof(Tables)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_sc, sizeof(Scalars)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_Y, cfg->d * sizeof(float)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_anchor, cfg->d * sizeof(float)) == hipSuccess;
    // A bucket of more than four chunks is shared by workgroups of four waves.  Per worker, the parts
    // of one bucket (the newest tickets) can be waiting for partners that have not started yet: up to
    // three, which must leave a place free on every XCD (see worker_span), so only for K <= 64.
    c->parts = (c->lay.waves_per_bucket > 4u && cfg->K <= 64u) ? (c->lay.waves_per_bucket + 3u) / 4u : 1u;
    const size_t n_units = (size_t)cfg->K * NB * c->parts;
    ok = ok && hipMalloc(&c->d_scan, n_units * sizeof(unsigned long long)) == hipSuccess;
    if (c->parts > 1u) {
        ok = ok && hipMalloc(&c->d_xch, n_units * 4 * sizeof(unsigned long long)) == hipSuccess;
        ok = ok && hipMemset(c->d_xch, 0, n_units * 4 * sizeof(unsigned long long)) == hipSuccess;
    }
    ok = ok && hipMalloc(&c->d_tickets, (size_t)cfg->K * kTicketStride * sizeof(unsigned long long)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_spartial, (size_t)c->lay.n_tasks * sizeof(double)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_hpartial, (size_t)c->h_groups * QGX_MAX_BINS * sizeof(double)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_hist, QGX_MAX_BINS * sizeof(double)) == hipSuccess;
    if (cfg->code == QGX_CODE_TABLE) {                     // (50 us, which a context without a fitted code is spared)
        ok = ok && hipHostMalloc(reinterpret_cast<void**>(&c->h_fit), sizeof(FitCodeResult), hipHostMallocMapped) == hipSuccess;
        ok = ok && hipHostGetDevicePointer(reinterpret_cast<void**>(&c->d_fit), c->h_fit, 0) == hipSuccess;
    }
    ok = ok && hipMalloc(&c->d_norm, (2 * kNormBlocks + 2) * sizeof(double)) == hipSuccess;
    ok = ok && hipMalloc(&c->d_metrics, (size_t)cfg->K * 3 * (kMetricBlocks + 1) * sizeof(double)) == hipSuccess;
    ok = ok && hipMemcpy(c->d_layout, flat.data(), n_lay * sizeof(uint32_t), hipMemcpyHostToDevice) == hipSuccess;
    ok = ok && hipMemset(c->d_tabs, 0, QGX_TABLES * sizeof(Tables)) == hipSuccess;
    ok = ok && hipMemset(c->d_sc, 0, sizeof(Scalars)) == hipSuccess;
    ok = ok && hipMemset(c->d_scan, 0, n_units * sizeof(unsigned long long)) == hipSuccess;
    ok = ok && hipMemset(c->d_tickets, 0, (size_t)cfg->K * kTicketStride * sizeof(unsigned long long)) == hipSuccess;
    if (ok) {
        const uint32_t kind = (uint32_t)cfg->code;
        for (int t = 0; ok && t < QGX_TABLES; ++t)
            ok = hipMemcpy(&c->d_tabs[t].code_kind, &kind, sizeof(kind), hipMemcpyHostToDevice) == hipSuccess;
    }
    ok = ok && hipDeviceSynchronize() == hipSuccess;
    if (!ok) { free_all(c); delete c; return QGX_ERR_HIP; }
    c->lay.bucket_start = c->d_layout;
    c->lay.bucket_chunk0 = c->d_layout + (NB + 1);
    c->lay.chunk_start = c->d_layout + 2 * (size_t)(NB + 1);
    c->lay.chunk_bucket = c->lay.chunk_start + (NC + 1);
    c->lay.task = all_full ? nullptr : c->lay.chunk_bucket + NC;
    *out = c;
    return QGX_OK;
}

void qgx_destroy(qgx_ctx* ctx)
{
    if (!ctx) return;
    (void)hipDeviceSynchronize();
    free_all(ctx);
    delete ctx;
}

qgx_status qgx_stream_sizes(const qgx_ctx* ctx, uint64_t* n_buckets, uint64_t* n_chunks,
                            uint64_t* worst_case_payload_words)
{
    if (!ctx) return QGX_ERR_ARG;
    if (n_buckets) *n_buckets = ctx->lay.NB;
    if (n_chunks) *n_chunks = ctx->lay.NC;
    if (worst_case_payload_words) *worst_case_payload_words = ctx->worst_words;
    return QGX_OK;
}

qgx_status qgx_slot_words(const qgx_ctx* ctx, uint64_t* slot_words)
{
    if (!ctx || !slot_words) return QGX_ERR_ARG;
    if (!T(ctx).levels_set || (ctx->cfg.code == QGX_CODE_TABLE && !T(ctx).code_set))
        return fail(const_cast<qgx_ctx*>(ctx), QGX_ERR_STATE,
                    "qgx_slot_words: the slot follows the longest code word: set the level table (and the code table) first");
    *slot_words = chunk_slot_words(ctx);
    return QGX_OK;
}

qgx_status qgx_compact(qgx_ctx* ctx, const qgx_stream* in, qgx_stream* out, void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    qgx_status s = check_stream(ctx, in, "qgx_compact(in)");
    if (s == QGX_OK) s = check_stream(ctx, out, "qgx_compact(out)");
    if (s != QGX_OK) return s;
    if (out->slot_words != 0) return fail(ctx, QGX_ERR_ARG, "qgx_compact: out must be a compact stream");
    if (in->payload == out->payload || in->chunk_off == out->chunk_off)
        return fail(ctx, QGX_ERR_ARG, "qgx_compact: in and out must not alias");
    hipStream_t st = (hipStream_t)stream;
    const Layout& lay = ctx->lay;
    if (in->norms != out->norms)
        QGX_HIP(ctx, hipMemcpyAsync(out->norms, in->norms, (size_t)lay.K * lay.NB * sizeof(float), hipMemcpyDeviceToDevice, st));
    if (in->sub_end != out->sub_end)
        QGX_HIP(ctx, hipMemcpyAsync(out->sub_end, in->sub_end, (size_t)lay.K * lay.NC * kSubs * sizeof(uint16_t),
                                    hipMemcpyDeviceToDevice, st));
    QGX_HIP(ctx, launch_compact(lay, in->sub_end, in->chunk_off, in->payload, in->payload_words_per_worker,
                                out->chunk_off, out->payload, out->payload_words_per_worker, ctx->d_sc, st));
    return QGX_OK;
}

qgx_status qgx_select_table(qgx_ctx* ctx, uint32_t table, uint32_t prev_table)
{
    if (!ctx) return QGX_ERR_ARG;
    if (table >= QGX_TABLES || prev_table >= QGX_TABLES)
        return fail(ctx, QGX_ERR_ARG, "qgx_select_table: a context has tables 0..%d", QGX_TABLES - 1);
    ctx->sel = table;
    ctx->sel_prev = prev_table;
    return QGX_OK;
}

qgx_status qgx_set_levels(qgx_ctx* ctx, const float* levels_host, uint32_t n_sym, void* stream)
{
    if (!ctx || !levels_host) return fail(ctx, QGX_ERR_ARG, "qgx_set_levels: null argument");
    if (n_sym < 2 || n_sym > QGX_MAX_SYM) return fail(ctx, QGX_ERR_ARG, "qgx_set_levels: n_sym out of range");
    if (levels_host[0] != 0.0f || levels_host[n_sym - 1] != 1.0f)
        return fail(ctx, QGX_ERR_LEVELS, "level table must start at 0 and end at 1");
    for (uint32_t j = 0; j + 1 < n_sym; ++j)
        if (!(levels_host[j] < levels_host[j + 1]))
            return fail(ctx, QGX_ERR_LEVELS, "level table not strictly increasing at %u", j);
    hipStream_t st = (hipStream_t)stream;
    if (ctx->cfg.code == QGX_CODE_TABLE && T(ctx).code_set && n_sym != T(ctx).n_sym) T(ctx).code_set = false;
    QGX_HIP(ctx, hipMemcpyAsync(tab_of(ctx)->levels, levels_host, n_sym * sizeof(float), hipMemcpyHostToDevice, st));
    QGX_HIP(ctx, hipMemcpyAsync(&tab_of(ctx)->n_sym, &n_sym, sizeof(n_sym), hipMemcpyHostToDevice, st));
    QGX_HIP(ctx, launch_build_tables(tab_of(ctx), st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    T(ctx).n_sym = n_sym;
    T(ctx).levels_set = true;
    T(ctx).crowded = levels_crowded(levels_host, n_sym, cell_mant(n_sym), kCellOct);
    if (ctx->cfg.code == QGX_CODE_ELIAS_OMEGA) {
        T(ctx).max_code_len = omega_length(n_sym);
        T(ctx).wide = n_sym <= 63u;     // the words of 1..63 differ within their first 11 bits, those of 64 and 65 do not
    }
    return QGX_OK;
}

qgx_status qgx_get_levels(qgx_ctx* ctx, float* levels_host, uint32_t* n_sym, void* stream)
{
    if (!ctx || !levels_host || !n_sym) return fail(ctx, QGX_ERR_ARG, "qgx_get_levels: null argument");
    if (!T(ctx).levels_set) return fail(ctx, QGX_ERR_STATE, "level table not set");
    hipStream_t st = (hipStream_t)stream;
    QGX_HIP(ctx, hipMemcpyAsync(levels_host, tab_of(ctx)->levels, T(ctx).n_sym * sizeof(float), hipMemcpyDeviceToHost, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    *n_sym = T(ctx).n_sym;
    return QGX_OK;
}

qgx_status qgx_set_code_table(qgx_ctx* ctx, const uint8_t* code_len, const uint32_t* code_bits, uint32_t n_sym,
                              void* stream)
{
    if (!ctx || !code_len || !code_bits) return fail(ctx, QGX_ERR_ARG, "qgx_set_code_table: null argument");
    if (ctx->cfg.code != QGX_CODE_TABLE) return fail(ctx, QGX_ERR_STATE, "context was not created with QGX_CODE_TABLE");
    if (!T(ctx).levels_set || n_sym != T(ctx).n_sym)
        return fail(ctx, QGX_ERR_STATE, "set the level table first; the code table must have as many entries");
    double kraft = 0.0;
    for (uint32_t j = 0; j < n_sym; ++j) {
        if (code_len[j] < 1 || code_len[j] > QGX_MAX_CODE_BITS || (code_bits[j] >> code_len[j]))
            return fail(ctx, QGX_ERR_ARG, "code word %u: length must be 1..13 and bits must fit it", j);
        kraft += std::ldexp(1.0, -(int)code_len[j]);
        for (uint32_t i = 0; i < j; ++i) {
            const uint32_t m = code_len[i] < code_len[j] ? code_len[i] : code_len[j];
            if (((code_bits[i] ^ code_bits[j]) & ((1u << m) - 1u)) == 0)
                return fail(ctx, QGX_ERR_ARG, "code words %u and %u: one is a prefix of the other", i, j);
        }
    }
    if (kraft > 1.0) return fail(ctx, QGX_ERR_ARG, "code table violates the Kraft inequality");
    uint32_t packed[kSymMax] = {0};
    for (uint32_t j = 0; j < n_sym; ++j) packed[j] = code_bits[j] | ((uint32_t)code_len[j] << 16);
    hipStream_t st = (hipStream_t)stream;
    QGX_HIP(ctx, hipMemcpyAsync(tab_of(ctx)->code, packed, sizeof(packed), hipMemcpyHostToDevice, st));
    QGX_HIP(ctx, launch_build_tables(tab_of(ctx), st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    T(ctx).code_set = true;
    T(ctx).max_code_len = 0;
    for (uint32_t j = 0; j < n_sym; ++j) T(ctx).max_code_len = code_len[j] > T(ctx).max_code_len ? code_len[j] : T(ctx).max_code_len;
    T(ctx).wide = wide_table_ok(packed, n_sym);
    return QGX_OK;
}

static qgx_status run_encode(qgx_ctx* ctx, EncMode mode, const float* V, uint32_t call_id, const float* norms_in,
                             float* norms_out, uint8_t* sym_out, const uint8_t* sym_in, qgx_stream* out, void* stream,
                             const GameArgs* game = nullptr)
{
    qgx_status s = need_levels(ctx);
    if (s != QGX_OK) return s;
    EncodeArgs a{};
    a.V = V; a.norms_in = norms_in; a.norms_out = norms_out; a.sym_out = sym_out; a.sym_in = sym_in;
    a.seed_lo = (uint32_t)ctx->cfg.seed; a.seed_hi = (uint32_t)(ctx->cfg.seed >> 32); a.call_id = call_id;
    a.call_mode = call_id == QGX_CALL_FIRST_HALF ? 1u : call_id == QGX_CALL_SECOND_HALF ? 2u : 0u;
    a.norm_kind = ctx->cfg.norm;
    a.cell_mant = (uint32_t)cell_mant(T(ctx).n_sym);
    a.pieces = enc_pieces((int)a.cell_mant, T(ctx).n_sym);
    {
        const uint32_t words = (kChunk * (T(ctx).max_code_len + 1) + 31) / 32 + 4;
        a.stage_bytes = (words + 3) / 4 * 16;
    }
    if (mode != EncMode::QuantOnly) {
        if (out->slot_words) {
            if (out->slot_words < chunk_slot_words(ctx))
                return fail(ctx, QGX_ERR_ARG, "slot_words %llu is below the %u words a chunk can take",
                            (unsigned long long)out->slot_words, chunk_slot_words(ctx));
            if (out->slot_words * ctx->lay.NC > out->payload_words_per_worker)
                return fail(ctx, QGX_ERR_CAPACITY, "slotted stream needs n_chunks * slot_words payload words per worker");
            a.slot_words = (uint32_t)out->slot_words;
        }
        a.chunk_off = out->chunk_off; a.sub_end = out->sub_end; a.payload = out->payload;
        a.cap_words = out->payload_words_per_worker;
        a.scan_state = ctx->d_scan;
    }
    if (game) a.game = *game;
    a.parts = ctx->parts;
    a.xch = ctx->d_xch;
    a.n_cu = ctx->n_simd / 4u;
    const bool powers = ctx->cfg.norm != QGX_NORM_L2 && ctx->cfg.norm != QGX_NORM_LINF;
    const uint64_t chunks = (uint64_t)ctx->lay.K * ctx->lay.NC;
    a.columns = a.parts == 1u && use_columns(chunks, ctx->lay.waves_per_bucket, ctx->lay.shared_chunks != 0u, a.slot_words == 0u, ctx->n_simd) &&
                columns_pay(chunks, ctx->lay.waves_per_bucket, ctx->rows, ctx->lay.shared_chunks != 0u, a.slot_words == 0u, powers, T(ctx).crowded, T(ctx).n_sym, ctx->n_simd);
    a.tickets = ctx->d_tickets;
    hipError_t le = launch_encode(mode, ctx->lay, tab_of(ctx), ctx->d_sc, a, (hipStream_t)stream);
    if (le != hipSuccess) return fail(ctx, QGX_ERR_HIP, "encode launch: %s", hipGetErrorString(le));
    return QGX_OK;
}

qgx_status qgx_quantize(qgx_ctx* ctx, const float* V, uint32_t call_id, const float* norms_in, float* norms_out,
                        uint8_t* sym, void* stream)
{
    if (!ctx || !V || !norms_out || !sym) return fail(ctx, QGX_ERR_ARG, "qgx_quantize: null argument");
    if (!aligned16(V) || !aligned16(sym) || !aligned16(norms_out) || !aligned16(norms_in))
        return fail(ctx, QGX_ERR_ARG, "qgx_quantize: buffers must be 16-byte aligned");
    return run_encode(ctx, EncMode::QuantOnly, V, call_id, norms_in, norms_out, sym, nullptr, nullptr, stream);
}

qgx_status qgx_encode(qgx_ctx* ctx, const float* norms, const uint8_t* sym, qgx_stream* out, void* stream)
{
    if (!ctx || !norms || !sym) return fail(ctx, QGX_ERR_ARG, "qgx_encode: null argument");
    qgx_status s = check_stream(ctx, out, "qgx_encode");
    if (s != QGX_OK) return s;
    if (!aligned16(sym)) return fail(ctx, QGX_ERR_ARG, "qgx_encode: sym must be 16-byte aligned");
    if (norms != out->norms)
        QGX_HIP(ctx, hipMemcpyAsync(out->norms, norms, (size_t)ctx->lay.K * ctx->lay.NB * sizeof(float),
                                    hipMemcpyDeviceToDevice, (hipStream_t)stream));
    return run_encode(ctx, EncMode::EncodeOnly, nullptr, 0, nullptr, nullptr, nullptr, sym, out, stream);
}

qgx_status qgx_quantize_encode(qgx_ctx* ctx, const float* V, uint32_t call_id, const float* norms_in, qgx_stream* out,
                               void* stream)
{
    if (!ctx || !V) return fail(ctx, QGX_ERR_ARG, "qgx_quantize_encode: null argument");
    qgx_status s = check_stream(ctx, out, "qgx_quantize_encode");
    if (s != QGX_OK) return s;
    if (!aligned16(V) || !aligned16(norms_in)) return fail(ctx, QGX_ERR_ARG, "qgx_quantize_encode: V must be 16-byte aligned");
    return run_encode(ctx, EncMode::Fused, V, call_id, norms_in, out->norms, nullptr, nullptr, out, stream);
}

// qgx_game -> kernel arguments, with the checks the kernels rely on (four coordinates at a time)
static qgx_status game_args(qgx_ctx* ctx, const qgx_game* game, GameArgs& g, const char* what)
{
    if (!game || !game->z || !game->a || !game->b) return fail(ctx, QGX_ERR_ARG, "%s: null game pointer", what);
    if (!aligned16(game->z) || !aligned16(game->b) || (reinterpret_cast<uintptr_t>(game->a) & 7u))
        return fail(ctx, QGX_ERR_ARG, "%s: z and b must be 16-byte aligned, a 8-byte aligned", what);
    if (ctx->cfg.d & 3u) return fail(ctx, QGX_ERR_ARG, "%s: the vector length must be a multiple of 4", what);
    if (!(game->sigma >= 0.0f) || !(std::fabs(game->mu) <= 3.402823466e+38f))
        return fail(ctx, QGX_ERR_ARG, "%s: sigma must be >= 0 and mu finite", what);
    g.z = game->z; g.a = game->a; g.b = game->b; g.mu = game->mu; g.sigma = game->sigma;
    g.seed_lo = (uint32_t)game->noise_seed; g.seed_hi = (uint32_t)(game->noise_seed >> 32);
    g.V_out = nullptr;
    return QGX_OK;
}

qgx_status qgx_game_operator(qgx_ctx* ctx, const qgx_game* game, float* F_out, void* stream)
{
    if (!ctx || !F_out || !aligned16(F_out)) return fail(ctx, QGX_ERR_ARG, "qgx_game_operator: F_out null or misaligned");
    GameArgs g{};
    qgx_status s = game_args(ctx, game, g, "qgx_game_operator");
    if (s != QGX_OK) return s;
    QGX_HIP(ctx, launch_game_operator(g, ctx->lay.d, F_out, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_game_dual_vectors(qgx_ctx* ctx, const qgx_game* game, uint32_t call_id, float* V_out, void* stream)
{
    if (!ctx || !V_out || !aligned16(V_out)) return fail(ctx, QGX_ERR_ARG, "qgx_game_dual_vectors: V_out null or misaligned");
    GameArgs g{};
    qgx_status s = game_args(ctx, game, g, "qgx_game_dual_vectors");
    if (s != QGX_OK) return s;
    const uint32_t mode = call_id == QGX_CALL_FIRST_HALF ? 1u : call_id == QGX_CALL_SECOND_HALF ? 2u : 0u;
    QGX_HIP(ctx, launch_game_dual_vectors(g, ctx->lay.d, ctx->lay.K, call_id, mode, ctx->d_sc, V_out, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_quantize_encode_game(qgx_ctx* ctx, const qgx_game* game, uint32_t call_id, qgx_stream* out, float* V_out,
                                    void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    qgx_status s = check_stream(ctx, out, "qgx_quantize_encode_game");
    if (s != QGX_OK) return s;
    GameArgs g{};
    s = game_args(ctx, game, g, "qgx_quantize_encode_game");
    if (s != QGX_OK) return s;
    if (!aligned16(V_out)) return fail(ctx, QGX_ERR_ARG, "qgx_quantize_encode_game: V_out misaligned");
    if (ctx->lay.shared_chunks || ctx->seg.size() != 1)
        return fail(ctx, QGX_ERR_ARG, "qgx_quantize_encode_game: one segment, and buckets that do not share chunks (not 256..2048)");
    if (ctx->cfg.norm != QGX_NORM_L2 && ctx->cfg.norm != QGX_NORM_LINF)
        return fail(ctx, QGX_ERR_ARG, "qgx_quantize_encode_game: L2 or L-infinity norm");
    g.V_out = V_out;
    return run_encode(ctx, EncMode::Generate, nullptr, call_id, nullptr, out->norms, nullptr, nullptr, out, stream, &g);
}

qgx_status qgx_norm2(qgx_ctx* ctx, const float* x, uint64_t n, double* result_host, void* stream)
{
    if (!ctx || !x || !result_host || n == 0) return fail(ctx, QGX_ERR_ARG, "qgx_norm2: null argument or empty vector");
    hipStream_t st = (hipStream_t)stream;
    QGX_HIP(ctx, launch_norm2(x, n, ctx->d_norm, st));
    QGX_HIP(ctx, hipMemcpyAsync(result_host, ctx->d_norm + kNormBlocks, sizeof(double), hipMemcpyDeviceToHost, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    return QGX_OK;
}

qgx_status qgx_game_gap(qgx_ctx* ctx, const qgx_game* game, const float* centre, double radius, double* result_host,
                        void* stream)
{
    if (!ctx || !result_host) return fail(ctx, QGX_ERR_ARG, "qgx_game_gap: null argument");
    GameArgs g;
    qgx_status s = game_args(ctx, game, g, "qgx_game_gap");
    if (s != QGX_OK) return s;
    if (!(game->mu > 0.0f) || !(radius >= 0.0) || !(radius <= 1.7976931348623157e308))
        return fail(ctx, QGX_ERR_ARG, "qgx_game_gap: mu must be positive and the radius finite and >= 0");
    hipStream_t st = (hipStream_t)stream;
    QGX_HIP(ctx, launch_game_gap(g, centre, radius, ctx->lay.d, ctx->d_norm, st));
    QGX_HIP(ctx, hipMemcpyAsync(result_host, ctx->d_norm + 2 * kNormBlocks + 1, sizeof(double), hipMemcpyDeviceToHost, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    return QGX_OK;
}

qgx_status qgx_quantization_metrics(qgx_ctx* ctx, const float* V, const float* Vhat, uint64_t* nonzeros_host,
                                    double* sq_error_host, double* sq_norm_host, void* stream)
{
    if (!ctx || !V || !Vhat) return fail(ctx, QGX_ERR_ARG, "qgx_quantization_metrics: null argument");
    hipStream_t st = (hipStream_t)stream;
    const uint32_t K = ctx->lay.K;
    double* result = ctx->d_metrics + (size_t)K * 3 * kMetricBlocks;
    QGX_HIP(ctx, launch_metrics(V, Vhat, ctx->lay.d, K, ctx->d_metrics, result, st));
    std::vector<double> h((size_t)K * 3);
    QGX_HIP_DRAIN(ctx, st, hipMemcpyAsync(h.data(), result, h.size() * sizeof(double), hipMemcpyDeviceToHost, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    for (uint32_t k = 0; k < K; ++k) {
        if (nonzeros_host) nonzeros_host[k] = (uint64_t)h[(size_t)k * 3];
        if (sq_error_host) sq_error_host[k] = h[(size_t)k * 3 + 1];
        if (sq_norm_host) sq_norm_host[k] = h[(size_t)k * 3 + 2];
    }
    return QGX_OK;
}

static void fill_decode_args(const qgx_ctx* ctx, DecodeArgs& a, const qgx_stream* cur, const qgx_stream* prev, bool second_half = false)
{
    a.sym_bits = longest_code(ctx) + 1;
    a.stage_words = (uint32_t)(kChunk / 2) * a.sym_bits / 32u + 8u;      // half a chunk, from a multiple of 4 words to one
    a.stage_stride = (a.stage_words + a.stage_words / 16 + 20 + 3) / 4 * 4;   // padded layout, four zero words below the end, zero words above the first
    if (a.stage_stride < 576u) a.stage_stride = 576u;     // a buffer also turns the output (16 rows of 36 floats)
    a.wide = (T(ctx).wide && (!prev || ctx->ts[ctx->sel_prev].wide)) ? 1u : 0u;   // one kernel variant reads both streams
    a.ksplit = waves_per_task(ctx->lay.n_tasks, ctx->lay.K, ctx->n_simd, prev ? 2u : 1u);
    if (eight_waves(ctx->lay.n_tasks, ctx->lay.K, ctx->n_simd, prev ? 2u : 1u, second_half)) a.ksplit = 8;
    if (ctx->ksplit_forced >= 0 && (uint32_t)ctx->ksplit_forced <= ctx->lay.K) a.ksplit = (uint32_t)ctx->ksplit_forced;
    a.n_cu = ctx->n_simd / 4u;
    a.norms = cur->norms; a.chunk_off = cur->chunk_off; a.sub_end = cur->sub_end; a.payload = cur->payload;
    a.cap_words = cur->payload_words_per_worker;
    if (prev) {
        a.norms_p = prev->norms; a.chunk_off_p = prev->chunk_off; a.sub_end_p = prev->sub_end;
        a.payload_p = prev->payload; a.cap_words_p = prev->payload_words_per_worker;
        a.tab_p = ctx->sel_prev != ctx->sel ? ctx->d_tabs + ctx->sel_prev : nullptr;
    }
}

qgx_status qgx_decode(qgx_ctx* ctx, const qgx_stream* in, float* Vhat, void* stream)
{
    if (!ctx || !Vhat) return fail(ctx, QGX_ERR_ARG, "qgx_decode: null argument");
    qgx_status s = check_stream(ctx, in, "qgx_decode");
    if (s == QGX_OK) s = need_levels(ctx);
    if (s != QGX_OK) return s;
    DecodeArgs a{};
    fill_decode_args(ctx, a, in, nullptr);
    a.out = Vhat;
    QGX_HIP(ctx, launch_decode(DecMode::Decode, ctx->lay, tab_of(ctx), ctx->d_sc, a, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_decode_average(qgx_ctx* ctx, const qgx_stream* in, float* mean, void* stream)
{
    if (!ctx || !mean || !aligned16(mean)) return fail(ctx, QGX_ERR_ARG, "qgx_decode_average: mean null or misaligned");
    qgx_status s = check_stream(ctx, in, "qgx_decode_average");
    if (s == QGX_OK) s = need_levels(ctx);
    if (s != QGX_OK) return s;
    DecodeArgs a{};
    fill_decode_args(ctx, a, in, nullptr);
    a.out = mean;
    QGX_HIP(ctx, launch_decode(DecMode::Average, ctx->lay, tab_of(ctx), ctx->d_sc, a, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_fit_levels(qgx_ctx* ctx, const float* V, uint32_t n_sym, uint32_t n_bins, uint32_t sweeps,
                          double* hist_out, void* stream)
{
    if (!ctx || !V || !aligned16(V)) return fail(ctx, QGX_ERR_ARG, "qgx_fit_levels: V null or misaligned");
    if (!T(ctx).levels_set) return fail(ctx, QGX_ERR_STATE, "qgx_fit_levels starts from the current table: set one first");
    if (n_sym != T(ctx).n_sym) return fail(ctx, QGX_ERR_ARG, "qgx_fit_levels: n_sym differs from the current table");
    if (n_bins == 0 || (n_bins & 63u) || n_bins > QGX_MAX_BINS)
        return fail(ctx, QGX_ERR_ARG, "qgx_fit_levels: n_bins must be a multiple of 64, at most 4096");
    hipStream_t st = (hipStream_t)stream;
    // The caller's histogram is written by the kernel that has it; through a copy where it is no memory of this device's.
    const bool direct = hist_out && writable_here(ctx, hist_out);
    QGX_HIP(ctx, launch_histogram(ctx->lay, V, ctx->cfg.norm, n_bins, ctx->d_hpartial, ctx->h_groups, ctx->d_hist,
                                  direct ? hist_out : nullptr, ctx->d_sc, st));
    if (hist_out && !direct)
        QGX_HIP(ctx, hipMemcpyAsync(hist_out, ctx->d_hist, n_bins * sizeof(double), hipMemcpyDeviceToDevice, st));
    QGX_HIP(ctx, launch_fit(tab_of(ctx), ctx->d_hist, n_bins, sweeps, st));
    if (sweeps != 0u) T(ctx).crowded = false;             // (not known)
    ctx->hist_bins = n_bins;
    return QGX_OK;
}

qgx_status qgx_fit_code(qgx_ctx* ctx, double* p_host, uint8_t* code_len_host, uint32_t* code_bits_host, void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    if (ctx->cfg.code != QGX_CODE_TABLE) return fail(ctx, QGX_ERR_STATE, "context was not created with QGX_CODE_TABLE");
    if (!T(ctx).levels_set || ctx->hist_bins == 0)
        return fail(ctx, QGX_ERR_STATE, "qgx_fit_code needs the histogram of a qgx_fit_levels call (sweeps = 0 leaves the table as it is)");
    uint32_t need = 1;
    while ((1u << need) < T(ctx).n_sym) ++need;
    if (need > QGX_FIT_CODE_BITS) return fail(ctx, QGX_ERR_ARG, "too many symbols for the longest code word");
    hipStream_t st = (hipStream_t)stream;
    // (a copy of the result took 4 us of the stream and the host's staging of it: an update step of 8 x 2^20 208.6 us, now 183.0, of which the copy of the histogram 4)
    QGX_HIP(ctx, launch_fit_code(tab_of(ctx), ctx->d_hist, ctx->hist_bins, QGX_FIT_CODE_BITS, ctx->d_fit, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    const FitCodeResult& host = *ctx->h_fit;
    const uint32_t* packed = host.code;
    if (p_host) std::memcpy(p_host, host.p, T(ctx).n_sym * sizeof(double));
    T(ctx).max_code_len = 0;
    for (uint32_t j = 0; j < T(ctx).n_sym; ++j) {
        const uint32_t len = packed[j] >> 16;
        T(ctx).max_code_len = len > T(ctx).max_code_len ? len : T(ctx).max_code_len;
        if (code_len_host) code_len_host[j] = (uint8_t)len;
        if (code_bits_host) code_bits_host[j] = packed[j] & 0xFFFFu;
    }
    T(ctx).code_set = true;
    T(ctx).wide = wide_table_ok(packed, T(ctx).n_sym);
    return QGX_OK;
}

qgx_status qgx_state_init(qgx_ctx* ctx, const float* X1, void* stream)
{
    if (!ctx || !aligned16(X1)) return fail(ctx, QGX_ERR_ARG, "qgx_state_init: null context or misaligned X1");
    QGX_HIP(ctx, launch_state_init(ctx->lay, ctx->d_sc, ctx->d_Y, ctx->d_anchor, X1, (hipStream_t)stream));
    ctx->has_anchor = X1 != nullptr;
    ctx->state_ready = true;
    return QGX_OK;
}

static qgx_status eg_step_with(qgx_ctx* ctx, int half, const qgx_stream* cur, const qgx_stream* prev, float* X_out,
                               void* stream, double* s_partial)
{
    if (!ctx || (half != 0 && half != 1)) return fail(ctx, QGX_ERR_ARG, "qgx_eg_step: half must be 0 or 1");
    if (!ctx->state_ready) return fail(ctx, QGX_ERR_STATE, "qgx_eg_step before qgx_state_init");
    qgx_status s = check_stream(ctx, cur, "qgx_eg_step(cur)");
    if (s == QGX_OK && prev) s = check_stream(ctx, prev, "qgx_eg_step(prev)");
    if (s == QGX_OK) s = need_levels(ctx);
    if (s == QGX_OK && prev) s = need_levels(ctx, ctx->sel_prev);
    if (s != QGX_OK) return s;
    if (!aligned16(X_out)) return fail(ctx, QGX_ERR_ARG, "qgx_eg_step: X_out misaligned");
    hipStream_t st = (hipStream_t)stream;
    DecodeArgs a{};
    a.Y = ctx->d_Y;
    a.anchor = ctx->has_anchor ? ctx->d_anchor : nullptr;
    if (half == 0) {
        if (prev) return fail(ctx, QGX_ERR_ARG, "qgx_eg_step: prev must be NULL for half = 0");
        if (!X_out) return fail(ctx, QGX_ERR_ARG, "qgx_eg_step: X_out is required for half = 0");
        fill_decode_args(ctx, a, cur, nullptr);
        a.out = X_out;
        a.x_sum = ctx->xsum_on ? ctx->d_xsum : nullptr;
        QGX_HIP(ctx, launch_decode(DecMode::Half0, ctx->lay, tab_of(ctx), ctx->d_sc, a, st));
        return QGX_OK;
    }
    fill_decode_args(ctx, a, cur, prev, true);
    a.s_partial = s_partial;
    a.x_out = X_out;
    Half1End left;
    QGX_HIP(ctx, launch_decode(DecMode::Half1, ctx->lay, tab_of(ctx), ctx->d_sc, a, st, &left));
    QGX_HIP(ctx, launch_finish_half1(ctx->lay, ctx->d_sc, s_partial, ctx->d_Y, a.anchor, X_out, left, st));
    return QGX_OK;
}

qgx_status qgx_eg_step(qgx_ctx* ctx, int half, const qgx_stream* cur, const qgx_stream* prev, float* X_out,
                       void* stream)
{
    return eg_step_with(ctx, half, cur, prev, X_out, stream, ctx ? ctx->d_spartial : nullptr);
}

qgx_status qgx_eg_step_static(qgx_ctx* ctx, int half, const qgx_stream* cur, const qgx_stream* prev, float* X_out,
                              void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    if (ctx->lay.NC > QGX_STATIC_MAX_CHUNKS)
        return fail(ctx, QGX_ERR_CAPACITY, "qgx_eg_step_static: %u chunks per worker exceed the %u the static scratch holds; use qgx_eg_step",
                    ctx->lay.NC, (unsigned)QGX_STATIC_MAX_CHUNKS);
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != ctx->device)
        return fail(ctx, QGX_ERR_STATE, "qgx_eg_step_static: the context's device must be current");
    return eg_step_with(ctx, half, cur, prev, X_out, stream, ctx->d_static_scratch);
}

qgx_status qgx_average_reset(qgx_ctx* ctx, int on, void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    ctx->xsum_on = on != 0;
    if (!ctx->xsum_on) return QGX_OK;
    if (!ctx->d_xsum && hipMalloc(&ctx->d_xsum, ctx->cfg.d * sizeof(double)) != hipSuccess)
        return fail(ctx, QGX_ERR_HIP, "qgx_average_reset: no memory for the running sum");
    QGX_HIP(ctx, launch_average_reset(ctx->lay.d, ctx->d_xsum, ctx->d_sc, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_average_export(qgx_ctx* ctx, float* X_bar, uint64_t* count, void* stream)
{
    if (!ctx || !aligned16(X_bar)) return fail(ctx, QGX_ERR_ARG, "qgx_average_export: null context or misaligned X_bar");
    if (!ctx->xsum_on) return fail(ctx, QGX_ERR_STATE, "qgx_average_export: averaging is off (qgx_average_reset)");
    unsigned long long n = 0;                               // the count lives on the device: replayed graphs add to it too
    QGX_HIP(ctx, hipMemcpyAsync(&n, &ctx->d_sc->avg_count, sizeof(n), hipMemcpyDeviceToHost, (hipStream_t)stream));
    QGX_HIP(ctx, hipStreamSynchronize((hipStream_t)stream));
    if (count) *count = n;
    if (X_bar) {
        if (n == 0) return fail(ctx, QGX_ERR_STATE, "qgx_average_export: no half-step since the reset");
        QGX_HIP(ctx, launch_average(ctx->lay.d, ctx->d_xsum, ctx->d_sc, X_bar, (hipStream_t)stream));
    }
    return QGX_OK;
}

qgx_status qgx_get_scalars(qgx_ctx* ctx, double* S, double* gamma, uint64_t* t, void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    hipStream_t st = (hipStream_t)stream;
    Scalars h;
    QGX_HIP(ctx, hipMemcpyAsync(&h, ctx->d_sc, sizeof(h), hipMemcpyDeviceToHost, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    if (S) *S = h.S;
    if (gamma) *gamma = h.gamma;
    if (t) *t = h.t;
    return QGX_OK;
}

qgx_status qgx_stream_bits(qgx_ctx* ctx, const qgx_stream* coded, uint64_t* total_bits, void* stream)
{
    if (!ctx || !total_bits) return fail(ctx, QGX_ERR_ARG, "qgx_stream_bits: null argument");
    qgx_status s = check_stream(ctx, coded, "qgx_stream_bits");
    if (s != QGX_OK) return s;
    hipStream_t st = (hipStream_t)stream;
    QGX_HIP(ctx, launch_sum_bits(ctx->lay, coded->sub_end, ctx->d_sc, st));
    unsigned long long bits = 0;
    QGX_HIP(ctx, hipMemcpyAsync(&bits, &ctx->d_sc->total_bits, sizeof(bits), hipMemcpyDeviceToHost, st));
    QGX_HIP(ctx, hipStreamSynchronize(st));
    *total_bits = bits;
    return QGX_OK;
}

qgx_status qgx_debug_set_waves_per_position(qgx_ctx* ctx, int waves)
{
    if (!ctx) return QGX_ERR_ARG;
    if (waves != 0 && waves != 1 && waves != 2 && waves != 4)
        return fail(ctx, QGX_ERR_ARG, "qgx_debug_set_waves_per_position: 0 (by the rule), 1, 2 or 4");
    ctx->ksplit_forced = waves == 0 ? -1 : waves;
    return QGX_OK;
}

qgx_status qgx_state_export(qgx_ctx* ctx, float* Y, float* anchor, void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    if (!ctx->state_ready) return fail(ctx, QGX_ERR_STATE, "state not initialised");
    hipStream_t st = (hipStream_t)stream;
    const size_t bytes = (size_t)ctx->lay.d * sizeof(float);
    if (Y) QGX_HIP(ctx, hipMemcpyAsync(Y, ctx->d_Y, bytes, hipMemcpyDeviceToDevice, st));
    if (anchor) QGX_HIP(ctx, hipMemcpyAsync(anchor, ctx->d_anchor, bytes, hipMemcpyDeviceToDevice, st));
    return QGX_OK;
}

qgx_status qgx_state_import(qgx_ctx* ctx, const float* Y, const float* anchor, double S, uint64_t t, void* stream)
{
    if (!ctx) return QGX_ERR_ARG;
    if (!(S >= 0.0) || t == 0) return fail(ctx, QGX_ERR_ARG, "qgx_state_import: S must be >= 0 and t >= 1");
    hipStream_t st = (hipStream_t)stream;
    const size_t bytes = (size_t)ctx->lay.d * sizeof(float);
    if (!ctx->state_ready) {
        QGX_HIP(ctx, launch_state_init(ctx->lay, ctx->d_sc, ctx->d_Y, ctx->d_anchor, nullptr, st));
        ctx->state_ready = true;
    }
    if (Y) QGX_HIP(ctx, hipMemcpyAsync(ctx->d_Y, Y, bytes, hipMemcpyDeviceToDevice, st));
    if (anchor) {
        QGX_HIP(ctx, hipMemcpyAsync(ctx->d_anchor, anchor, bytes, hipMemcpyDeviceToDevice, st));
        ctx->has_anchor = true;
    }
    QGX_HIP(ctx, launch_state_set(ctx->d_sc, S, t, ctx->lay.K, st));
    return QGX_OK;
}

// ---- between a model's backward pass and the dual vectors -----------------------------------------------------------

static uint32_t element_size(int dtype) { return dtype == QGX_F32 ? 4u : 2u; }
static bool known_type(int dtype) { return dtype == QGX_F32 || dtype == QGX_F16 || dtype == QGX_BF16; }
static bool aligned_to(const void* p, uint32_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1u)) == 0; }

// A list's table: the pieces, then the workers' partial sums and factors.
static uint64_t list_pieces(const qgx_tensor* tensors, uint32_t n_tensors)
{
    uint64_t pieces = 0;
    for (uint32_t i = 0; i < n_tensors; ++i) pieces += tensors[i].n / kClipPiece + (tensors[i].n % kClipPiece != 0);
    return pieces;
}
static uint64_t list_pieces_bytes(uint64_t pieces) { return (pieces * sizeof(TensorPiece) + 15u) / 16u * 16u; }
static uint64_t list_bytes(uint64_t pieces, uint32_t K)
{
    return list_pieces_bytes(pieces) + (uint64_t)K * (kClipParts + 1u) * sizeof(double);
}

// The sizes, types and places of a list's tensors.
static qgx_status check_tensors(qgx_ctx* ctx, const qgx_tensor* tensors, uint32_t n_tensors)
{
    if (!ctx) return QGX_ERR_ARG;
    if (n_tensors && !tensors) return fail(ctx, QGX_ERR_ARG, "tensor list: null argument");
    const uint64_t d = ctx->lay.d;
    for (uint32_t i = 0; i < n_tensors; ++i) {
        const qgx_tensor& t = tensors[i];
        if (!known_type(t.dtype)) return fail(ctx, QGX_ERR_ARG, "tensor %u: unknown type", i);
        if (t.n == 0) continue;
        if (!t.data || !aligned_to(t.data, element_size(t.dtype))) return fail(ctx, QGX_ERR_ARG, "tensor %u: null or misaligned data", i);
        if (t.n > d || t.offset > d - t.n) return fail(ctx, QGX_ERR_ARG, "tensor %u: elements beyond the %llu coordinates", i, (unsigned long long)d);
        if (t.stride >= (1ull << 60) / ctx->lay.K) return fail(ctx, QGX_ERR_ARG, "tensor %u: stride out of range", i);
    }
    return QGX_OK;
}

qgx_status qgx_tensor_list_size(qgx_ctx* ctx, const qgx_tensor* tensors, uint32_t n_tensors, uint64_t* bytes)
{
    const qgx_status s = check_tensors(ctx, tensors, n_tensors);
    if (s != QGX_OK) return s;
    if (!bytes) return fail(ctx, QGX_ERR_ARG, "qgx_tensor_list_size: null argument");
    *bytes = list_bytes(list_pieces(tensors, n_tensors), ctx->lay.K);
    return QGX_OK;
}

qgx_status qgx_tensor_list_set(qgx_ctx* ctx, const qgx_tensor* tensors, uint32_t n_tensors, void* table, uint64_t table_bytes,
                               qgx_tensor_list* list, void* stream)
{
    qgx_status s = check_tensors(ctx, tensors, n_tensors);
    if (s != QGX_OK) return s;
    if (!table || !list || !aligned16(table)) return fail(ctx, QGX_ERR_ARG, "qgx_tensor_list_set: null or misaligned argument");
    const uint64_t pieces = list_pieces(tensors, n_tensors), need = list_bytes(pieces, ctx->lay.K);
    if (table_bytes < need) return fail(ctx, QGX_ERR_CAPACITY, "qgx_tensor_list_set: the table needs %llu bytes", (unsigned long long)need);
    bool shared = false;
    for (uint32_t i = 0; i < n_tensors; ++i) shared = shared || (tensors[i].stride < tensors[i].n && ctx->lay.K > 1u);
    const uint64_t d = ctx->lay.d;
    // ranges of V, in order; two that follow each other may not overlap
    uint32_t* order = new (std::nothrow) uint32_t[n_tensors ? n_tensors : 1];
    if (!order) return fail(ctx, QGX_ERR_ARG, "qgx_tensor_list_set: no memory for %u tensors", n_tensors);
    uint32_t used = 0;
    for (uint32_t i = 0; i < n_tensors; ++i)
        if (tensors[i].n) order[used++] = i;
    std::sort(order, order + used, [&](uint32_t a, uint32_t b) { return tensors[a].offset < tensors[b].offset; });
    for (uint32_t i = 1; i < used && s == QGX_OK; ++i)
        if (tensors[order[i]].offset < tensors[order[i - 1]].offset + tensors[order[i - 1]].n)
            s = fail(ctx, QGX_ERR_ARG, "tensors %u and %u overlap in V", order[i - 1], order[i]);
    delete[] order;
    if (s != QGX_OK) return s;

    TensorBatch batch{};
    for (uint32_t i = 0; i < n_tensors; ++i) {
        const qgx_tensor& t = tensors[i];
        batch.entry[batch.count++] = TensorBatch::Entry{(uint64_t)reinterpret_cast<uintptr_t>(t.data), t.stride, t.n, batch.first_piece + batch.pieces,
                                                        (uint32_t)t.offset, (uint32_t)t.dtype};
        batch.pieces += t.n / kClipPiece + (t.n % kClipPiece != 0);
        if (batch.count < kTensorBatch && i + 1u < n_tensors) continue;
        if (batch.pieces) QGX_HIP(ctx, launch_tensor_list(batch, (TensorPiece*)table, (hipStream_t)stream));
        batch.first_piece += batch.pieces;
        batch.pieces = 0;
        batch.count = 0;
    }
    *list = qgx_tensor_list{};
    list->table = table; list->table_bytes = table_bytes; list->n_pieces = pieces;
    list->d = d; list->K = ctx->lay.K; list->n_tensors = n_tensors;
    list->shared_rows = shared ? 1u : 0u;
    list->dtype = -2;                                      // (none yet)
    for (uint32_t i = 0; i < n_tensors; ++i) {
        const qgx_tensor& t = tensors[i];
        if (!t.n) continue;
        list->dtype = list->dtype == -2 || list->dtype == t.dtype ? t.dtype : -1;
        if (pieces > QGX_FEW_TENSORS) continue;            // (a tensor with elements has a piece at least)
        const uint64_t size = element_size(t.dtype);
        list->few[list->n_few].at = (uint64_t)reinterpret_cast<uintptr_t>(t.data);
        list->few[list->n_few].step = t.stride * size;
        list->few[list->n_few++].bytes = t.n * size;
    }
    return QGX_OK;
}

// Do some of the bytes from v on belong to one of the few tensors?
static bool shares_memory(const qgx_tensor_list* list, uint64_t v, uint64_t bytes)
{
    for (uint32_t i = 0; i < list->n_few; ++i) {
        const uint64_t at = list->few[i].at, step = list->few[i].step, n = list->few[i].bytes;
        // the first worker whose elements end past v, if any
        const uint64_t k = at + n > v ? 0 : step ? (v - at - n) / step + 1u : list->K;
        if (k < list->K && at + k * step < v + bytes) return true;
    }
    return false;
}

qgx_status qgx_clip_gradients(qgx_ctx* ctx, const qgx_tensor_list* list, int norm, float max_norm, float* V, float* norms,
                              void* stream)
{
    if (!ctx || !list || !list->table) return fail(ctx, QGX_ERR_ARG, "qgx_clip_gradients: null argument");
    if (norm != QGX_NORM_L2 && norm != QGX_NORM_LINF) return fail(ctx, QGX_ERR_ARG, "qgx_clip_gradients: the norm is L2 or L-infinity");
    if (!(max_norm >= 0.0f)) return fail(ctx, QGX_ERR_ARG, "qgx_clip_gradients: max_norm must be >= 0");
    if (!aligned16(V) || !aligned_to(norms, 4u)) return fail(ctx, QGX_ERR_ARG, "qgx_clip_gradients: V must be 16-byte aligned, norms 4-byte");
    if (!V && list->shared_rows) return fail(ctx, QGX_ERR_ARG, "qgx_clip_gradients: the workers share elements, which in-place clipping would scale more than once");
    if (list->d != ctx->lay.d || list->K != ctx->lay.K)
        return fail(ctx, QGX_ERR_ARG, "qgx_clip_gradients: the list was made for %u workers of %llu coordinates", list->K, (unsigned long long)list->d);
    if (list->table_bytes < list_bytes(list->n_pieces, ctx->lay.K))
        return fail(ctx, QGX_ERR_CAPACITY, "qgx_clip_gradients: the list's table is too small for this context");
    ClipArgs a{};
    a.table = (const TensorPiece*)list->table;
    a.partial = (double*)((char*)list->table + list_pieces_bytes(list->n_pieces));
    a.scale = a.partial + (uint64_t)ctx->lay.K * kClipParts;
    a.V = V; a.norms = norms; a.d = ctx->lay.d;
    a.n_pieces = list->n_pieces; a.max_norm = max_norm;
    a.dtype = list->dtype;
    a.apart = V && list->n_few && !shares_memory(list, (uint64_t)reinterpret_cast<uintptr_t>(V), (uint64_t)ctx->lay.K * ctx->lay.d * sizeof(float));
    QGX_HIP(ctx, launch_clip(a, ctx->lay.K, norm == QGX_NORM_LINF, ctx->n_simd / 4u, ctx->d_sc, (hipStream_t)stream));
    return QGX_OK;
}

// Whether the runs of `run` elements that n indices by strides st (at most 2^60 / n) give are apart: smallest stride first, every one has to
// step over what the ones before reach.
static bool steps_apart(const uint64_t* n, const uint64_t* st, int dims, uint64_t run)
{
    uint64_t reach = run;
    bool done[4] = {true, true, true, true};
    for (int i = 0; i < dims; ++i) done[i] = n[i] == 1;
    for (;;) {
        int at = -1;
        for (int i = 0; i < dims; ++i)
            if (!done[i] && (at < 0 || st[i] < st[at])) at = i;
        if (at < 0) return true;
        if (st[at] < reach) return false;
        reach += (n[at] - 1) * st[at];
        done[at] = true;
    }
}

// Rows of a tensor: null, misaligned, or with strides beyond what 64-bit addresses hold; rows that are written may not overlap.
static qgx_status check_rows(qgx_ctx* ctx, const char* what, const void* p, int dtype, uint64_t workers, uint64_t rows, uint64_t cols,
                             uint64_t worker, uint64_t row, bool written)
{
    if (!p || !aligned_to(p, element_size(dtype))) return fail(ctx, QGX_ERR_ARG, "%s: null or misaligned", what);
    if (worker >= (1ull << 62) / workers || row >= (1ull << 62) / rows) return fail(ctx, QGX_ERR_ARG, "%s: stride out of range", what);
    if (written) {
        // either the rows of a worker lie within the step to the next worker's, or the workers of a row within that to the next row
        const bool by_worker = (rows == 1 || row >= cols) && (workers == 1 || worker >= (rows - 1) * row + cols);
        const bool by_row = (workers == 1 || worker >= cols) && (rows == 1 || row >= (workers - 1) * worker + cols);
        if (!by_worker && !by_row) return fail(ctx, QGX_ERR_ARG, "%s: rows overlap", what);
    }
    return QGX_OK;
}

static qgx_status check_norm(qgx_ctx* ctx, const char* what, int dtype, uint64_t workers, uint64_t rows, uint64_t cols)
{
    if (!ctx) return QGX_ERR_ARG;
    if (!known_type(dtype)) return fail(ctx, QGX_ERR_ARG, "%s: unknown type", what);
    if (cols == 0 || cols > (1u << 24)) return fail(ctx, QGX_ERR_ARG, "%s: cols must be 1 .. 2^24", what);
    if (workers > 65535u || rows >= (1ull << 31) || workers * rows >= (1ull << 31))
        return fail(ctx, QGX_ERR_ARG, "%s: workers must be at most 65535, and workers * rows below 2^31", what);
    return QGX_OK;
}

qgx_status qgx_layer_norm(qgx_ctx* ctx, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, const void* x, uint64_t x_worker,
                          uint64_t x_row, const float* weight, const float* bias, float eps, void* y, uint64_t y_worker,
                          uint64_t y_row, float* mean, float* rstd, void* stream)
{
    qgx_status s = check_norm(ctx, "qgx_layer_norm", dtype, workers, rows, cols);
    if (s != QGX_OK) return s;
    if (!(eps >= 0.0f)) return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm: eps must be >= 0");
    if (workers == 0 || rows == 0) return QGX_OK;
    s = check_rows(ctx, "qgx_layer_norm(x)", x, dtype, workers, rows, cols, x_worker, x_row, false);
    if (s == QGX_OK) s = check_rows(ctx, "qgx_layer_norm(y)", y, dtype, workers, rows, cols, y_worker, y_row, true);
    if (s != QGX_OK) return s;
    if (x == y && ((workers > 1 && x_worker != y_worker) || (rows > 1 && x_row != y_row)))
        return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm: y at x's memory must have its strides");
    if (!aligned_to(weight, 4u) || !aligned_to(bias, 4u) || !aligned_to(mean, 4u) || !aligned_to(rstd, 4u))
        return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm: binary32 buffers must be 4-byte aligned");
    NormArgs a{};
    a.x = x; a.y = y; a.w = weight; a.b = bias; a.mean = mean; a.rstd = rstd;
    a.x_worker = x_worker; a.x_row = x_row; a.y_worker = y_worker; a.y_row = y_row;
    a.rows = (uint32_t)rows; a.n_rows = (uint32_t)(workers * rows); a.cols = (uint32_t)cols; a.eps = eps;
    QGX_HIP(ctx, launch_layer_norm(dtype, a, ctx->n_simd / 4u, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_layer_norm_scratch(qgx_ctx* ctx, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, uint64_t* bytes)
{
    const qgx_status s = check_norm(ctx, "qgx_layer_norm_scratch", dtype, workers, rows, cols);
    if (s != QGX_OK) return s;
    if (!bytes) return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_scratch: null argument");
    *bytes = workers ? norm_back_plan(dtype, (uint32_t)workers, (uint32_t)rows, (uint32_t)cols, ctx->n_simd / 4u).scratch : 0;
    return QGX_OK;
}

qgx_status qgx_layer_norm_backward(qgx_ctx* ctx, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, const void* dy,
                                   uint64_t dy_worker, uint64_t dy_row, const void* x, uint64_t x_worker, uint64_t x_row,
                                   const float* weight, const float* mean, const float* rstd, void* dx, uint64_t dx_worker,
                                   uint64_t dx_row, float* dweight, float* dbias, uint64_t param_stride, void* scratch,
                                   uint64_t scratch_bytes, void* stream)
{
    qgx_status s = check_norm(ctx, "qgx_layer_norm_backward", dtype, workers, rows, cols);
    if (s != QGX_OK) return s;
    if (workers == 0) return QGX_OK;
    if (rows) {
        s = check_rows(ctx, "qgx_layer_norm_backward(dy)", dy, dtype, workers, rows, cols, dy_worker, dy_row, false);
        if (s == QGX_OK) s = check_rows(ctx, "qgx_layer_norm_backward(x)", x, dtype, workers, rows, cols, x_worker, x_row, false);
        if (s == QGX_OK && dx) s = check_rows(ctx, "qgx_layer_norm_backward(dx)", dx, dtype, workers, rows, cols, dx_worker, dx_row, true);
        if (s != QGX_OK) return s;
        if (!mean || !rstd) return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_backward: null mean or rstd");
        if (dx && (dx == dy || dx == x)) return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_backward: dx may not be dy or x");
    }
    if ((dweight || dbias) && workers > 1 && param_stride < cols)
        return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_backward: param_stride below cols");
    if (param_stride >= (1ull << 62) / workers) return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_backward: stride out of range");
    if (!aligned_to(weight, 4u) || !aligned_to(mean, 4u) || !aligned_to(rstd, 4u) || !aligned_to(dweight, 4u) || !aligned_to(dbias, 4u))
        return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_backward: binary32 buffers must be 4-byte aligned");
    const NormBackPlan plan = norm_back_plan(dtype, (uint32_t)workers, (uint32_t)rows, (uint32_t)cols, ctx->n_simd / 4u);
    const uint64_t need = plan.scratch;
    if (need && (!scratch || !aligned16(scratch))) return fail(ctx, QGX_ERR_ARG, "qgx_layer_norm_backward: null or misaligned scratch");
    if (scratch_bytes < need) return fail(ctx, QGX_ERR_CAPACITY, "qgx_layer_norm_backward: scratch needs %llu bytes", (unsigned long long)need);
    NormBackArgs a{};
    a.dy = dy; a.x = x; a.w = weight; a.mean = mean; a.rstd = rstd; a.dx = dx; a.dw = dweight; a.db = dbias;
    a.dy_worker = dy_worker; a.dy_row = dy_row; a.x_worker = x_worker; a.x_row = x_row; a.dx_worker = dx_worker; a.dx_row = dx_row;
    a.param_stride = param_stride;
    a.rows = (uint32_t)rows; a.n_rows = (uint32_t)(workers * rows); a.cols = (uint32_t)cols;
    a.scratch = (float*)scratch;
    QGX_HIP(ctx, launch_layer_norm_back(dtype, a, (uint32_t)workers, plan, (hipStream_t)stream));
    return QGX_OK;
}

static qgx_status bucket_args(qgx_ctx* ctx, const char* what, const qgx_buckets* b, uint32_t table_rows, BucketArgs& out)
{
    if (!b || !b->bounds || !b->rows) return fail(ctx, QGX_ERR_ARG, "%s: null buckets", what);
    if (b->n == 0 || b->n > QGX_MAX_INTERVALS) return fail(ctx, QGX_ERR_ARG, "%s: 1 .. %u intervals", what, QGX_MAX_INTERVALS);
    out.n = b->n;
    for (uint32_t i = 0; i <= b->n; ++i) {
        if (i && b->bounds[i] <= b->bounds[i - 1]) return fail(ctx, QGX_ERR_ARG, "%s: bounds not strictly ascending at %u", what, i);
        out.bounds[i] = b->bounds[i];
        if (i == b->n) break;
        if (b->rows[i] >= table_rows) return fail(ctx, QGX_ERR_ARG, "%s: interval %u takes row %u of a table of %u", what, i, b->rows[i], table_rows);
        out.rows[i] = (uint16_t)b->rows[i];
    }
    return QGX_OK;
}

static bool no_scores(const qgx_scores* s) { return s->workers == 0 || s->batch == 0 || s->q == 0 || s->k == 0; }

// The shape is one the kernels' 32-bit counts hold, and the addresses fit 64 bits.
static qgx_status check_scores(qgx_ctx* ctx, const char* what, const qgx_scores* s, bool written)
{
    if (!known_type(s->dtype)) return fail(ctx, QGX_ERR_ARG, "%s: unknown type", what);
    if (s->heads == 0 || s->heads > 65535u || s->q > (1u << 29) || s->k > (1u << 29) || s->q * s->k > (1ull << 34) || s->workers > 65535u || s->batch >= (1ull << 31) ||
        s->workers * s->batch * s->heads >= (1ull << 31))
        return fail(ctx, QGX_ERR_ARG, "%s: size out of range", what);
    if (no_scores(s)) return QGX_OK;
    if (!s->data || !aligned_to(s->data, element_size(s->dtype))) return fail(ctx, QGX_ERR_ARG, "%s: null or misaligned scores", what);
    const uint64_t n[4] = {s->workers, s->batch, s->heads, s->q}, st[4] = {s->s_worker, s->s_batch, s->s_head, s->s_row};
    for (int i = 0; i < 4; ++i)
        if (st[i] >= (1ull << 60) / n[i]) return fail(ctx, QGX_ERR_ARG, "%s: stride out of range", what);
    if (written && !steps_apart(n, st, 4, s->k)) return fail(ctx, QGX_ERR_ARG, "%s: rows overlap", what);
    return QGX_OK;
}

static void in_args(BiasArgs& a, const qgx_scores* s)
{
    a.in = s->data;
    a.i_worker = s->s_worker; a.i_batch = s->s_batch; a.i_head = s->s_head; a.i_row = s->s_row;
}

static void shape_args(BiasArgs& a, const qgx_scores* s)
{
    a.batch = (uint32_t)s->batch; a.heads = s->heads; a.q = (uint32_t)s->q; a.k = (uint32_t)s->k;
    a.planes = (uint32_t)(s->workers * s->batch * s->heads);
}

static bool offset_ok(int64_t q_offset) { return q_offset >= -(1ll << 30) && q_offset <= (1ll << 30); }

qgx_status qgx_position_bias(qgx_ctx* ctx, const qgx_buckets* buckets, const float* table, uint32_t table_rows, const qgx_scores* in,
                             const qgx_scores* out, int64_t q_offset, const int32_t* positions, void* stream)
{
    if (!ctx || !table || !out) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias: null argument");
    BucketArgs b{};
    qgx_status s = bucket_args(ctx, "qgx_position_bias", buckets, table_rows, b);
    if (s == QGX_OK) s = check_scores(ctx, "qgx_position_bias(out)", out, true);
    if (s != QGX_OK) return s;
    if (table_rows > 65535u || !offset_ok(q_offset)) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias: table_rows or q_offset out of range");
    if (!aligned_to(table, 4u) || !aligned_to(positions, 4u)) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias: table and positions must be 4-byte aligned");
    BiasArgs a{};
    if (in) {
        s = check_scores(ctx, "qgx_position_bias(in)", in, false);
        if (s != QGX_OK) return s;
        if (in->dtype != out->dtype || in->workers != out->workers || in->batch != out->batch || in->heads != out->heads || in->q != out->q || in->k != out->k)
            return fail(ctx, QGX_ERR_ARG, "qgx_position_bias: in and out differ in type or shape");
        if (in->data == out->data && ((in->workers > 1 && in->s_worker != out->s_worker) || (in->batch > 1 && in->s_batch != out->s_batch) ||
                                      (in->heads > 1 && in->s_head != out->s_head) || (in->q > 1 && in->s_row != out->s_row)))
            return fail(ctx, QGX_ERR_ARG, "qgx_position_bias: out at in's memory must have its strides");
        in_args(a, in);
    }
    if (no_scores(out)) return QGX_OK;
    shape_args(a, out);
    a.out = out->data;
    a.o_worker = out->s_worker; a.o_batch = out->s_batch; a.o_head = out->s_head; a.o_row = out->s_row;
    a.table = table; a.positions = positions; a.q_offset = q_offset;
    QGX_HIP(ctx, launch_position_bias(out->dtype, a, b, ctx->n_simd / 4u, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_position_bias_scratch(qgx_ctx* ctx, const qgx_buckets* buckets, const qgx_scores* grad, int64_t q_offset, uint64_t* bytes)
{
    if (!ctx || !grad || !bytes) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_scratch: null argument");
    BucketArgs b{};
    qgx_status s = bucket_args(ctx, "qgx_position_bias_scratch", buckets, 65535u, b);
    if (s == QGX_OK) s = check_scores(ctx, "qgx_position_bias_scratch", grad, false);
    if (s != QGX_OK) return s;
    if (!offset_ok(q_offset)) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_scratch: q_offset out of range");
    BiasArgs a{};
    shape_args(a, grad);
    a.q_offset = q_offset;
    *bytes = bias_back_plan(grad->dtype, a, b, (uint32_t)grad->workers, ctx->n_simd / 4u).scratch;
    return QGX_OK;
}

qgx_status qgx_position_bias_backward(qgx_ctx* ctx, const qgx_buckets* buckets, const qgx_scores* grad, int64_t q_offset, float* dtable,
                                      uint32_t table_rows, uint64_t param_stride, void* scratch, uint64_t scratch_bytes, void* stream)
{
    if (!ctx || !grad || !dtable) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_backward: null argument");
    BucketArgs b{};
    qgx_status s = bucket_args(ctx, "qgx_position_bias_backward", buckets, table_rows, b);
    if (s == QGX_OK) s = check_scores(ctx, "qgx_position_bias_backward", grad, false);
    if (s != QGX_OK) return s;
    if (table_rows > 65535u || (uint64_t)table_rows * grad->heads >= (1u << 24) || !offset_ok(q_offset))
        return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_backward: table_rows * heads or q_offset out of range");
    if (grad->workers > 1 && param_stride < (uint64_t)table_rows * grad->heads)
        return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_backward: param_stride below the table's size");
    if (param_stride >= (1ull << 46) || !aligned_to(dtable, 4u)) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_backward: stride out of range or misaligned dtable");
    if (grad->workers == 0) return QGX_OK;
    BiasArgs a{};
    in_args(a, grad);
    shape_args(a, grad);
    a.q_offset = q_offset;
    const BiasBackPlan plan = bias_back_plan(grad->dtype, a, b, (uint32_t)grad->workers, ctx->n_simd / 4u);
    const uint64_t need = plan.scratch;
    if (need && (!scratch || !aligned16(scratch))) return fail(ctx, QGX_ERR_ARG, "qgx_position_bias_backward: null or misaligned scratch");
    if (scratch_bytes < need) return fail(ctx, QGX_ERR_CAPACITY, "qgx_position_bias_backward: scratch needs %llu bytes", (unsigned long long)need);
    QGX_HIP(ctx, launch_position_bias_back(grad->dtype, a, b, plan, dtable, table_rows, param_stride, scratch, (hipStream_t)stream));
    return QGX_OK;
}

// ---- an image or video model's block --------------------------------------------------------------------------------

// Kept rows: their number and shape, and the addresses.
static qgx_status check_kept(qgx_ctx* ctx, const char* what, const qgx_kept* kept, uint64_t rows, uint64_t cols)
{
    if (kept->cols == 0 || kept->cols > (1u << 24) || kept->rows >= (1ull << 31)) return fail(ctx, QGX_ERR_ARG, "%s: kept rows or columns out of range", what);
    if (kept->rows != rows || kept->cols != cols) return fail(ctx, QGX_ERR_ARG, "%s: kept rows of another shape", what);
    if (rows && (!kept->codes || !kept->powers || !aligned16(kept->codes))) return fail(ctx, QGX_ERR_ARG, "%s: null or misaligned codes or powers", what);
    return QGX_OK;
}

// The same of rows that are to be kept: their tensor's number too.
static qgx_status check_keep(qgx_ctx* ctx, const char* what, const qgx_kept* kept, uint64_t rows, uint64_t cols)
{
    if (kept->tensor >= (1u << 24)) return fail(ctx, QGX_ERR_ARG, "%s: a kept tensor's number must be below 2^24", what);
    return check_kept(ctx, what, kept, rows, cols);
}

static uint32_t kept_blocks(uint64_t cols) { return (uint32_t)((cols + QGX_KEPT_BLOCK - 1u) / QGX_KEPT_BLOCK); }
static uint32_t kept_top(int dtype) { return dtype == QGX_F16 ? kKeptTopF16 : kKeptTop; }

static KeptDraws kept_draws(const qgx_ctx* ctx, const qgx_kept* out, int unbiased, uint32_t call_id)
{
    KeptDraws d{};
    d.seed_lo = (uint32_t)ctx->cfg.seed; d.seed_hi = (uint32_t)(ctx->cfg.seed >> 32); d.call_id = call_id;
    d.call_mode = call_id == QGX_CALL_FIRST_HALF ? 1u : call_id == QGX_CALL_SECOND_HALF ? 2u : 0u;
    d.domain = 2u + 256u * out->tensor;
    d.on = unbiased != 0;
    return d;
}

qgx_status qgx_checkpoint(qgx_ctx* ctx, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, const void* x, uint64_t x_worker,
                          uint64_t x_row, int unbiased, uint32_t call_id, const qgx_kept* out, void* stream)
{
    qgx_status s = check_norm(ctx, "qgx_checkpoint", dtype, workers, rows, cols);
    if (s != QGX_OK) return s;
    if (!out) return fail(ctx, QGX_ERR_ARG, "qgx_checkpoint: null argument");
    s = check_keep(ctx, "qgx_checkpoint", out, workers * rows, cols);
    if (s != QGX_OK) return s;
    if (workers == 0 || rows == 0) return QGX_OK;
    s = check_rows(ctx, "qgx_checkpoint(x)", x, dtype, workers, rows, cols, x_worker, x_row, false);
    if (s != QGX_OK) return s;
    KeepArgs a{};
    a.x = x; a.codes = out->codes; a.powers = out->powers; a.x_worker = x_worker; a.x_row = x_row;
    a.rows = (uint32_t)rows; a.batch = 1; a.n_rows = (uint32_t)(workers * rows); a.cols = (uint32_t)cols; a.blocks = kept_blocks(cols); a.top = kept_top(dtype);
    QGX_HIP(ctx, launch_checkpoint(dtype, a, kept_draws(ctx, out, unbiased, call_id), ctx->d_sc, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_restore(qgx_ctx* ctx, const qgx_kept* in, int dtype, void* y, uint64_t y_row, void* stream)
{
    if (!ctx || !in) return fail(ctx, QGX_ERR_ARG, "qgx_restore: null argument");
    qgx_status s = check_norm(ctx, "qgx_restore", dtype, 1, in->rows, in->cols);
    if (s == QGX_OK) s = check_kept(ctx, "qgx_restore", in, in->rows, in->cols);
    if (s != QGX_OK || in->rows == 0) return s;
    s = check_rows(ctx, "qgx_restore(y)", y, dtype, 1, in->rows, in->cols, 0, y_row, true);
    if (s != QGX_OK) return s;
    KeepArgs a{};
    a.y = y; a.codes = in->codes; a.powers = in->powers; a.y_row = y_row;
    a.rows = a.n_rows = (uint32_t)in->rows; a.cols = (uint32_t)in->cols; a.blocks = kept_blocks(in->cols);
    QGX_HIP(ctx, launch_restore(dtype, a, (hipStream_t)stream));
    return QGX_OK;
}

static qgx_status check_gradient(qgx_ctx* ctx, const char* what, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, uint64_t out)
{
    const qgx_status s = check_norm(ctx, what, dtype, workers, rows, cols);
    if (s != QGX_OK) return s;
    if (out == 0 || out > (1u << 24) || cols * out >= (1ull << 31)) return fail(ctx, QGX_ERR_ARG, "%s: out must be 1 .. 2^24, and cols * out below 2^31", what);
    return QGX_OK;
}

// The plan, and that its grid (of one dimension, 2^32 threads at most) holds it.
static qgx_status gradient_plan(qgx_ctx* ctx, const char* what, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, uint64_t out, uint64_t dy_row,
                                WeightGradPlan& plan)
{
    plan = weight_grad_plan(dtype, (uint32_t)workers, (uint32_t)rows, (uint32_t)cols, (uint32_t)out, dy_row, ctx->n_simd / 4u);
    if ((uint64_t)plan.tiles_i * plan.tiles_o * plan.parts * workers >= (1u << 24)) return fail(ctx, QGX_ERR_ARG, "%s: more tiles than a launch has", what);
    return QGX_OK;
}

qgx_status qgx_weight_gradient_scratch(qgx_ctx* ctx, int dtype, uint64_t workers, uint64_t rows, uint64_t cols, uint64_t out, uint64_t dy_row, uint64_t* bytes)
{
    qgx_status s = check_gradient(ctx, "qgx_weight_gradient_scratch", dtype, workers, rows, cols, out);
    if (s != QGX_OK) return s;
    if (!bytes) return fail(ctx, QGX_ERR_ARG, "qgx_weight_gradient_scratch: null argument");
    WeightGradPlan plan;
    s = gradient_plan(ctx, "qgx_weight_gradient_scratch", dtype, workers, rows, cols, out, dy_row, plan);
    if (s == QGX_OK) *bytes = plan.scratch;
    return s;
}

qgx_status qgx_weight_gradient(qgx_ctx* ctx, const qgx_kept* x, int dtype, uint64_t workers, uint64_t rows, uint64_t out, const void* dy,
                               uint64_t dy_worker, uint64_t dy_row, float* dweight, uint64_t dw_worker, float* dbias, uint64_t db_worker,
                               void* scratch, uint64_t scratch_bytes, void* stream)
{
    if (!ctx || !x) return fail(ctx, QGX_ERR_ARG, "qgx_weight_gradient: null argument");
    const uint64_t cols = x->cols;
    qgx_status s = check_gradient(ctx, "qgx_weight_gradient", dtype, workers, rows, cols, out);
    if (s == QGX_OK) s = check_kept(ctx, "qgx_weight_gradient", x, workers * rows, cols);
    if (s != QGX_OK || workers == 0) return s;
    if (rows) s = check_rows(ctx, "qgx_weight_gradient(dy)", dy, dtype, workers, rows, out, dy_worker, dy_row, false);
    if (s != QGX_OK) return s;
    if (!dweight || !aligned_to(dweight, 4u) || !aligned_to(dbias, 4u)) return fail(ctx, QGX_ERR_ARG, "qgx_weight_gradient: null or misaligned gradients");
    if ((workers > 1 && (dw_worker < cols * out || (dbias && db_worker < out))) || dw_worker >= (1ull << 60) / workers || db_worker >= (1ull << 60) / workers)
        return fail(ctx, QGX_ERR_ARG, "qgx_weight_gradient: the workers' gradients overlap, or a stride out of range");
    WeightGradPlan plan;
    s = gradient_plan(ctx, "qgx_weight_gradient", dtype, workers, rows, cols, out, dy_row, plan);
    if (s != QGX_OK) return s;
    if (plan.scratch && (!scratch || !aligned16(scratch))) return fail(ctx, QGX_ERR_ARG, "qgx_weight_gradient: null or misaligned scratch");
    if (scratch_bytes < plan.scratch) return fail(ctx, QGX_ERR_CAPACITY, "qgx_weight_gradient: scratch needs %llu bytes", (unsigned long long)plan.scratch);
    WeightGradArgs a{};
    a.codes = x->codes; a.powers = x->powers; a.dy = dy; a.dw = dweight; a.db = dbias; a.scratch = (float*)scratch;
    a.dy_worker = dy_worker; a.dy_row = dy_row; a.dw_worker = dw_worker; a.db_worker = db_worker;
    a.rows = (uint32_t)rows; a.cols = (uint32_t)cols; a.out = (uint32_t)out; a.blocks = kept_blocks(cols);
    QGX_HIP(ctx, launch_weight_grad(dtype, a, (uint32_t)workers, plan, (hipStream_t)stream));
    return QGX_OK;
}

// The shape is one the kernels' counts and grids hold.
static qgx_status check_group(qgx_ctx* ctx, const char* what, const qgx_group_shape* g)
{
    if (!ctx || !g) return fail(ctx, QGX_ERR_ARG, "%s: null argument", what);
    if (!known_type(g->dtype)) return fail(ctx, QGX_ERR_ARG, "%s: unknown type", what);
    if (g->activation < QGX_ACT_NONE || g->activation > QGX_ACT_LEAKY) return fail(ctx, QGX_ERR_ARG, "%s: unknown activation", what);
    if (g->activation == QGX_ACT_LEAKY && !(std::fabs(g->slope) <= FLT_MAX)) return fail(ctx, QGX_ERR_ARG, "%s: slope must be finite", what);
    if (g->channels == 0 || g->channels > (1u << 20)) return fail(ctx, QGX_ERR_ARG, "%s: channels must be 1 .. 2^20", what);
    if (g->groups == 0 || g->channels % g->groups) return fail(ctx, QGX_ERR_ARG, "%s: groups must divide channels", what);
    if (g->workers > 65535u || g->batch > 65535u || g->workers * g->batch > 65535u || g->places >= (1ull << 31) || g->workers * g->batch * g->places >= (1ull << 31) ||
        g->places * g->channels >= (1ull << 36))
        return fail(ctx, QGX_ERR_ARG, "%s: size out of range", what);
    return QGX_OK;
}

// The plan, and that its grid holds it: 2^32 threads at most.
static qgx_status plan_of(qgx_ctx* ctx, const char* what, const qgx_group_shape* g, bool backward, GroupPlan& plan)
{
    const uint64_t samples = g->workers * g->batch;
    plan = group_plan(g->dtype, (uint32_t)g->workers, (uint32_t)samples, (uint32_t)g->places, (uint32_t)g->channels, g->groups, backward, ctx->n_simd / 4u);
    if (plan.whole && samples * plan.spans * plan.threads >= (1ull << 32)) return fail(ctx, QGX_ERR_ARG, "%s: more samples and channels than a launch has", what);
    return QGX_OK;
}

static bool no_places(const qgx_group_shape* g) { return g->workers == 0 || g->batch == 0 || g->places == 0; }

// A tensor of the shape: addresses, strides, and, where it is written, places that do not overlap.
static qgx_status check_places(qgx_ctx* ctx, const char* what, const qgx_group_shape* g, const qgx_places* p, bool written)
{
    if (!p->data || !aligned_to(p->data, element_size(g->dtype))) return fail(ctx, QGX_ERR_ARG, "%s: null or misaligned", what);
    const uint64_t n[3] = {g->workers, g->batch, g->places}, st[3] = {p->s_worker, p->s_batch, p->s_place};
    for (int i = 0; i < 3; ++i)
        if (st[i] >= (1ull << 60) / n[i]) return fail(ctx, QGX_ERR_ARG, "%s: stride out of range", what);
    if (written && !steps_apart(n, st, 3, g->channels)) return fail(ctx, QGX_ERR_ARG, "%s: places overlap", what);
    return QGX_OK;
}

static bool same_places(const qgx_group_shape* g, const qgx_places* a, const qgx_places* b)
{
    return (g->workers == 1 || a->s_worker == b->s_worker) && (g->batch == 1 || a->s_batch == b->s_batch) && (g->places == 1 || a->s_place == b->s_place);
}

static GroupArgs group_args(const qgx_group_shape* g)
{
    GroupArgs a{};
    a.samples = (uint32_t)(g->workers * g->batch); a.places = (uint32_t)g->places; a.channels = (uint32_t)g->channels;
    a.groups = g->groups; a.per = a.channels / a.groups;
    a.activation = g->activation; a.slope = g->slope;
    return a;
}

static qgx_status check_group_scratch(qgx_ctx* ctx, const char* what, const GroupPlan& plan, const void* scratch, uint64_t bytes)
{
    if (plan.scratch && (!scratch || !aligned16(scratch))) return fail(ctx, QGX_ERR_ARG, "%s: null or misaligned scratch", what);
    if (bytes < plan.scratch) return fail(ctx, QGX_ERR_CAPACITY, "%s: scratch needs %llu bytes", what, (unsigned long long)plan.scratch);
    return QGX_OK;
}

qgx_status qgx_group_norm_scratch(qgx_ctx* ctx, const qgx_group_shape* shape, int backward, uint64_t* bytes)
{
    qgx_status s = check_group(ctx, "qgx_group_norm_scratch", shape);
    if (s != QGX_OK) return s;
    if (!bytes) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_scratch: null argument");
    GroupPlan plan{};
    if (!no_places(shape)) s = plan_of(ctx, "qgx_group_norm_scratch", shape, backward != 0, plan);
    if (s == QGX_OK) *bytes = plan.scratch;
    return s;
}

qgx_status qgx_group_norm(qgx_ctx* ctx, const qgx_group_shape* shape, const qgx_places* x, const float* weight, const float* bias, float eps,
                          const qgx_places* y, float* mean, float* rstd, const qgx_kept* keep, int unbiased, uint32_t call_id,
                          void* scratch, uint64_t scratch_bytes, void* stream)
{
    qgx_status s = check_group(ctx, "qgx_group_norm", shape);
    if (s != QGX_OK) return s;
    if (!x || !y) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm: null argument");
    if (!(eps >= 0.0f)) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm: eps must be >= 0");
    if (keep) s = check_keep(ctx, "qgx_group_norm(keep)", keep, shape->workers * shape->batch * shape->places, shape->channels);
    if (s != QGX_OK) return s;
    const bool none = no_places(shape);
    if (!none) s = check_places(ctx, "qgx_group_norm(x)", shape, x, false);
    if (!none && s == QGX_OK) s = check_places(ctx, "qgx_group_norm(y)", shape, y, true);
    if (s != QGX_OK) return s;
    if (!none && x->data == y->data && !same_places(shape, x, y)) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm: y at x's memory must have its strides");
    if (!aligned_to(weight, 4u) || !aligned_to(bias, 4u) || !aligned_to(mean, 4u) || !aligned_to(rstd, 4u))
        return fail(ctx, QGX_ERR_ARG, "qgx_group_norm: binary32 buffers must be 4-byte aligned");
    GroupArgs a = group_args(shape);
    if (none) {
        a.mean = mean; a.rstd = rstd;
        QGX_HIP(ctx, launch_group_no_places(a, (hipStream_t)stream));
        return QGX_OK;
    }
    GroupPlan plan;
    s = plan_of(ctx, "qgx_group_norm", shape, false, plan);
    if (s == QGX_OK) s = check_group_scratch(ctx, "qgx_group_norm", plan, scratch, scratch_bytes);
    if (s != QGX_OK) return s;
    a.x = x->data; a.x_worker = x->s_worker; a.x_batch = x->s_batch; a.x_place = x->s_place;
    a.y = y->data; a.y_worker = y->s_worker; a.y_batch = y->s_batch; a.y_place = y->s_place;
    a.w = weight; a.b = bias; a.mean = mean; a.rstd = rstd; a.eps = eps; a.scratch = (float*)scratch;
    if (keep && group_keeps(plan, a.channels)) {
        a.keep_codes = keep->codes; a.keep_powers = keep->powers; a.keep_top = kept_top(shape->dtype); a.draws = kept_draws(ctx, keep, unbiased, call_id);
    } else if (keep) {
        KeepArgs k{};
        k.x = x->data; k.codes = keep->codes; k.powers = keep->powers; k.x_worker = x->s_worker; k.x_batch = x->s_batch; k.x_row = x->s_place;
        k.batch = (uint32_t)shape->batch; k.rows = a.places; k.n_rows = a.samples * a.places; k.cols = a.channels; k.blocks = kept_blocks(a.channels);
        k.top = kept_top(shape->dtype);
        QGX_HIP(ctx, launch_checkpoint(shape->dtype, k, kept_draws(ctx, keep, unbiased, call_id), ctx->d_sc, (hipStream_t)stream));
    }
    QGX_HIP(ctx, launch_group_norm(shape->dtype, a, (uint32_t)shape->workers, plan, ctx->d_sc, (hipStream_t)stream));
    return QGX_OK;
}

qgx_status qgx_group_norm_backward(qgx_ctx* ctx, const qgx_group_shape* shape, const qgx_places* dy, const qgx_places* x, const qgx_kept* kept,
                                   const float* weight, const float* bias, const float* mean, const float* rstd, const qgx_places* dx,
                                   float* dweight, float* dbias, uint64_t param_stride, void* scratch, uint64_t scratch_bytes, void* stream)
{
    qgx_status s = check_group(ctx, "qgx_group_norm_backward", shape);
    if (s != QGX_OK) return s;
    if (!x == !kept) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_backward: either x or what was kept of it");
    if (kept) s = check_kept(ctx, "qgx_group_norm_backward", kept, shape->workers * shape->batch * shape->places, shape->channels);
    if (s != QGX_OK || shape->workers == 0) return s;
    if (!no_places(shape)) {
        if (!dy || !mean || !rstd) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_backward: null dy, mean or rstd");
        s = check_places(ctx, "qgx_group_norm_backward(dy)", shape, dy, false);
        if (s == QGX_OK && x) s = check_places(ctx, "qgx_group_norm_backward(x)", shape, x, false);
        if (s == QGX_OK && dx) s = check_places(ctx, "qgx_group_norm_backward(dx)", shape, dx, true);
        if (s != QGX_OK) return s;
        if (dx && (dx->data == dy->data || (x && dx->data == x->data))) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_backward: dx may not be dy or x");
    }
    if ((dweight || dbias) && shape->workers > 1 && param_stride < shape->channels)
        return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_backward: param_stride below channels");
    if (param_stride >= (1ull << 62) / shape->workers) return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_backward: stride out of range");
    if (!aligned_to(weight, 4u) || !aligned_to(bias, 4u) || !aligned_to(mean, 4u) || !aligned_to(rstd, 4u) || !aligned_to(dweight, 4u) || !aligned_to(dbias, 4u))
        return fail(ctx, QGX_ERR_ARG, "qgx_group_norm_backward: binary32 buffers must be 4-byte aligned");
    GroupPlan plan{};
    if (!no_places(shape)) s = plan_of(ctx, "qgx_group_norm_backward", shape, true, plan);
    if (s == QGX_OK) s = check_group_scratch(ctx, "qgx_group_norm_backward", plan, scratch, scratch_bytes);
    if (s != QGX_OK) return s;
    GroupArgs a = group_args(shape);
    if (!no_places(shape)) {
        a.dy = dy->data; a.dy_worker = dy->s_worker; a.dy_batch = dy->s_batch; a.dy_place = dy->s_place;
        if (x) {
            a.x = x->data; a.x_worker = x->s_worker; a.x_batch = x->s_batch; a.x_place = x->s_place;
        } else {
            a.codes = kept->codes; a.powers = kept->powers; a.power_place = kept_blocks(shape->channels); a.code_place = a.power_place * QGX_KEPT_BLOCK;
        }
        if (dx) { a.y = dx->data; a.y_worker = dx->s_worker; a.y_batch = dx->s_batch; a.y_place = dx->s_place; }
    }
    a.w = weight; a.b = bias; a.mean_in = mean; a.rstd_in = rstd; a.dw = dweight; a.db = dbias; a.param_stride = param_stride; a.scratch = (float*)scratch;
    QGX_HIP(ctx, launch_group_norm_back(shape->dtype, a, (uint32_t)shape->workers, plan, (hipStream_t)stream));
    return QGX_OK;
}

static qgx_status check_heads(qgx_ctx* ctx, const char* what, const qgx_heads* h, bool written)
{
    if (!known_type(h->dtype)) return fail(ctx, QGX_ERR_ARG, "%s: unknown type", what);
    if (h->heads == 0 || h->heads > 65535u || h->dim == 0 || h->dim > 4096u || h->workers >= (1ull << 31) || h->batch >= (1ull << 31) || h->tokens >= (1ull << 31) ||
        (h->workers && h->batch && h->tokens && (h->workers * h->batch >= (1ull << 31) || h->workers * h->batch * h->tokens >= (1ull << 31))))
        return fail(ctx, QGX_ERR_ARG, "%s: size out of range", what);
    if (h->workers == 0 || h->batch == 0 || h->tokens == 0) return QGX_OK;
    if (!h->data || !aligned_to(h->data, element_size(h->dtype))) return fail(ctx, QGX_ERR_ARG, "%s: null or misaligned", what);
    const uint64_t n[4] = {h->workers, h->batch, h->tokens, h->heads}, st[4] = {h->s_worker, h->s_batch, h->s_token, h->s_head};
    for (int i = 0; i < 4; ++i)
        if (st[i] >= (1ull << 60) / n[i]) return fail(ctx, QGX_ERR_ARG, "%s: stride out of range", what);
    if (written && !steps_apart(n, st, 4, h->dim)) return fail(ctx, QGX_ERR_ARG, "%s: heads overlap", what);
    return QGX_OK;
}

qgx_status qgx_rotate(qgx_ctx* ctx, const qgx_rotary* rotary, const int32_t* positions, uint64_t p_axis, uint64_t p_worker, uint64_t p_batch,
                      const qgx_heads* in, const qgx_heads* out, int back, void* stream)
{
    if (!ctx || !rotary || !in || !out || !rotary->frequencies) return fail(ctx, QGX_ERR_ARG, "qgx_rotate: null argument");
    if (rotary->axes == 0 || rotary->axes > QGX_MAX_AXES) return fail(ctx, QGX_ERR_ARG, "qgx_rotate: 1 .. %u axes", QGX_MAX_AXES);
    RotaryArgs a{};
    uint64_t pairs = 0;
    for (uint32_t i = 0; i < rotary->axes; ++i) {
        pairs += rotary->pairs[i];
        if (pairs > QGX_MAX_PAIRS) break;
        a.axis_end[i] = (uint32_t)pairs;
    }
    if (pairs == 0 || pairs > QGX_MAX_PAIRS) return fail(ctx, QGX_ERR_ARG, "qgx_rotate: 1 .. %u pairs", QGX_MAX_PAIRS);
    for (uint32_t i = rotary->axes; i < QGX_MAX_AXES; ++i) a.axis_end[i] = (uint32_t)pairs;
    for (uint32_t p = 0; p < pairs; ++p)
        if (!(std::fabs(rotary->frequencies[p]) <= DBL_MAX / 2147483648.0)) return fail(ctx, QGX_ERR_ARG, "qgx_rotate: frequency %u is not finite at every position", p);
    qgx_status s = check_heads(ctx, "qgx_rotate(in)", in, false);
    if (s == QGX_OK) s = check_heads(ctx, "qgx_rotate(out)", out, true);
    if (s != QGX_OK) return s;
    if (in->dtype != out->dtype || in->heads != out->heads || in->dim != out->dim || in->workers != out->workers || in->batch != out->batch || in->tokens != out->tokens)
        return fail(ctx, QGX_ERR_ARG, "qgx_rotate: in and out differ in type or shape");
    if (2u * pairs > in->dim) return fail(ctx, QGX_ERR_ARG, "qgx_rotate: %u pairs in heads of %u elements", (uint32_t)pairs, in->dim);
    if (in->workers == 0 || in->batch == 0 || in->tokens == 0) return QGX_OK;
    if (in->data == out->data && ((in->workers > 1 && in->s_worker != out->s_worker) || (in->batch > 1 && in->s_batch != out->s_batch) ||
                                  (in->tokens > 1 && in->s_token != out->s_token) || (in->heads > 1 && in->s_head != out->s_head)))
        return fail(ctx, QGX_ERR_ARG, "qgx_rotate: out at in's memory must have its strides");
    if (!positions || !aligned_to(positions, 4u)) return fail(ctx, QGX_ERR_ARG, "qgx_rotate: null or misaligned positions");
    if (p_axis >= (1ull << 58) || p_worker >= (1ull << 60) / in->workers || p_batch >= (1ull << 60) / in->batch)
        return fail(ctx, QGX_ERR_ARG, "qgx_rotate: stride of the positions out of range");
    a.in = in->data; a.out = out->data; a.positions = positions; a.p_axis = p_axis; a.p_worker = p_worker; a.p_batch = p_batch;
    a.i_worker = in->s_worker; a.i_batch = in->s_batch; a.i_token = in->s_token; a.i_head = in->s_head;
    a.o_worker = out->s_worker; a.o_batch = out->s_batch; a.o_token = out->s_token; a.o_head = out->s_head;
    a.batch = (uint32_t)in->batch; a.tokens = (uint32_t)in->tokens; a.heads = in->heads; a.dim = in->dim; a.pairs = (uint32_t)pairs;
    a.n_tokens = (uint32_t)(in->workers * in->batch * in->tokens);
    a.neighbours = rotary->neighbours != 0; a.back = back != 0;
    QGX_HIP(ctx, launch_rotary(in->dtype, a, rotary->frequencies, ctx->n_simd / 4u, (hipStream_t)stream));
    return QGX_OK;
}

uint32_t qgx_poll_error(qgx_ctx* ctx, void* stream)
{
    if (!ctx) return 0;
    hipStream_t st = (hipStream_t)stream;
    uint32_t e = 0;
    const uint32_t zero = 0;
    if (hipMemcpyAsync(&e, &ctx->d_sc->err, sizeof(e), hipMemcpyDeviceToHost, st) != hipSuccess) return QGX_EBIT_STATE;
    if (hipStreamSynchronize(st) != hipSuccess) return QGX_EBIT_STATE;
    if (e) {
        (void)hipMemcpyAsync(&ctx->d_sc->err, &zero, sizeof(zero), hipMemcpyHostToDevice, st);
        (void)hipStreamSynchronize(st);
    }
    return e;
}

const char* qgx_last_error(const qgx_ctx* ctx) { return ctx ? ctx->err : "null context"; }

}  // extern "C"
