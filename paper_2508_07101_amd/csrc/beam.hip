// Host side of beam search over paged caches: argument checks and launches.  Nothing here allocates or synchronises.
#include "host.hpp"

#include "beam_attn.hpp"
#include "beam_kernels.hpp"

using namespace cusa;

namespace {

cusa_status check_group(int32_t rows, int32_t width) {
    if (rows < 1 || width < 1 || rows % width != 0) return CUSA_ERR_INVALID_ARG;
    return rows > MAX_BATCH || width > BEAM_WIDTH ? CUSA_ERR_UNSUPPORTED : CUSA_OK;
}

cusa_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws || ((uintptr_t)ws & 255)) return CUSA_ERR_INVALID_ARG;
    return have < need ? CUSA_ERR_WORKSPACE_TOO_SMALL : CUSA_OK;
}

// Parts of a row, a wave each: enough waves for the chip, but parts of about 4 KB at least (3 KB where rows are little longer than a multiple of that; a last part is what is left), and a lane each where they come
// together.  (512 rows of 131072 bf16 logits: 1024 waves 47 us, 2048 35, 4096 31, 6144 35.  Selection and merge of 4 rows of 32000 for 8 places: parts of 2 KB 12.7, 4 KB 12.3, 8 KB 12.5; 52 rows of 67306 for 59 places 21.5, 19, 24; 256 rows of 32000 for 64 places 39, 36.5, 44.)
constexpr int PART_WAVES = 4096, PART_LEAST = 256;   // loads of 16 bytes
struct BeamParts {
    int parts, len;                        // len: loads of 16 bytes
};
BeamParts beam_parts(int32_t rows, int32_t vocab, int size) {
    const int64_t loads = std::max<int64_t>(1, ((int64_t)vocab * size + 15) / 16);
    const int64_t want = std::min<int64_t>({(loads + PART_LEAST - 1) / PART_LEAST, std::max(1, PART_WAVES / rows), 64});
    const int64_t len = ((loads + want - 1) / want + 63) / 64 * 64;
    return {(int)((loads + len - 1) / len), (int)len};
}

struct BeamWs {
    size_t sum, top, best, total;
};
BeamWs beam_ws(int32_t rows, int parts, int32_t n) {
    BeamWs w;
    w.sum = 0;
    w.top = align256((size_t)rows * parts * 8);
    w.best = w.top + align256((size_t)rows * parts * 4);
    w.total = w.best + align256((size_t)rows * parts * n * 8);
    return w;
}

template <int DTYPE>
void launch_rows(hipStream_t s, const BeamArgs& a) {
    const dim3 grid((unsigned)(((int64_t)a.rows * a.parts + BEAM_WAVES - 1) / BEAM_WAVES));
    // Eight loads a lane under way, or four where a part has no more.  (512 rows of 131072 bf16 logits: eight 31 us, four 35; parts of 4 KB: 256 rows of 32000 for 64 places 15 and 12.5, 52 rows of 67306 for 59 places 11.5 and 9.9.)
    if (a.part_len <= PART_LEAST) launch(KID_BEAM_ROWS, beam_rows_kernel<DTYPE, 4>, grid, 64 * BEAM_WAVES, 0, s, a);
    else launch(KID_BEAM_ROWS, beam_rows_kernel<DTYPE, 8>, grid, 64 * BEAM_WAVES, 0, s, a);
}

cusa_status check_beams(int32_t rows, int32_t vocab, int32_t n) {
    if (rows < 1 || vocab < 1 || n < 1) return CUSA_ERR_INVALID_ARG;
    return rows > MAX_BATCH || n > BEAM_MOST ? CUSA_ERR_UNSUPPORTED : CUSA_OK;
}

// Entries of a table that one workgroup changes.  (One launch and three, as a program sees them: 1100 entries 10.5 and 15.9 us, 4400 13.6 and 15.7, 4500 of short rows 15.5 and 16.1, 17000 27 and 16.)
constexpr int64_t FORK_ALL = 4096;

// Columns that a workgroup changes, PLAN_THREADS entries, in FORK_COLS columns at most.
constexpr int FORK_COLS = 256;
int fork_rows(int32_t width) { return width <= 4 ? 4 : width <= 8 ? 8 : width <= 16 ? 16 : 32; }
// Chunks of the columns that a row can have tokens in: lengths are 31 bits, and 2^30 columns would be more threads than a launch has.
int64_t chunks_of(int64_t max_pages, int cols) { return (std::min<int64_t>(max_pages, (0x7fffffff + (int64_t)PAGE - 1) / PAGE) + cols - 1) / cols; }

struct ForkWs {
    size_t rows, counts, freed, total;
};
ForkWs fork_ws(int32_t batch, int32_t max_pages) {
    const size_t chunks = (size_t)batch * chunks_of(max_pages, FORK_COLS);   // (a group of more than 4 rows has shorter chunks, but not more than FORK_COLS columns of each of its rows would be)
    ForkWs w;
    w.rows = 256;
    w.counts = w.rows + align256((size_t)batch * sizeof(ForkRow));
    w.freed = w.counts + align256(chunks * 4);
    w.total = w.freed + align256(chunks * FORK_COLS * 4);
    return w;
}

cusa_status check_shared(const cusa_shared* s, int32_t batch, int32_t max_seq_len, int64_t n_pages) {
    if (!s || !s->entries || !s->count || ((uintptr_t)s->entries & 15)) return CUSA_ERR_INVALID_ARG;
    const cusa_status st = check_group(batch, s->width);
    if (st != CUSA_OK) return st;
    const int64_t pages = ((int64_t)max_seq_len + PAGE - 1) / PAGE;
    return s->max_entries < std::min<int64_t>(s->width * pages, n_pages) ? CUSA_ERR_INVALID_ARG : CUSA_OK;
}

// Pages of a group that a pass may have to look at.
int64_t group_pages(const cusa_shared* s, int32_t max_seq_len) { return std::min<int64_t>(s->max_entries, s->width * (((int64_t)max_seq_len + PAGE - 1) / PAGE)); }

}  // namespace

extern "C" {

cusa_status cusa_beam_workspace_bytes(int32_t rows, int32_t vocab, int32_t n, size_t* bytes) {
    const cusa_status st = check_beams(rows, vocab, n);
    if (st != CUSA_OK) return st;
    if (!bytes) return CUSA_ERR_INVALID_ARG;
    *bytes = beam_ws(rows, std::max(beam_parts(rows, vocab, 2).parts, beam_parts(rows, vocab, 4).parts), n).total;   // of any type
    return CUSA_OK;
}

cusa_status cusa_beam_select(const cusa_beams* beams, const float* scores, const int32_t* ended, float* out_scores, int32_t* parents, int32_t* tokens,
                             int32_t* out_ended, void* ws, size_t ws_bytes, void* stream) {
    if (!beams) return CUSA_ERR_INVALID_ARG;
    cusa_status st = check_beams(beams->rows, beams->vocab, beams->n);
    if (st != CUSA_OK) return st;
    if ((st = check_group(beams->rows, beams->width)) != CUSA_OK) return st;
    if (!beams->logits || !scores || !out_scores || !parents || !tokens || beams->stride < beams->vocab) return CUSA_ERR_INVALID_ARG;
    if (beams->dtype != CUSA_BF16 && beams->dtype != CUSA_F16 && beams->dtype != CUSA_F32) return CUSA_ERR_INVALID_ARG;
    if ((uintptr_t)beams->logits & (beams->dtype == CUSA_F32 ? 3 : 1)) return CUSA_ERR_INVALID_ARG;
    if (beams->end_token < -1 || beams->end_token >= beams->vocab || (ended && beams->end_token < 0)) return CUSA_ERR_INVALID_ARG;
    if (beams->n != beams->width && (out_scores == scores || (out_ended && out_ended == ended))) return CUSA_ERR_INVALID_ARG;
    const BeamParts parts = beam_parts(beams->rows, beams->vocab, beams->dtype == CUSA_F32 ? 4 : 2);
    const BeamWs w = beam_ws(beams->rows, parts.parts, beams->n);
    if ((st = check_workspace(ws, ws_bytes, w.total)) != CUSA_OK) return st;
    BeamArgs a = {};
    a.logits = beams->logits;
    a.stride = beams->stride;
    a.scores = scores;
    a.ended = ended;
    a.out_scores = out_scores;
    a.parents = parents;
    a.tokens = tokens;
    a.out_ended = out_ended;
    a.sum = ws_ptr<double>(ws, w.sum);
    a.top = ws_ptr<float>(ws, w.top);
    a.best = ws_ptr<uint64_t>(ws, w.best);
    a.rows = beams->rows;
    a.width = beams->width;
    a.vocab = beams->vocab;
    a.n = beams->n;
    a.end_token = beams->end_token;
    a.parts = parts.parts;
    a.part_len = parts.len;
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (beams->dtype) {
        case CUSA_BF16: launch_rows<CUSA_BF16>(s, a); break;
        case CUSA_F16: launch_rows<CUSA_F16>(s, a); break;
        default: launch_rows<CUSA_F32>(s, a); break;
    }
    if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    launch(KID_BEAM_MERGE, beam_merge_kernel, dim3((unsigned)(beams->rows / beams->width)), 64 * MERGE_WAVES, 0, s, a);
    return launch_status();
}

size_t cusa_kv_fork_workspace_bytes(int32_t batch, int32_t max_pages) {
    return batch < 1 || batch > MAX_BATCH || max_pages < 1 || (int64_t)batch * max_pages > 0x7fffffff ? 0 : fork_ws(batch, max_pages).total;
}

cusa_status cusa_kv_fork(const cusa_pool* pool, int32_t width, const int32_t* held, const int32_t* parents, const int32_t* ended, int32_t grow, int32_t* table_out,
                         int32_t* lens, int64_t* slots, int32_t* copies, int32_t* granted, void* ws, size_t ws_bytes, void* stream) {
    cusa_status st = check_pool(pool);
    if (st != CUSA_OK) return st;
    if (pool->layout != CUSA_KV_PAGED) return CUSA_ERR_UNSUPPORTED;
    if ((st = check_group(pool->batch, width)) != CUSA_OK) return st;
    if (!held || !parents || !table_out || !lens || !slots || !copies || ((uintptr_t)copies & 15) || lens == parents || lens == ended) return CUSA_ERR_INVALID_ARG;
    const ForkWs w = fork_ws(pool->batch, pool->max_pages);
    if ((st = check_workspace(ws, ws_bytes, w.total)) != CUSA_OK) return st;
    ForkArgs a = {};
    a.held = held;
    a.parents = parents;
    a.ended = ended;
    a.table = pool->block_table;
    a.table_out = table_out;
    a.lens = lens;
    a.ring = pool->ring;
    a.slots = slots;
    a.copies = copies;
    a.granted = granted;
    a.state = pool->state;
    a.state_out = pool->state_out;
    a.head = ws_ptr<ForkHead>(ws, 0);
    a.rows = ws_ptr<ForkRow>(ws, w.rows);
    a.counts = ws_ptr<int32_t>(ws, w.counts);
    a.freed = ws_ptr<int32_t>(ws, w.freed);
    a.batch = pool->batch;
    a.width = width;
    a.max_pages = pool->max_pages;
    a.n_pages = (int32_t)pool->n_pages;
    a.cap = (int32_t)std::min<int64_t>((int64_t)pool->max_pages * PAGE, 0x7fffffff);
    a.grow = grow != 0;
    a.cols = PLAN_THREADS / fork_rows(width);
    a.chunks = (int32_t)chunks_of(pool->max_pages, a.cols);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (width <= FORK_ALL_WIDTH && a.batch <= PLAN_THREADS && (int64_t)a.batch * a.max_pages <= FORK_ALL) {
        launch(KID_KV_FORK, kv_fork_kernel<true>, 1, PLAN_THREADS, 0, s, a);
        return launch_status();
    }
    launch(KID_KV_FORK, kv_fork_kernel<false>, 1, PLAN_THREADS, 0, s, a);
    if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    const auto tables = width <= 4 ? fork_tables_kernel<4> : width <= 8 ? fork_tables_kernel<8> : width <= 16 ? fork_tables_kernel<16> : fork_tables_kernel<32>;
    launch(KID_FORK_TABLES, tables, dim3((unsigned)a.chunks, (unsigned)(a.batch / width)), PLAN_THREADS, 0, s, a);
    if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    launch(KID_FORK_PAGES, fork_pages_kernel, 1, PLAN_THREADS, 0, s, a);
    return launch_status();
}

cusa_status cusa_kv_copy(const cusa_params* params, int32_t n_layers, const cusa_kv* kv_layers, const int32_t* copies, int32_t n, void* stream) {
    cusa_status st = check_params(params, false);
    if (st != CUSA_OK) return st;
    if (n_layers < 1 || !kv_layers || n < 0 || (n > 0 && !copies) || ((uintptr_t)copies & 15)) return CUSA_ERR_INVALID_ARG;
    for (int i = 0; i < n_layers; ++i) {
        cusa_kv c = kv_layers[i];
        c.max_seq_len = 1;                 // not read
        if (c.layout == CUSA_KV_CONTIGUOUS) return CUSA_ERR_UNSUPPORTED;
        if ((st = check_cache(params, &c, false)) != CUSA_OK) return st;
    }
    if (n == 0) return CUSA_OK;
    if (n > COPY_MOST) return CUSA_ERR_UNSUPPORTED;
    CopyArgs a = {};
    a.copies = copies;
    a.G = params->n_kv_heads;
    for (int i = 0; i < n_layers; i += COPY_LAYERS) {
        const int m = std::min(n_layers - i, COPY_LAYERS);
        for (int j = 0; j < m; ++j) {
            const cusa_kv& c = kv_layers[i + j];
            a.layer[j] = {static_cast<uint16_t*>(const_cast<void*>(c.k)), static_cast<uint16_t*>(const_cast<void*>(c.v)), (int32_t)c.n_pages};
        }
        launch(KID_KV_COPY, kv_copy_kernel, dim3((unsigned)n, (unsigned)m), COPY_THREADS, 0, static_cast<hipStream_t>(stream), a);
        if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    }
    return CUSA_OK;
}

size_t cusa_shared_pages_workspace_bytes(int32_t batch, int32_t max_seq_len) { return batch < 1 || batch > MAX_BATCH || max_seq_len < 1 ? 0 : 256; }

cusa_status cusa_shared_pages(const cusa_kv* kv, int32_t batch, const cusa_shared* shared, void* ws, size_t ws_bytes, void* stream) {
    if (!kv || !kv->block_table || !kv->seq_lens || kv->max_seq_len < 1 || kv->n_pages < 1) return CUSA_ERR_INVALID_ARG;
    if (kv->layout != CUSA_KV_PAGED && kv->layout != CUSA_KV_CONTIGUOUS) return CUSA_ERR_INVALID_ARG;
    if (kv->layout != CUSA_KV_PAGED || kv->page_size != PAGE || kv->n_pages > 0x7fffffff || kv->max_seq_len > (1 << 30)) return CUSA_ERR_UNSUPPORTED;
    if ((int64_t)kv->max_pages * PAGE < kv->max_seq_len) return CUSA_ERR_INVALID_ARG;
    cusa_status st = check_shared(shared, batch, kv->max_seq_len, kv->n_pages);
    if (st != CUSA_OK) return st;
    if ((st = check_workspace(ws, ws_bytes, cusa_shared_pages_workspace_bytes(batch, kv->max_seq_len))) != CUSA_OK) return st;
    SharedArgs a = {};
    a.table = kv->block_table;
    a.lens = kv->seq_lens;
    a.entries = shared->entries;
    a.count = shared->count;
    a.batch = batch;
    a.width = shared->width;
    a.max_pages = kv->max_pages;
    a.n_pages = (int32_t)kv->n_pages;
    a.max_len = kv->max_seq_len;
    a.max_entries = shared->max_entries;
    const auto kernel = a.width <= 1 ? shared_pages_kernel<1> : a.width <= 2 ? shared_pages_kernel<2> : a.width <= 4 ? shared_pages_kernel<4> : a.width <= 8 ? shared_pages_kernel<8> : a.width <= 16 ? shared_pages_kernel<16> : shared_pages_kernel<32>;
    launch(KID_SHARED_PAGES, kernel, dim3((unsigned)(batch / a.width)), SHARED_THREADS, 0, static_cast<hipStream_t>(stream), a);
    return launch_status();
}

cusa_status cusa_beam_attn_workspace_bytes(const cusa_params* params, int32_t max_seq_len, const cusa_shared* shared, size_t* bytes) {
    cusa_status st = check_params(params, false);
    if (st != CUSA_OK) return st;
    if (!bytes || max_seq_len < 1 || !shared || shared->max_entries < 1) return CUSA_ERR_INVALID_ARG;
    if ((st = check_group(params->batch, shared->width)) != CUSA_OK) return st;
    const int64_t pages = group_pages(shared, max_seq_len);
    if (!beam_pages_served(pages)) return CUSA_ERR_UNSUPPORTED;
    const int groups = params->batch / shared->width, g = params->n_q_heads / params->n_kv_heads;
    const BeamPlan pl = plan_beams(pages, groups, params->n_kv_heads, shared->width * g);
    if (!beam_units_served(beam_units(pl, groups, params->n_kv_heads))) return CUSA_ERR_UNSUPPORTED;
    *bytes = beam_attn_workspace(pl, params->batch, params->n_q_heads, groups).total;
    return CUSA_OK;
}

cusa_status cusa_beam_attn(const cusa_params* params, const void* q, int64_t q_stride, const cusa_kv* kv, const cusa_shared* shared, void* out,
                           void* ws, size_t ws_bytes, void* stream) {
    cusa_status st = check_params(params, false);
    if (st != CUSA_OK) return st;
    if (!kv) return CUSA_ERR_INVALID_ARG;
    if (kv->layout == CUSA_KV_CONTIGUOUS) return CUSA_ERR_UNSUPPORTED;
    if (!kv->seq_lens) return CUSA_ERR_INVALID_ARG;
    if ((st = check_cache(params, kv, false)) != CUSA_OK) return st;
    if (!q || !out || ((uintptr_t)q & 15) || ((uintptr_t)out & 15) || q_stride < (int64_t)params->n_q_heads * D || (q_stride & 7)) return CUSA_ERR_INVALID_ARG;
    if ((st = check_shared(shared, params->batch, kv->max_seq_len, kv->n_pages)) != CUSA_OK) return st;
    const int g = params->n_q_heads / params->n_kv_heads, G = params->n_kv_heads, width = shared->width, groups = params->batch / width;
    const int64_t pages = group_pages(shared, kv->max_seq_len);
    if (!beam_pages_served(pages)) return CUSA_ERR_UNSUPPORTED;
    const BeamPlan pl = plan_beams(pages, groups, G, width * g);
    const int64_t units = beam_units(pl, groups, G);
    if (!beam_units_served(units)) return CUSA_ERR_UNSUPPORTED;
    const BeamAttnWs w = beam_attn_workspace(pl, params->batch, params->n_q_heads, groups);
    if ((st = check_workspace(ws, ws_bytes, w.total)) != CUSA_OK) return st;
    BeamAttnArgs a = {};
    a.cache = cache_args(params, kv);
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.entries = shared->entries;
    a.count = shared->count;
    a.entry_stride = shared->max_entries;
    a.max_entries = (int32_t)pages;
    a.out = static_cast<uint16_t*>(out);
    a.part_acc = ws_ptr<float>(ws, w.acc);
    a.part_ml = ws_ptr<float>(ws, w.ml);
    a.pieces = ws_ptr<int32_t>(ws, w.pieces);
    a.scale_log2e = params->sm_scale * 1.4426950408889634f;
    a.groups = groups;
    a.width = width;
    a.H = params->n_q_heads;
    a.g_shift = g == 1 ? 0 : g == 2 ? 1 : g == 4 ? 2 : 3;
    a.blocks = pl.blocks;
    a.n_splits = pl.n_splits;
    const dim3 grid((unsigned)units);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (width * g <= 16) launch(KID_BEAM_ATTN, beam_attn_kernel<1>, grid, BEAM_ATTN_THREADS, 0, s, a);
    else launch(KID_BEAM_ATTN, beam_attn_kernel<2>, grid, BEAM_ATTN_THREADS, 0, s, a);
    if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    if (pl.n_splits > 1) {                 // as many workgroups as have a row each, but not more than a few rounds of the chip
        const int64_t rows = ((int64_t)width * params->n_q_heads + BEAM_REDUCE_WAVES - 1) / BEAM_REDUCE_WAVES, most = std::max(1, 8192 / groups);
        launch(KID_BEAM_REDUCE, beam_reduce_kernel, dim3((unsigned)std::min(rows, most), (unsigned)groups), 64 * BEAM_REDUCE_WAVES, 0, s, a);
    }
    return launch_status();
}

}  // extern "C"
