// C-ABI of the backend operators: argument checks, workspace layout, launches.
#include <cstdio>
#include <new>
#include <string>

#include "backend.cuh"

using namespace wwws;

struct wwws_backend {
    wwws_backend_config cfg;
    cudaStream_t stream;
    int device;
    AttendScratch scratch;
    unsigned long long* best; uint32_t* row_ticket;
    uint32_t* owner; uint32_t* need;      // of wwws_pages_fork
    uint32_t* err;
    std::string text;
};

namespace {

thread_local std::string g_text;

wwws_status fail(wwws_backend* b, wwws_status st, const std::string& msg)
{
    (b ? b->text : g_text) = msg;
    return st;
}

struct DeviceScope {     // the backend's GPU for the duration of a call, the caller's afterwards
    int prev = -1; bool switched = false; cudaError_t err;
    explicit DeviceScope(int want)
    {
        err = cudaGetDevice(&prev);
        if (err == cudaSuccess && prev != want) { err = cudaSetDevice(want); switched = err == cudaSuccess; }
    }
    ~DeviceScope() { if (switched) cudaSetDevice(prev); }
    DeviceScope(const DeviceScope&) = delete;
    DeviceScope& operator=(const DeviceScope&) = delete;
};
#define ON_DEVICE(b)                                                                             \
    DeviceScope device_scope_((b)->device);                                                      \
    if (device_scope_.err != cudaSuccess)                                                        \
        return fail(b, WWWS_ERR_CUDA, std::string("selecting the backend's device: ") + cudaGetErrorString(device_scope_.err))

const char* check_config(const wwws_backend_config* c)
{
    if (!c) return "config is NULL";
    if (c->max_rows > 65535) return "max_rows must be <= 65535";
    if (c->n_heads == 0) return c->max_rows ? nullptr : "n_heads and max_rows are both 0: nothing to do";
    if (c->n_kv_heads == 0 || c->n_heads % c->n_kv_heads) return "n_heads must be a multiple of n_kv_heads";
    if (c->n_heads / c->n_kv_heads > 16) return "n_heads / n_kv_heads must be <= 16";
    if (c->n_heads > 1024) return "n_heads must be <= 1024";
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return "page_tokens must be 16, 32, 64 or 128";
    if (c->n_pages == 0 || uint64_t(c->n_pages) * c->n_kv_heads * c->page_tokens >= (1ull << 31)) return "n_pages must be >= 1 and n_pages * n_kv_heads * page_tokens < 2^31";
    if (c->max_seqs < 1 || c->max_seqs > 2048) return "max_seqs must be 1..2048";
    if (c->max_tokens < 1 || c->max_tokens >= (1u << 27) || uint64_t(c->max_tokens) * c->n_kv_heads >= (1ull << 31)) return "max_tokens must be 1..2^27-1 and max_tokens * n_kv_heads < 2^31";
    if (c->max_pages < 1 || uint64_t(c->max_pages) * c->page_tokens >= (1u << 30)) return "max_pages must be >= 1 and max_pages * page_tokens < 2^30";
    if (uint64_t(c->max_pages) * c->page_tokens * c->n_kv_heads >= (1ull << 37)) return "max_pages * page_tokens * n_kv_heads must be < 2^37";
    if (c->dtype != WWWS_BF16 && c->dtype != WWWS_F16) return "dtype must be WWWS_BF16 or WWWS_F16";
    if (c->cache > WWWS_CACHE_E4M3) return "cache must be a wwws_cache_kind";
    return nullptr;
}

uint64_t carve(const wwws_backend_config& c, uint8_t* base, wwws_backend* b)
{
    uint64_t off = 0;
    auto take = [&](uint64_t bytes) { off = (off + 255) & ~uint64_t(255); uint8_t* p = base ? base + off : nullptr; off += bytes; return p; };
    // what has to start at zero comes first
    uint8_t* err = take(256);
    uint8_t* best = take(8ull * c.max_rows);
    uint8_t* row_ticket = take(4ull * c.max_rows);
    constexpr uint64_t kRowSlots = uint64_t(kDecodeSlots) * kDecodeRows, kTileRows = uint64_t(kTileSlots) * 256, rows = kRowSlots > kTileRows ? kRowSlots : kTileRows;
    uint8_t* ticket = c.n_heads ? take(sizeof(uint32_t) * kTickets) : nullptr;
    uint8_t* part_ml = c.n_heads ? take(8 * rows) : nullptr;
    uint8_t* part_o = c.n_heads ? take(4 * rows * c.head_dim) : nullptr;
    uint8_t* owner = c.n_heads ? take(4ull * c.n_pages) : nullptr;
    uint8_t* need = c.n_heads ? take(4ull * c.max_seqs) : nullptr;
    if (b) {
        b->err = reinterpret_cast<uint32_t*>(err);
        b->best = reinterpret_cast<unsigned long long*>(best);
        b->row_ticket = reinterpret_cast<uint32_t*>(row_ticket);
        b->owner = reinterpret_cast<uint32_t*>(owner);
        b->need = reinterpret_cast<uint32_t*>(need);
        b->scratch = AttendScratch{ reinterpret_cast<float*>(part_o), reinterpret_cast<float2*>(part_ml), reinterpret_cast<uint32_t*>(ticket) };
    }
    return (off + 255) & ~uint64_t(255);
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

const char* check_pages(const wwws_backend* b, const wwws_kv_pages* p)
{
    if (!p->k || !p->v || !aligned(p->k) || !aligned(p->v)) return "k and v pages must be given and 16-byte aligned";
    if (b->cfg.cache != WWWS_CACHE_16 && (!p->k_scale || !p->v_scale)) return "a quantised cache needs k_scale and v_scale";
    return nullptr;
}

const char* check_batch(const wwws_backend* b, const wwws_batch* s, const wwws_kv_pages* p)
{
    const wwws_backend_config& c = b->cfg;
    if (c.n_heads == 0) return "the backend was created without heads";
    if (!s || !p) return "batch or pages is NULL";
    if (s->n_seqs > c.max_seqs) return "n_seqs exceeds max_seqs";
    if (s->n_tokens > c.max_tokens) return "n_tokens exceeds max_tokens";
    if (s->max_q_len > s->n_tokens) return "max_q_len exceeds n_tokens";
    if (uint64_t(s->max_kv_len) > uint64_t(c.max_pages) * c.page_tokens) return "max_kv_len exceeds the page table";
    if (s->n_seqs && (!s->kv_len || !s->page_table)) return "a batch array is NULL";
    return check_pages(b, p);
}

const char* check_layers(const wwws_backend* b, const wwws_kv_pages* layers, uint32_t n)
{
    if (b->cfg.n_heads == 0) return "the backend was created without heads";
    if (!layers && n) return "layers is NULL";
    if (n > 65535) return "n_layers must be <= 65535";
    for (uint32_t i = 0; i < n; ++i) if (const char* m = check_pages(b, layers + i)) return m;
    return nullptr;
}

const char* check_rotation(const wwws_backend* b, const wwws_rotation* r)
{
    if (!r || !r->turns) return "rotation or its turns is NULL";
    if (reinterpret_cast<uintptr_t>(r->turns) & 7) return "turns must be 8-byte aligned";
    if (r->dim < 16 || r->dim % 16 || r->dim > b->cfg.head_dim) return "a rotation's dim must be a multiple of 16, 16 .. head_dim";
    if (r->n_axes < 1 || r->n_axes > 8) return "a rotation's n_axes must be 1..8";
    if (r->interleaved > 1) return "a rotation's interleaved must be 0 or 1";
    if (!(r->eps >= 0.0f) || !(r->eps - r->eps == 0.0f)) return "a rotation's eps must be finite and >= 0";
    if (!aligned(r->q_weight) || !aligned(r->k_weight)) return "a rotation's weights must be 16-byte aligned";
    return nullptr;
}

const char* check_rows(const void* p, uint64_t stride, uint32_t heads, uint32_t dim)
{
    if (!p || !aligned(p)) return "an array of rows is NULL or not 16-byte aligned";
    if (stride % 8 || stride < uint64_t(heads) * dim) return "a stride must be a multiple of 8 and cover a token's heads";
    if (stride >= (1ull << 32)) return "a stride must be < 2^32";
    return nullptr;
}

SeqBatch seqs_of(const wwws_backend* b, const wwws_batch* s)
{
    return SeqBatch{ s->q_start, s->kv_len, s->page_table, s->n_seqs, s->n_tokens, s->max_q_len, s->max_kv_len, b->cfg.max_pages, 3 };
}

Pages pages_of(const wwws_backend* b, const wwws_kv_pages* p)
{
    uint32_t shift = 4;
    while ((1u << shift) < b->cfg.page_tokens) ++shift;
    return Pages{ static_cast<uint8_t*>(p->k), static_cast<uint8_t*>(p->v), p->k_scale, p->v_scale, b->cfg.n_pages, b->cfg.n_kv_heads, shift };
}

// One launch for every kMaxLayers layers.
template <class F> wwws_status by_layers(wwws_backend* b, const wwws_kv_pages* layers, uint32_t n, const char* what, F&& launch)
{
    LayerArgs a{};
    uint32_t shift = 4;
    while ((1u << shift) < b->cfg.page_tokens) ++shift;
    a.n_pages = b->cfg.n_pages; a.n_kv_heads = b->cfg.n_kv_heads; a.page_shift = shift; a.err = b->err;
    a.row_bytes = b->cfg.head_dim * (b->cfg.cache == WWWS_CACHE_16 ? 2 : 1);
    cudaError_t e = cudaSuccess;
    for (uint32_t first = 0; e == cudaSuccess && first < n; first += kMaxLayers) {
        const uint32_t some = n - first < kMaxLayers ? n - first : kMaxLayers;
        for (uint32_t i = 0; i < some; ++i) {
            const wwws_kv_pages& p = layers[first + i];
            const bool scales = b->cfg.cache != WWWS_CACHE_16;
            a.layer[i] = Layer{ static_cast<uint8_t*>(p.k), static_cast<uint8_t*>(p.v), scales ? p.k_scale : nullptr, scales ? p.v_scale : nullptr };
        }
        e = launch(a, some);
    }
    if (e == cudaSuccess) return WWWS_OK;
    return fail(b, WWWS_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

wwws_status launched(wwws_backend* b, cudaError_t e, const char* what)
{
    if (e == cudaSuccess) return WWWS_OK;
    return fail(b, WWWS_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// Attention of the batch's new tokens; `tree`: NULL, or the masks of wwws_attend_tree.
wwws_status attend(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* q, uint64_t q_stride, void* out, uint64_t out_stride, float scale, uint32_t window, uint32_t sinks,
                   const uint32_t* tree, uint32_t tree_words)
{
    if (const char* m = check_batch(b, batch, pages)) return fail(b, WWWS_ERR_ARG, m);
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return WWWS_OK;
    if (!batch->q_start) return fail(b, WWWS_ERR_ARG, "q_start is NULL");
    if (const char* m = check_rows(q, q_stride, b->cfg.n_heads, b->cfg.head_dim)) return fail(b, WWWS_ERR_ARG, m);
    if (const char* m = check_rows(out, out_stride, b->cfg.n_heads, b->cfg.head_dim)) return fail(b, WWWS_ERR_ARG, m);
    if (!(scale - scale == 0.0f)) return fail(b, WWWS_ERR_ARG, "scale must be finite");
    ON_DEVICE(b);
    AttendArgs a{};
    a.b = seqs_of(b, batch); a.p = pages_of(b, pages); a.s = b->scratch;
    a.q = static_cast<const uint8_t*>(q); a.out = static_cast<uint8_t*>(out); a.q_stride = q_stride; a.out_stride = out_stride;
    a.group = b->cfg.n_heads / b->cfg.n_kv_heads;
    a.scale_log2 = float(double(scale) * 1.4426950408889634);
    // a product that has to keep -infinity at hidden keys: the smallest normal number stands for 0 (scores of any size times it are below 4)
    if (a.scale_log2 == 0.0f) a.scale_log2 = 0x1p-126f;
    a.window = window < batch->max_kv_len ? window : 0;          // one that hides nothing is none
    a.sinks = sinks < batch->max_kv_len ? sinks : batch->max_kv_len;
    a.err = b->err;
    a.tree = tree; a.tree_words = tree_words;
    // A call goes by the rows per kv head (new tokens * group) of its longest sequence: few to the row kernel, which reads the cache once per 16 rows, more to
    // the tile kernel.  24 requests of 3,000 tokens, row kernel / tile kernel in us: 16-bit cache at head_dim 64, 30 rows 36 / 42, 36 rows 46 / 42, at 128 58 / 54 and
    // 73 / 53; e4m3 at 64, 48 rows 48 / 56, 60 rows 62 / 56, at 128 61 / 77 and 79 / 79; int8 at 64 50 / 60 and 65 / 62, at 128 66 / 91 and 87 / 91.  (One request of
    // 60,000 tokens would favour the row kernel beyond these: 60 rows at 128 84 / 92 in 16 bits, 70 / 95 in e4m3.)
    const uint32_t few_rows = b->cfg.cache == WWWS_CACHE_16 ? kFewRows : kFewRowsQuant;
    const uint64_t most = uint64_t(batch->max_q_len) * a.group;
    if (tree) {
        // The same with the tree kernel for the tile kernel (the figures are that one's; the tree kernel has not been held against the row kernel).  It counts tiles in
        // 31 bits: a launch takes as many sequences as the bounds allow to fit, and what does not fit even alone goes to the row kernel.
        const uint64_t tiles = ((uint64_t(batch->max_kv_len) + 127) / 128 + 4) * ((most + 63) / 64) * b->cfg.n_kv_heads;       // of a sequence, at most, with its units' fixed cost
        const uint64_t fit = most <= few_rows ? 0 : ((1ull << 31) - 1) / tiles;
        if (fit == 0) return launched(b, launch_attend_rows_tree(a, uint32_t(most), b->cfg.head_dim, b->cfg.dtype, b->cfg.cache, b->stream), "wwws_attend_tree");
        const uint32_t at_once = uint32_t(fit < kTreeSeqs ? fit : kTreeSeqs);
        cudaError_t e = cudaSuccess;
        for (uint32_t first = 0; e == cudaSuccess && first < batch->n_seqs; first += at_once) {
            a.b.q_start = batch->q_start + first; a.b.kv_len = batch->kv_len + first; a.b.page_table = batch->page_table + uint64_t(first) * b->cfg.max_pages;
            a.b.n_seqs = batch->n_seqs - first < at_once ? batch->n_seqs - first : at_once;
            a.b.ends = (first == 0 ? 1u : 0u) | (first + a.b.n_seqs == batch->n_seqs ? 2u : 0u);
            e = launch_tree(a, b->cfg.head_dim, b->cfg.dtype, b->cfg.cache, b->stream);
        }
        return launched(b, e, "wwws_attend_tree");
    }
    if (most <= few_rows) return launched(b, launch_attend_rows(a, uint32_t(most), b->cfg.head_dim, b->cfg.dtype, b->cfg.cache, b->stream), "wwws_attend");
    // Short sequences beside long ones stay with the tile kernel.  They went to the row kernel in a second launch, and two such pairs of launches ended in a fault of
    // the GPU (129 sequences of both kinds, and a form of the tile kernel with masks over 22) that neither reading nor checks of every access in memory explained.
    // So a call has one kernel for all its sequences, none of which it leaves out.  32 a launch is what the tile kernel has been run with in every mixture; whether the
    // number matters is not known.  (63 single tokens beside a chunk of 512, 32 on 8 heads of 128: 160 us, over 8-bit caches 295 to 311; in calls of their own 86 + 43, 63 to 65 + 66 to 68.)
    cudaError_t e = cudaSuccess;
    for (uint32_t first = 0; e == cudaSuccess && first < batch->n_seqs; first += kTileSeqs) {
        a.b.q_start = batch->q_start + first; a.b.kv_len = batch->kv_len + first; a.b.page_table = batch->page_table + uint64_t(first) * b->cfg.max_pages;
        a.b.n_seqs = batch->n_seqs - first < kTileSeqs ? batch->n_seqs - first : kTileSeqs;
        a.b.ends = (first == 0 ? 1u : 0u) | (first + a.b.n_seqs == batch->n_seqs ? 2u : 0u);
        e = launch_attend_tile(a, b->cfg.head_dim, b->cfg.dtype, b->cfg.cache, b->stream);
    }
    return launched(b, e, "wwws_attend");
}

}  // namespace

extern "C" {

wwws_status wwws_backend_workspace_bytes(const wwws_backend_config* cfg, uint64_t* bytes_out)
{
    if (!bytes_out) return fail(nullptr, WWWS_ERR_ARG, "bytes_out is NULL");
    if (const char* m = check_config(cfg)) return fail(nullptr, WWWS_ERR_ARG, m);
    *bytes_out = carve(*cfg, nullptr, nullptr);
    return WWWS_OK;
}

wwws_status wwws_create_backend(const wwws_backend_config* cfg, void* workspace, uint64_t workspace_bytes, void* cuda_stream, wwws_backend** out)
{
    if (!out) return fail(nullptr, WWWS_ERR_ARG, "out is NULL");
    *out = nullptr;
    if (const char* m = check_config(cfg)) return fail(nullptr, WWWS_ERR_ARG, m);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255)) return fail(nullptr, WWWS_ERR_ALLOC, "workspace is NULL or not 256-byte aligned");
    if (carve(*cfg, nullptr, nullptr) > workspace_bytes) return fail(nullptr, WWWS_ERR_ALLOC, "workspace too small");
    cudaPointerAttributes wa;
    if (cudaError_t e = cudaPointerGetAttributes(&wa, workspace); e != cudaSuccess) {
        cudaGetLastError();
        return fail(nullptr, WWWS_ERR_CUDA, std::string("cudaPointerGetAttributes(workspace): ") + cudaGetErrorString(e));
    }
    if (wa.type != cudaMemoryTypeDevice && wa.type != cudaMemoryTypeManaged) return fail(nullptr, WWWS_ERR_ARG, "workspace is not device memory");
    wwws_backend* b = new (std::nothrow) wwws_backend();
    if (!b) return fail(nullptr, WWWS_ERR_ALLOC, "host allocation failed");
    b->cfg = *cfg; b->device = wa.device; b->stream = static_cast<cudaStream_t>(cuda_stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    carve(*cfg, ws, b);
    DeviceScope scope(b->device);
    cudaError_t e = scope.err;
    // the error word, the rows' words and the tickets start at zero and are left at zero by every call
    const uint64_t zeroed = cfg->n_heads ? reinterpret_cast<uint8_t*>(b->scratch.part_ml) - ws : reinterpret_cast<uint8_t*>(b->row_ticket) + 4ull * cfg->max_rows - ws;
    if (e == cudaSuccess) e = cudaMemsetAsync(ws, 0, zeroed, b->stream);
    if (e != cudaSuccess) {
        delete b;
        return fail(nullptr, WWWS_ERR_CUDA, std::string("preparing the workspace: ") + cudaGetErrorString(e));
    }
    *out = b;
    return WWWS_OK;
}

wwws_status wwws_destroy_backend(wwws_backend* b)
{
    if (!b) return WWWS_OK;
    { DeviceScope scope(b->device); cudaStreamSynchronize(b->stream); }
    delete b;
    return WWWS_OK;
}

wwws_status wwws_cache_append(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (const char* m = check_batch(b, batch, pages)) return fail(b, WWWS_ERR_ARG, m);
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return WWWS_OK;
    if (!batch->q_start) return fail(b, WWWS_ERR_ARG, "q_start is NULL");
    if (const char* m = check_rows(k, k_stride, b->cfg.n_kv_heads, b->cfg.head_dim)) return fail(b, WWWS_ERR_ARG, m);
    if (const char* m = check_rows(v, v_stride, b->cfg.n_kv_heads, b->cfg.head_dim)) return fail(b, WWWS_ERR_ARG, m);
    ON_DEVICE(b);
    return launched(b, launch_cache_append(seqs_of(b, batch), pages_of(b, pages), k, k_stride, v, v_stride, b->cfg.head_dim, b->cfg.dtype, b->cfg.cache, b->err, b->stream), "wwws_cache_append");
}

wwws_status wwws_cache_read(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const int32_t* row_start, uint64_t n_rows, void* k_out, void* v_out)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (const char* m = check_batch(b, batch, pages)) return fail(b, WWWS_ERR_ARG, m);
    if (n_rows >= (1ull << 31)) return fail(b, WWWS_ERR_ARG, "n_rows must be < 2^31");
    if (batch->n_seqs == 0 || n_rows == 0) return WWWS_OK;
    if (!row_start || !k_out || !v_out || !aligned(k_out) || !aligned(v_out)) return fail(b, WWWS_ERR_ARG, "row_start, k_out or v_out is NULL or not 16-byte aligned");
    ON_DEVICE(b);
    return launched(b, launch_cache_read(seqs_of(b, batch), pages_of(b, pages), row_start, n_rows, k_out, v_out, b->cfg.head_dim, b->cfg.dtype, b->cfg.cache, b->err, b->stream), "wwws_cache_read");
}

wwws_status wwws_attend(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* q, uint64_t q_stride, void* out, uint64_t out_stride, float scale, uint32_t window, uint32_t sinks)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    return attend(b, batch, pages, q, q_stride, out, out_stride, scale, window, sinks, nullptr, 0);
}

wwws_status wwws_attend_tree(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* q, uint64_t q_stride, void* out, uint64_t out_stride, float scale, uint32_t window, uint32_t sinks,
                             const uint32_t* tree, uint32_t tree_words)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (batch && batch->n_seqs && batch->n_tokens) {
        if (!tree || (reinterpret_cast<uintptr_t>(tree) & 3)) return fail(b, WWWS_ERR_ARG, "tree is NULL or not aligned to its words");
        if (uint64_t(tree_words) * 32 < batch->max_q_len) return fail(b, WWWS_ERR_ARG, "tree_words must cover max_q_len");
    }
    return attend(b, batch, pages, q, q_stride, out, out_stride, scale, window, sinks, tree, tree_words);
}

wwws_status wwws_rotate(wwws_backend* b, const wwws_rotation* rotation, uint32_t n_tokens, const int32_t* positions, const void* q, uint64_t q_stride, const void* k, uint64_t k_stride, void* q_out, uint64_t q_out_stride,
                        void* k_out, uint64_t k_out_stride)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    const wwws_backend_config& c = b->cfg;
    if (c.n_heads == 0) return fail(b, WWWS_ERR_ARG, "the backend was created without heads");
    if (const char* m = check_rotation(b, rotation)) return fail(b, WWWS_ERR_ARG, m);
    if (n_tokens >= (1u << 31)) return fail(b, WWWS_ERR_ARG, "n_tokens must be < 2^31");
    if (n_tokens == 0) return WWWS_OK;
    if (!positions) return fail(b, WWWS_ERR_ARG, "positions is NULL");
    for (const char* m : { check_rows(q, q_stride, c.n_heads, c.head_dim), check_rows(k, k_stride, c.n_kv_heads, c.head_dim), check_rows(q_out, q_out_stride, c.n_heads, c.head_dim),
                           check_rows(k_out, k_out_stride, c.n_kv_heads, c.head_dim), q == q_out && q_stride != q_out_stride ? "in place, both strides must be the same" : nullptr,
                           k == k_out && k_stride != k_out_stride ? "in place, both strides must be the same" : nullptr })
        if (m) return fail(b, WWWS_ERR_ARG, m);
    ON_DEVICE(b);
    RotateArgs a{};
    a.r = *rotation; a.positions = positions; a.n_tokens = n_tokens; a.n_heads = c.n_heads; a.n_kv_heads = c.n_kv_heads; a.err = b->err;
    a.q = static_cast<const uint8_t*>(q); a.k = static_cast<const uint8_t*>(k); a.q_out = static_cast<uint8_t*>(q_out); a.k_out = static_cast<uint8_t*>(k_out);
    a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
    return launched(b, launch_rotate(a, false, c.head_dim, c.dtype, c.cache, b->stream), "wwws_rotate");
}

wwws_status wwws_rotate_append(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const wwws_rotation* rotation, const int32_t* positions, const void* q, uint64_t q_stride, const void* k, uint64_t k_stride,
                               const void* v, uint64_t v_stride, void* q_out, uint64_t q_out_stride)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    const wwws_backend_config& c = b->cfg;
    if (const char* m = check_batch(b, batch, pages)) return fail(b, WWWS_ERR_ARG, m);
    if (const char* m = check_rotation(b, rotation)) return fail(b, WWWS_ERR_ARG, m);
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return WWWS_OK;
    if (!batch->q_start) return fail(b, WWWS_ERR_ARG, "q_start is NULL");
    for (const char* m : { check_rows(q, q_stride, c.n_heads, c.head_dim), check_rows(k, k_stride, c.n_kv_heads, c.head_dim), check_rows(v, v_stride, c.n_kv_heads, c.head_dim),
                           check_rows(q_out, q_out_stride, c.n_heads, c.head_dim), q == q_out && q_stride != q_out_stride ? "in place, both strides must be the same" : nullptr })
        if (m) return fail(b, WWWS_ERR_ARG, m);
    ON_DEVICE(b);
    RotateArgs a{};
    a.r = *rotation; a.b = seqs_of(b, batch); a.p = pages_of(b, pages); a.positions = positions; a.n_tokens = batch->n_tokens; a.n_heads = c.n_heads; a.n_kv_heads = c.n_kv_heads; a.err = b->err;
    a.q = static_cast<const uint8_t*>(q); a.k = static_cast<const uint8_t*>(k); a.v = static_cast<const uint8_t*>(v); a.q_out = static_cast<uint8_t*>(q_out);
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    return launched(b, launch_rotate(a, true, c.head_dim, c.dtype, c.cache, b->stream), "wwws_rotate_append");
}

wwws_status wwws_pages_fork(wwws_backend* b, const wwws_fork* f)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (b->cfg.n_heads == 0) return fail(b, WWWS_ERR_ARG, "the backend was created without heads");
    if (!f || !f->refs || !f->refs_out) return fail(b, WWWS_ERR_ARG, "fork or its refs is NULL");
    if (f->n_old > b->cfg.max_seqs || f->n_new > b->cfg.max_seqs) return fail(b, WWWS_ERR_ARG, "n_old or n_new exceeds max_seqs");
    if (f->n_old && (!f->table || !f->held)) return fail(b, WWWS_ERR_ARG, "table or held is NULL");
    if (f->n_new && (!f->source || !f->keep || !f->room || !f->table_out || !f->held_out || !f->moves)) return fail(b, WWWS_ERR_ARG, "an array of the new sequences is NULL");
    if (f->n_new && f->n_old && (f->table_out == f->table || f->held_out == f->held)) return fail(b, WWWS_ERR_ARG, "the new tables must not lie over the old ones");
    ON_DEVICE(b);
    ForkArgs a{};
    a.refs = f->refs; a.refs_out = f->refs_out; a.table = f->table; a.held = f->held; a.source = f->source; a.keep = f->keep; a.room = f->room;
    a.table_out = f->table_out; a.held_out = f->held_out; a.moves = f->moves; a.n_old = f->n_old; a.n_new = f->n_new;
    a.n_pages = b->cfg.n_pages; a.max_pages = b->cfg.max_pages; a.page_shift = 4;
    while ((1u << a.page_shift) < b->cfg.page_tokens) ++a.page_shift;
    a.owner = b->owner; a.need = b->need; a.err = b->err;
    return launched(b, launch_fork(a, b->stream), "wwws_pages_fork");
}

wwws_status wwws_cache_copy(wwws_backend* b, const wwws_kv_pages* layers, uint32_t n_layers, const int32_t* moves, uint32_t n_moves)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (const char* m = check_layers(b, layers, n_layers)) return fail(b, WWWS_ERR_ARG, m);
    if (n_layers == 0 || n_moves == 0) return WWWS_OK;
    if (!moves) return fail(b, WWWS_ERR_ARG, "moves is NULL");
    if (n_moves >= (1u << 31)) return fail(b, WWWS_ERR_ARG, "n_moves must be < 2^31");
    ON_DEVICE(b);
    return by_layers(b, layers, n_layers, "wwws_cache_copy", [&](const LayerArgs& a, uint32_t n) { return launch_copy_pages(a, n, moves, n_moves, b->stream); });
}

wwws_status wwws_cache_compact(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* layers, uint32_t n_layers, const int32_t* path, const int32_t* path_len, uint32_t path_stride)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (const char* m = check_layers(b, layers, n_layers)) return fail(b, WWWS_ERR_ARG, m);
    if (n_layers == 0) return WWWS_OK;
    if (const char* m = check_batch(b, batch, layers)) return fail(b, WWWS_ERR_ARG, m);
    if (path_stride > 2048) return fail(b, WWWS_ERR_ARG, "path_stride must be <= 2048");
    if (batch->n_seqs == 0 || path_stride == 0) return WWWS_OK;
    if (!batch->q_start || !path || !path_len) return fail(b, WWWS_ERR_ARG, "q_start, path or path_len is NULL");
    ON_DEVICE(b);
    return by_layers(b, layers, n_layers, "wwws_cache_compact", [&](const LayerArgs& a, uint32_t n) { return launch_compact(a, n, seqs_of(b, batch), path, path_len, path_stride, b->stream); });
}

wwws_status wwws_beams_scratch_bytes(uint32_t n_rows, uint32_t vocab, uint32_t dtype, uint32_t keep, uint64_t* bytes_out)
{
    if (!bytes_out) return fail(nullptr, WWWS_ERR_ARG, "bytes_out is NULL");
    if (n_rows > 65535 || vocab == 0 || vocab > (1u << 24) || dtype > WWWS_F32 || keep < 1 || keep > kMaxKeep) return fail(nullptr, WWWS_ERR_ARG, "n_rows must be <= 65535, vocab 1..2^24, dtype a wwws_dtype, keep 1..128");
    *bytes_out = beams_scratch(n_rows, vocab, int(dtype));
    return WWWS_OK;
}

wwws_status wwws_select_beams(wwws_backend* b, uint32_t n_rows, uint32_t beams, uint32_t vocab, uint32_t dtype, const void* logits, uint64_t stride, const float* total, uint32_t keep, void* scratch, uint64_t scratch_bytes,
                              float* score, int32_t* parent, int32_t* token)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (dtype > WWWS_F32) return fail(b, WWWS_ERR_ARG, "dtype must be a wwws_dtype");
    if (beams < 1 || beams > kMaxBeams || n_rows % beams) return fail(b, WWWS_ERR_ARG, "beams must be 1..256 and divide n_rows");
    if (keep < 1 || keep > kMaxKeep) return fail(b, WWWS_ERR_ARG, "keep must be 1..128");
    if (n_rows > b->cfg.max_rows) return fail(b, WWWS_ERR_ARG, "n_rows exceeds max_rows");
    if (vocab == 0 || vocab > (1u << 24)) return fail(b, WWWS_ERR_ARG, "vocab must be 1..2^24");
    if (n_rows == 0) return WWWS_OK;
    const uintptr_t size = dtype == WWWS_F32 ? 4 : 2;
    if (!logits || reinterpret_cast<uintptr_t>(logits) % size || stride < vocab) return fail(b, WWWS_ERR_ARG, "logits is NULL or not aligned to its elements, or its stride is below vocab");
    if (!total || !score || !parent || !token) return fail(b, WWWS_ERR_ARG, "total, score, parent or token is NULL");
    if (!scratch || !aligned(scratch) || scratch_bytes < beams_scratch(n_rows, vocab, int(dtype))) return fail(b, WWWS_ERR_ALLOC, "scratch is NULL, not 16-byte aligned or too small");
    ON_DEVICE(b);
    BeamArgs a{};
    a.in = static_cast<const uint8_t*>(logits); a.stride = stride; a.total = total; a.ticket = b->row_ticket; a.score = score; a.parent = parent; a.token = token;
    a.beams = beams; a.vocab = vocab; a.keep = keep;
    return launched(b, launch_beams(a, n_rows, int(dtype), scratch, b->stream), "wwws_select_beams");
}

wwws_status wwws_shape_logits(wwws_backend* b, const wwws_shaping* s, uint32_t n_rows, uint32_t vocab, uint32_t dtype, const void* logits, uint64_t stride, void* out, uint64_t out_stride, int32_t* token)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    if (!s) return fail(b, WWWS_ERR_ARG, "shaping is NULL");
    if (dtype > WWWS_F32) return fail(b, WWWS_ERR_ARG, "dtype must be a wwws_dtype");
    if (n_rows > b->cfg.max_rows) return fail(b, WWWS_ERR_ARG, "n_rows exceeds max_rows");
    if (vocab == 0 || vocab >= (1u << 30)) return fail(b, WWWS_ERR_ARG, "vocab must be 1..2^30-1");
    if (n_rows == 0) return WWWS_OK;
    const uintptr_t size = dtype == WWWS_F32 ? 4 : 2;
    if (!logits || !out || reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(out) % size) return fail(b, WWWS_ERR_ARG, "logits or out is NULL or not aligned to its elements");
    if (stride < vocab || out_stride < vocab) return fail(b, WWWS_ERR_ARG, "a stride must be >= vocab");
    if (logits == out && stride != out_stride) return fail(b, WWWS_ERR_ARG, "in place, both strides must be the same");
    if (s->history && !s->history_start) return fail(b, WWWS_ERR_ARG, "history needs history_start");
    if (s->bias_id && (!s->bias_value || !s->bias_start)) return fail(b, WWWS_ERR_ARG, "bias_id needs bias_value and bias_start");
    if (s->mask && uint64_t(s->mask_stride) * 32 < vocab) return fail(b, WWWS_ERR_ARG, "mask_stride must cover the vocabulary");
    if (s->mask && !s->mask_index && s->n_masks < n_rows) return fail(b, WWWS_ERR_ARG, "without mask_index there must be a mask per row");
    ON_DEVICE(b);
    ShapeArgs a{};
    a.s = *s;
    a.in = static_cast<const uint8_t*>(logits); a.out = static_cast<uint8_t*>(out); a.in_stride = stride; a.out_stride = out_stride;
    a.n_rows = n_rows; a.vocab = vocab;
    a.token = token; a.best = b->best; a.ticket = b->row_ticket; a.err = b->err;
    return launched(b, launch_shape_logits(a, int(dtype), b->stream), "wwws_shape_logits");
}

wwws_status wwws_backend_sync(wwws_backend* b)
{
    if (!b) return fail(nullptr, WWWS_ERR_ARG, "backend is NULL");
    ON_DEVICE(b);
    uint32_t bits = 0;
    cudaError_t e = cudaMemcpyAsync(&bits, b->err, sizeof bits, cudaMemcpyDeviceToHost, b->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(b->stream);
    if (e == cudaSuccess && bits) e = cudaMemsetAsync(b->err, 0, sizeof bits, b->stream);
    // blocks that gave up did not take their tickets: those of the next call start at zero all the same
    if (e == cudaSuccess && (bits & beTimeout) && b->scratch.ticket) e = cudaMemsetAsync(b->scratch.ticket, 0, kTickets * sizeof(uint32_t), b->stream);
    if (e != cudaSuccess) return launched(b, e, "wwws_backend_sync");
    if (bits == 0) return WWWS_OK;
    std::string text;
    if (bits & bePage) text += "a page id outside the pool; ";
    if (bits & beToken) text += "a token id outside the vocabulary; ";
    if (bits & beMask) text += "a mask index outside the masks; ";
    if (bits & bePool) text += "the page pool ran out; ";
    if (bits & beTimeout) return fail(b, WWWS_ERR_TIMEOUT, "a wait inside wwws_attend ran out; its results are not to be trusted");
    if (bits & beOffset) text += "offsets or lengths outside the batch's bounds; ";
    return fail(b, bits & (bePage | beToken | beMask) ? WWWS_ERR_INDEX : bits & bePool ? WWWS_ERR_ALLOC : WWWS_ERR_ARG, text + "what they named was skipped");
}

const char* wwws_backend_last_error(const wwws_backend* b) { return b ? b->text.c_str() : g_text.c_str(); }

}  // extern "C"
