// C ABI of the paged key-value cache and its attention (see include/lif.h for the contract of every call).
// Host side only: argument checks, workspace layout, launch geometry.
#include "../../include/lif.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <new>

#include "lif_host.h"
#include "lif_kv.h"
#include "lif_kv_pages.h"
#include "lif_kv_append.h"
#include "lif_kv_attend.h"

using namespace lif;

struct lif_kv {
    lif_kv_config cfg;
    KvView view;
    const double* frequencies;
    float* parts;
    unsigned* arrived;
    size_t part_bytes;
    int expected;            // cached tokens of a sequence as a rule (0: as many as the table holds)
};

namespace {

constexpr long long kMaxPositions = 1 << 24;     // of a sequence: the steps of 1024 of them are counted in 32 bits
constexpr int kAttendFew = 4096;                 // steps that run at once, or nearly
constexpr int kAppendGroups = 2048;              // workgroups for queries and keys that fill the chip
constexpr int kMoveBlocks = 2048;                // 8 workgroups of copies per compute unit
constexpr int kCopyBlocks = 128;                 // workgroups of lif_kv_reserve, which has a page to copy once in a while

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
int elem_bytes(int dtype) { return dtype == LIF_F32 ? 4 : 2; }
int log_of(int v) { return __builtin_ctz((unsigned)v); }

bool config_ok(const lif_kv_config* c, const char** why) {
    *why = "";
    if (!c) return (*why = "null config", false);
    if (c->dtype != LIF_F32 && c->dtype != LIF_F16 && c->dtype != LIF_BF16) return (*why = "dtype", false);
    if (c->layers < 1 || c->layers > 65536) return (*why = "layers", false);
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return (*why = "head_dim must be a multiple of 8 in 8..256", false);
    if (c->kv_heads < 1 || c->heads < c->kv_heads || c->heads % c->kv_heads || c->heads > 65536)
        return (*why = "heads must be a multiple of kv_heads", false);
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)))
        return (*why = "page_tokens must be 16, 32, 64, 128 or 256", false);
    if (c->pages < 1 || c->pages > 1 << 24) return (*why = "pages must be in 1..2^24", false);
    if (c->max_seqs < 1 || c->max_seqs > kKvMaxSeqs) return (*why = "max_seqs must be in 1..1024", false);
    if (c->max_pages < 1 || c->max_pages > 1 << 20 || (long long)c->max_pages * c->page_tokens > kMaxPositions)
        return (*why = "max_pages must be in 1..2^20, and a sequence of at most 2^24 tokens", false);
    if ((long long)c->kv_heads * c->page_tokens * c->head_dim * elem_bytes(c->dtype) >= 1ll << 31)
        return (*why = "a page of the keys of one layer must stay below 2 GiB", false);
    if (c->max_tokens < 1 || c->max_tokens > 256) return (*why = "max_tokens must be in 1..256", false);
    if (c->norm != LIF_NORM_NONE && c->norm != LIF_NORM_RMS && c->norm != LIF_NORM_LAYER) return (*why = "norm", false);
    if (c->rotary != LIF_ROTARY_HALF && c->rotary != LIF_ROTARY_INTERLEAVED) return (*why = "rotary", false);
    if (c->rotary_dim < 0 || c->rotary_dim > c->head_dim || c->rotary_dim % (c->rotary == LIF_ROTARY_HALF ? 16 : 2))
        return (*why = "rotary_dim must be 0..head_dim, a multiple of 16 (half layout) or 2 (interleaved)", false);
    if (!std::isfinite(c->scale) || !(c->scale > 0.f) || !std::isfinite(c->rotary_scale) || !(c->norm_eps >= 0.f) || !std::isfinite(c->norm_eps))
        return (*why = "scale, rotary_scale and norm_eps must be finite, scale positive, norm_eps not negative", false);
    return true;
}

struct KvLayout {
    size_t state, arrived, free_bits, moves, remap, parts, total;
};

// How the rows of an item, tokens x query heads of a key head, are dealt: blocks of 16 * tiles rows, and workgroups for each of them.
// `positions`: of a sequence to go through, at most.
// A workgroup reads the keys once for its block, so blocks are as large as registers allow; where there are so few that all their steps
// run at once, or nearly, the time is that of one workgroup with its parts, and smaller ones are faster (16 tokens of 2 sequences of 4000, 32
// heads of 128 on 8: 22.2 us in blocks of 16 rows, 45.2 in ones of 64).
// Tables are wider than their sequences as a rule, so blocks can come out too large: ones of 64 rows that leave a compute unit four waves only are taken for
// 128 rows and more (16 tokens of one sequence of 1000 in a table for 32768: 15.4 us in blocks of 32 rows, 28.3 in ones of 64; 16 sequences of 4000: 64.1
// and 61.7).  With lif_kv_set_expected_tokens(1000) that call takes 11.5 us.
struct Tiling {
    int tiles, waves, blocks, block_rows, units, round_units, round_steps;
    long long steps;                     // of a block's items, at most
};
// The workgroups of few blocks are what fits the chip, in eights (those of one XCD share keys); of many blocks four rounds and more of
// shorter ones, in eights too; of very many blocks they are enough by themselves, and no item has parts.  What a workgroup costs beside its
// steps is worth about five of them, so rounds of short ones are slow (20 tokens of 32 sequences of 2000, 71 heads of 64 on one: 162 us): of
// fewer steps than 16 per workgroup (64 if nine tenths of the chip have work) only one round of them is in use (73 us; 20 tokens
// of 64 sequences of 8000 467 -> 383 us).
int units_of(int blocks, int resident) {
    if (blocks == 1) return resident;
    if (blocks <= 8) return std::max(8, resident / blocks / 8 * 8);
    if (blocks <= 128) return (128 + blocks - 1) / blocks * 8;
    return 1;
}
bool lean(const lif_kv_config& c, int tiles) {
    const int pad = attend_dim_pad(c.head_dim);
    return attend_lean(pad, pad == c.head_dim, tiles, elem_bytes(c.dtype));
}
Tiling tiling(const lif_kv_config& c, int batch, int rows, long long positions) {
    const int bytes = elem_bytes(c.dtype), pad = attend_dim_pad(c.head_dim), need = (rows + 15) / 16;
    auto steps_of = [&](int waves) {
        const int step = 4 * 16 / bytes * waves;
        return (long long)batch * c.kv_heads * ((positions + step - 1) / step + 1);
    };
    Tiling g;
    g.tiles = std::min(attend_most_tiles(c.head_dim), need <= (pad > 128 ? 2 : 1) ? 1 : need <= 2 || (need >= 4 && need < 8 && !lean(c, 4)) ? 2 : 4);
    while (g.tiles > 1 && steps_of(4) * ((need + g.tiles / 2 - 1) / (g.tiles / 2)) <= kAttendFew) g.tiles /= 2;
    // of several blocks the last one may be mostly empty: 71 rows, 8 x 16000 positions, heads of 64: 33.5 us in two blocks of 64
    while (g.tiles > 1 && need > g.tiles && 4 * ((need + g.tiles - 1) / g.tiles * g.tiles) > 5 * need) g.tiles /= 2;
    g.blocks = (need + g.tiles - 1) / g.tiles;
    g.block_rows = std::min(rows, 16 * g.tiles);
    // Eight waves share a part, or four: the larger parts are fewer to add, the smaller ones fill the chip sooner, and two workgroups of them hide
    // each other's beginnings and ends.  Larger ones pay where a part has some rows, and where workgroups go through parts of one item and few are left
    // over (4 tokens of 4 sequences of up to 4000, 32 heads on 8: 20.8 us with four, 14.2 with eight; one of 32 sequences of 2000, 71 heads on one,
    // 160 items: 15.1 and 18.4; one of 64 sequences, 512 items: 144.5 and 149.3).  Between these points, and around the 768 and 2048 positions, nothing was
    // measured.
    const long long items = (long long)batch * c.kv_heads * g.blocks;
    const bool few = items <= kAttendUnits / 2 || (items <= kAttendUnits && 8 * items > 7 * kAttendUnits);
    const bool fits = lean(c, g.tiles), some = g.block_rows >= 4 && (positions > (g.block_rows >= 16 ? 768 : 2048) || items >= kAttendUnits / 2);
    g.waves = fits && (g.tiles > 1 || (some && few)) ? 8 : 4;
    g.steps = steps_of(4);
    const int at_once = kAttendUnits * attend_resident(fits, g.waves);
    g.units = units_of(g.blocks, at_once);
    g.round_units = g.blocks <= 8 ? g.units : std::min(g.units, std::max(1, at_once / g.blocks));
    g.round_steps = g.blocks <= 8 ? 0 : g.units * (10 * g.round_units * g.blocks >= 9 * at_once ? 64 : 16);
    return g;
}
// floats of the parts of any call
size_t most_part_floats(const lif_kv_config& c) {
    const int rows = c.max_tokens * (c.heads / c.kv_heads), need = (rows + 15) / 16, pad = attend_dim_pad(c.head_dim);
    size_t most = 0;
    for (int tiles = 1; tiles <= attend_most_tiles(c.head_dim); tiles *= 2) {
        // fewer rows than the largest call's make fewer blocks, and more workgroups for each: the products below are at their largest in between
        for (int blocks = 1; blocks <= std::min(129, (need + tiles - 1) / tiles); ++blocks) {
            const size_t groups = (size_t)blocks * units_of(blocks, kAttendUnits * attend_resident(lean(c, tiles), tiles > 1 ? 8 : 4));
            if (blocks <= 128) most = std::max(most, 4 * groups * std::min(rows, 16 * tiles) * (pad + 4));
        }
    }
    return most;
}

KvLayout make_layout(const lif_kv_config& c) {
    KvLayout L;
    size_t off = 0;
    L.state = off;
    off = align_up(off + sizeof(KvState), 256);
    L.arrived = off;                   // directly behind the state: a reset clears both
    off = align_up(off + sizeof(unsigned) * 4 * kAttendMost, 256);
    L.free_bits = off;
    off = align_up(off + sizeof(unsigned long long) * ((size_t)(c.pages + 63) / 64), 256);
    L.moves = off;
    off = align_up(off + sizeof(int2) * c.pages, 256);
    L.remap = off;
    off = align_up(off + sizeof(int32_t) * std::max(c.pages, c.max_seqs), 256);
    L.parts = off;
    off = align_up(off + sizeof(float) * most_part_floats(c), 256);
    L.total = off;
    return L;
}

int launched() {
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? LIF_OK : fail(LIF_HIP_ERROR, "launch: %s", hipGetErrorString(e));
}

int plan_threads(const lif_kv* kv) { return kv->cfg.max_seqs <= kKvPlanFew ? kKvPlanFew : kKvMaxSeqs; }

int batch_ok(const lif_kv* kv, int32_t layer, int32_t batch, int32_t n_tokens) {
    if (layer < 0 || layer >= kv->cfg.layers) return fail(LIF_INVALID_ARG, "layer out of range");
    if (batch < 1 || batch > kKvMaxSeqs) return fail(LIF_INVALID_ARG, "batch must be in 1..1024");
    if (n_tokens < 1 || n_tokens > kv->cfg.max_tokens) return fail(LIF_INVALID_ARG, "n_tokens must be in 1..max_tokens");
    return LIF_OK;
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// a stride of at least one row, in whole 16 bytes
int stride_ok(const lif_kv* kv, int64_t stride, int heads) {
    const int per = 16 / elem_bytes(kv->cfg.dtype);
    if (stride < (int64_t)heads * kv->cfg.head_dim || stride % per || stride > (int64_t)1 << 40)
        return fail(LIF_INVALID_ARG, "a row stride must hold the heads and be a multiple of 16 bytes");
    return LIF_OK;
}

// Whether rows of `width` elements, read from `from` and written to `to`, share memory in another way than that they are the same ones.  A stride
// holds a row, so a row of one array can touch two of the other, those that begin around it; with equal strides the same two for all rows.
bool overlap(const lif_kv* kv, const void* from, int64_t from_stride, const void* to, int64_t to_stride, int rows, int64_t width) {
    const int64_t e = elem_bytes(kv->cfg.dtype), size = width * e, step = from_stride * e, to_step = to_stride * e;
    const int64_t ahead = (int64_t)(reinterpret_cast<uintptr_t>(to) - reinterpret_cast<uintptr_t>(from));
    if (ahead >= (rows - 1) * step + size || -ahead >= (rows - 1) * to_step + size) return false;
    if (ahead == 0 && (step == to_step || rows == 1)) return false;
    auto touches = [&](int64_t at, int64_t first, int64_t last) {
        int64_t k = at / step - (at % step < 0);
        for (int i = 0; i < 2; ++i, ++k)
            if (k >= first && k <= last && std::abs(at - k * step) < size) return true;
        return false;
    };
    if (step == to_step) return touches(ahead, 1 - rows, rows - 1);
    for (int r = 0; r < rows; ++r)
        if (touches(ahead + r * to_step, 0, rows - 1)) return true;
    return false;
}

}  // namespace

#define LIF_TRY(call)              \
    do {                           \
        int rc_ = (call);          \
        if (rc_ != LIF_OK) return rc_; \
    } while (0)

extern "C" {

size_t lif_kv_workspace_bytes(const lif_kv_config* cfg) {
    const char* why;
    return config_ok(cfg, &why) ? make_layout(*cfg).total : 0;
}

int lif_kv_create(const lif_kv_config* cfg, const lif_kv_buffers* buf, lif_kv** out) {
    const char* why;
    if (!cfg || !buf || !out) return fail(LIF_INVALID_ARG, "null pointer");
    if (!config_ok(cfg, &why)) return fail(LIF_INVALID_ARG, "configuration: %s", why);
    if (!buf->k || !buf->v || !buf->table || !buf->lengths || !buf->fresh || !buf->refs || !buf->workspace)
        return fail(LIF_INVALID_ARG, "null buffer");
    if (cfg->rotary_dim > 0 && !buf->frequencies) return fail(LIF_INVALID_ARG, "rotary_dim without frequencies");
    if (!aligned16(buf->k) || !aligned16(buf->v)) return fail(LIF_INVALID_ARG, "keys and values must be 16-byte aligned");
    const KvLayout L = make_layout(*cfg);
    if (buf->workspace_bytes < L.total || reinterpret_cast<uintptr_t>(buf->workspace) % 256)
        return fail(LIF_INVALID_ARG, "workspace too small or not 256-byte aligned");
    lif_kv* kv = new (std::nothrow) lif_kv;
    if (!kv) return fail(LIF_INVALID_ARG, "out of host memory");
    char* w = static_cast<char*>(buf->workspace);
    kv->cfg = *cfg;
    KvView& v = kv->view;
    v.k = static_cast<char*>(buf->k);
    v.v = static_cast<char*>(buf->v);
    v.table = buf->table;
    v.lengths = buf->lengths;
    v.fresh = buf->fresh;
    v.refs = buf->refs;
    v.st = reinterpret_cast<KvState*>(w + L.state);
    v.arrived = reinterpret_cast<unsigned*>(w + L.arrived);
    v.n_arrived = 4 * kAttendMost;
    v.free_bits = reinterpret_cast<unsigned long long*>(w + L.free_bits);
    v.moves = reinterpret_cast<int2*>(w + L.moves);
    v.remap = reinterpret_cast<int32_t*>(w + L.remap);
    v.pages = cfg->pages;
    v.max_seqs = cfg->max_seqs;
    v.max_pages = cfg->max_pages;
    v.log_page = log_of(cfg->page_tokens);
    v.layers = cfg->layers;
    v.page_bytes = (unsigned long long)cfg->kv_heads * cfg->page_tokens * cfg->head_dim * elem_bytes(cfg->dtype);
    kv->frequencies = buf->frequencies;
    kv->parts = reinterpret_cast<float*>(w + L.parts);
    kv->arrived = reinterpret_cast<unsigned*>(w + L.arrived);
    kv->part_bytes = L.total - L.parts;
    kv->expected = 0;
    *out = kv;
    return LIF_OK;
}

int lif_kv_destroy(lif_kv* kv) {
    delete kv;
    return LIF_OK;
}

int lif_kv_reset(lif_kv* kv, void* stream) {
    if (!kv) return fail(LIF_INVALID_ARG, "null handle");
    const long long most = std::max<long long>(kv->cfg.pages, (long long)kv->cfg.max_seqs * kv->cfg.max_pages);
    hipLaunchKernelGGL((k_kv_clear<true>), dim3((unsigned)std::min<long long>((most + 255) / 256, 1024)), dim3(256), 0, (hipStream_t)stream, kv->view);
    return launched();
}

int lif_kv_adopt(lif_kv* kv, void* stream) {
    if (!kv) return fail(LIF_INVALID_ARG, "null handle");
    hipLaunchKernelGGL((k_kv_clear<false>), dim3(std::min((kv->cfg.pages + 255) / 256, 1024)), dim3(256), 0, (hipStream_t)stream, kv->view);
    hipLaunchKernelGGL(k_kv_adopt, dim3(kv->cfg.max_seqs), dim3(256), 0, (hipStream_t)stream, kv->view);
    return launched();
}

int lif_kv_reserve(lif_kv* kv, const int32_t* counts_dev, void* stream) {
    if (!kv || !counts_dev) return fail(LIF_INVALID_ARG, "null pointer");
    const int threads = plan_threads(kv);
    hipLaunchKernelGGL(threads == kKvPlanFew ? k_kv_reserve<kKvPlanFew> : k_kv_reserve<kKvMaxSeqs>, dim3(kCopyBlocks), dim3(threads), 0,
                       (hipStream_t)stream, kv->view, counts_dev);
    return launched();
}

int lif_kv_truncate(lif_kv* kv, const int32_t* lengths_dev, void* stream) {
    if (!kv || !lengths_dev) return fail(LIF_INVALID_ARG, "null pointer");
    hipLaunchKernelGGL(k_kv_truncate, dim3(kv->cfg.max_seqs), dim3(256), 0, (hipStream_t)stream, kv->view, lengths_dev);
    return launched();
}

int lif_kv_fork(lif_kv* kv, const int32_t* src_dev, const int32_t* dst_dev, int32_t n, void* stream) {
    if (!kv || !src_dev || !dst_dev) return fail(LIF_INVALID_ARG, "null pointer");
    if (n < 1 || n > kv->cfg.max_seqs) return fail(LIF_INVALID_ARG, "n must be in 1..max_seqs");
    const int threads = plan_threads(kv);
    hipLaunchKernelGGL(threads == kKvPlanFew ? k_kv_fork<kKvPlanFew> : k_kv_fork<kKvMaxSeqs>, dim3(1), dim3(threads), 0, (hipStream_t)stream,
                       kv->view, src_dev, dst_dev, n);
    hipLaunchKernelGGL((k_kv_move<KV_FORK>), dim3(n + kMoveBlocks), dim3(256), 0, (hipStream_t)stream, kv->view, src_dev, dst_dev, n);
    return launched();
}

int lif_kv_compact(lif_kv* kv, void* stream) {
    if (!kv) return fail(LIF_INVALID_ARG, "null handle");
    const int threads = plan_threads(kv);
    hipLaunchKernelGGL(threads == kKvPlanFew ? k_kv_compact<kKvPlanFew> : k_kv_compact<kKvMaxSeqs>, dim3(1), dim3(threads), 0, (hipStream_t)stream,
                       kv->view);
    hipLaunchKernelGGL((k_kv_move<KV_COMPACT>), dim3(kv->cfg.max_seqs + kMoveBlocks), dim3(256), 0, (hipStream_t)stream, kv->view, nullptr, nullptr,
                       kv->cfg.max_seqs);
    return launched();
}

int lif_kv_append(lif_kv* kv, int32_t layer, const lif_kv_rows* rows, void* stream) {
    if (!kv || !rows) return fail(LIF_INVALID_ARG, "null pointer");
    const lif_kv_config& c = kv->cfg;
    LIF_TRY(batch_ok(kv, layer, rows->batch, rows->n_tokens));
    if (!rows->q || !rows->k || !rows->v || !rows->q_out) return fail(LIF_INVALID_ARG, "null rows");
    if (!aligned16(rows->q) || !aligned16(rows->k) || !aligned16(rows->v) || !aligned16(rows->q_out))
        return fail(LIF_INVALID_ARG, "rows must be 16-byte aligned");
    LIF_TRY(stride_ok(kv, rows->q_stride, c.heads));
    LIF_TRY(stride_ok(kv, rows->q_out_stride, c.heads));
    LIF_TRY(stride_ok(kv, rows->k_stride, c.kv_heads));
    LIF_TRY(stride_ok(kv, rows->v_stride, c.kv_heads));
    if (overlap(kv, rows->q, rows->q_stride, rows->q_out, rows->q_out_stride, rows->batch * rows->n_tokens, (int64_t)c.heads * c.head_dim))
        return fail(LIF_INVALID_ARG, "q_out must not overlap q (or be q itself, with the same stride)");
    AppendArgs a{static_cast<const char*>(rows->q), static_cast<const char*>(rows->k), static_cast<const char*>(rows->v),
                 static_cast<char*>(rows->q_out), rows->q_stride, rows->k_stride, rows->v_stride, rows->q_out_stride,
                 rows->q_weight, rows->q_bias, rows->k_weight, rows->k_bias, kv->frequencies, rows->positions, rows->slots, rows->batch,
                 rows->n_tokens, c.heads, c.kv_heads, c.head_dim, layer, c.rotary_dim, c.norm, 0, 0, 0, 0, 0, c.norm_eps, c.rotary_scale, 1.f / c.head_dim};
    const int count = rows->batch * rows->n_tokens, all = c.heads + c.kv_heads, n = 16 / elem_bytes(c.dtype);
    while ((n << a.log_lanes) < c.head_dim) ++a.log_lanes;
    const int at_once = 256 >> a.log_lanes;
    // few tokens: a workgroup for as many heads as it takes at once, to have the whole chip at it; many: more heads each, angles once for them
    const int wanted = std::max(1, kAppendGroups / count), blocks = std::min((all + at_once - 1) / at_once, wanted);
    a.heads_per_block = ((all + blocks - 1) / blocks + at_once - 1) / at_once * at_once;
    a.head_blocks = (all + a.heads_per_block - 1) / a.heads_per_block;
    a.pieces = (rows->n_tokens + n - 2) / n + 1;
    a.value_blocks = (c.kv_heads * c.head_dim * elem_bytes(c.dtype) / 4 + 255) / 256;
    const bool interleaved = c.rotary == LIF_ROTARY_INTERLEAVED;
    hipStream_t s = (hipStream_t)stream;
    if (c.dtype == LIF_F32) launch_append_f32(kv->view, a, interleaved, s);
    else if (c.dtype == LIF_F16) launch_append_f16(kv->view, a, interleaved, s);
    else launch_append_bf16(kv->view, a, interleaved, s);
    return launched();
}

int lif_kv_attend(lif_kv* kv, int32_t layer, const lif_kv_query* query, void* stream) {
    if (!kv || !query) return fail(LIF_INVALID_ARG, "null pointer");
    const lif_kv_config& c = kv->cfg;
    LIF_TRY(batch_ok(kv, layer, query->batch, query->n_tokens));
    if (!query->q || !query->out) return fail(LIF_INVALID_ARG, "null rows");
    if (!aligned16(query->q) || !aligned16(query->out)) return fail(LIF_INVALID_ARG, "rows must be 16-byte aligned");
    LIF_TRY(stride_ok(kv, query->q_stride, c.heads));
    LIF_TRY(stride_ok(kv, query->out_stride, c.heads));
    if (query->window < 0) return fail(LIF_INVALID_ARG, "window must not be negative");
    if (query->tree && query->n_tokens > 64) return fail(LIF_INVALID_ARG, "a tree has at most 64 tokens");
    const int share = c.heads / c.kv_heads, rows = query->n_tokens * share;
    const long long width = (long long)c.max_pages * c.page_tokens;
    const Tiling g = tiling(c, query->batch, rows, kv->expected ? std::min<long long>(kv->expected, width) : width);
    if (tiling(c, query->batch, rows, width).steps >= (1ll << 31) - 4096)
        return fail(LIF_INVALID_ARG, "batch, heads and the width of the table are too large together");
    if (overlap(kv, query->q, query->q_stride, query->out, query->out_stride, query->batch * query->n_tokens, (int64_t)c.heads * c.head_dim))
        return fail(LIF_INVALID_ARG, "out must not overlap q (or be q itself, with the same stride)");
    const KvView& v = kv->view;
    const size_t layer_at = (size_t)layer * c.pages * v.page_bytes;
    AttendArgs a{static_cast<const char*>(query->q), static_cast<char*>(query->out), query->lse, query->q_stride, query->out_stride,
                 query->slots, query->starts, reinterpret_cast<const unsigned long long*>(query->tree), v.k + layer_at, v.v + layer_at, v.table,
                 v.lengths, v.fresh, &v.st->error, kv->parts, kv->arrived, (unsigned)kv->part_bytes, (unsigned)v.page_bytes,
                 (unsigned)(v.page_bytes / c.kv_heads), c.pages, c.max_seqs, c.max_pages, v.log_page, query->batch, query->n_tokens, c.heads,
                 c.kv_heads, share, c.head_dim, query->window, g.units, g.round_units, g.round_steps, g.blocks, g.block_rows, c.scale * kLog2e};
    hipStream_t s = (hipStream_t)stream;
    using Launch = bool (*)(const AttendArgs&, int, int, hipStream_t);
    static constexpr Launch kLaunch[3][3] = {{launch_attend_f32_1, launch_attend_f32_2, launch_attend_f32_4},
                                             {launch_attend_f16_1, launch_attend_f16_2, launch_attend_f16_4},
                                             {launch_attend_bf16_1, launch_attend_bf16_2, launch_attend_bf16_4}};
    if (!kLaunch[c.dtype][g.tiles >> 1](a, g.blocks * g.units, g.waves, s)) return fail(LIF_HIP_ERROR, "no kernel for this form of attention");
    return launched();
}

int lif_kv_set_expected_tokens(lif_kv* kv, int32_t tokens) {
    if (!kv) return fail(LIF_INVALID_ARG, "null handle");
    if (tokens < 0) return fail(LIF_INVALID_ARG, "tokens must not be negative");
    kv->expected = tokens;
    return LIF_OK;
}

int lif_kv_get_state(lif_kv* kv, lif_kv_state* out, void* stream) {
    if (!kv || !out) return fail(LIF_INVALID_ARG, "null pointer");
    KvState st;
    LIF_HIP(hipMemcpyAsync(&st, kv->view.st, sizeof(st), hipMemcpyDeviceToHost, (hipStream_t)stream));
    LIF_HIP(hipStreamSynchronize((hipStream_t)stream));
    *out = lif_kv_state{st.used, st.error, st.n_moves};
    return LIF_OK;
}

int lif_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double trained, double slow, double fast, double* out) {
    if (!out) return fail(LIF_INVALID_ARG, "null pointer");
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 65536) return fail(LIF_INVALID_ARG, "rotary_dim must be a positive even number");
    if (!(base > 0) || !std::isfinite(base)) return fail(LIF_INVALID_ARG, "base must be positive");
    if (scaling < LIF_ROPE_PLAIN || scaling > LIF_ROPE_RAMP) return fail(LIF_INVALID_ARG, "scaling");
    if (scaling != LIF_ROPE_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return fail(LIF_INVALID_ARG, "factor must be positive");
    if (scaling == LIF_ROPE_BASE && rotary_dim == 2) return fail(LIF_INVALID_ARG, "a single pair has no base to raise");
    if (scaling == LIF_ROPE_RAMP && (!(trained > 0) || !std::isfinite(trained) || !(fast > slow) || !std::isfinite(fast - slow)))
        return fail(LIF_INVALID_ARG, "the ramp needs a trained length and fast > slow");
    if (scaling == LIF_ROPE_BASE) base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rotary_dim);
        if (scaling == LIF_ROPE_LINEAR) f /= factor;
        if (scaling == LIF_ROPE_RAMP) {
            const double turns = trained * f / 6.283185307179586476925, keep = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
            f = keep * f + (1.0 - keep) * f / factor;
        }
        out[i] = f;
    }
    return LIF_OK;
}

}  // extern "C"
