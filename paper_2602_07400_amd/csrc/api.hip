// C-ABI front end of libbitlogic: argument checks on the host, workspace
// carving, launches.  Every check runs before any HIP runtime call, so a
// rejected call enqueues nothing (and needs no GPU to be rejected).
#include <float.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <mutex>

#include "bitlogic.h"
#include "bl_internal.h"
#include "adapters.h"
#include "logit_rows.h"

// Scratch of bitlogic_network_forward_noalloc: one copy of this array per GPU
// the library runs on, held until the process ends.  In host code `scratch`
// only names the symbol for hipGetSymbolAddress; the array's device address on
// each GPU is looked up once and kept in g_scratch_ptr below.
static __device__ __align__(256) unsigned char scratch[BITLOGIC_NOALLOC_SCRATCH_BYTES];

namespace {

thread_local char g_last_error[256] = "";

int fail(int status, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof g_last_error, fmt, ap);
    va_end(ap);
    return status;
}

int ok()
{
    g_last_error[0] = '\0';
    return BITLOGIC_OK;
}

int hip_status(hipError_t e, const char *what)
{
    if (e != hipSuccess)
        return fail(BITLOGIC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int32_t kDspMaxClasses = 128;   // quantized head: logits below 2^31
constexpr size_t kWsAlign = 256;

size_t round_up(size_t v) { return (v + kWsAlign - 1) / kWsAlign * kWsAlign; }

int64_t words_of(int64_t n) { return (n + 63) / 64; }

int check_encode(const uint8_t *x, int64_t n, int32_t d, const uint8_t *th, int32_t b,
                 const uint64_t *out)
{
    if (!x || !th || !out)
        return fail(BITLOGIC_ERR_NULL, "encode: NULL pointer");
    if (n < 0 || d <= 0 || b <= 0 || b > 64)
        return fail(BITLOGIC_ERR_SHAPE, "encode: need n >= 0, d > 0, 1 <= b <= 64");
    if ((int64_t)d * b > kMaxRows)
        return fail(BITLOGIC_ERR_SHAPE, "encode: d * b exceeds int32");
    if (!aligned(out, 8))
        return fail(BITLOGIC_ERR_ALIGN, "encode: bits_out not 8-byte aligned");
    return BITLOGIC_OK;
}

int check_layer(const uint64_t *in, int32_t w_in, int64_t n_words, const int32_t *conn,
                const uint64_t *tables, int32_t w_out, int32_t k, const uint64_t *out,
                const char *who)
{
    if (!in || !conn || !tables || !out)
        return fail(BITLOGIC_ERR_NULL, "%s: NULL pointer", who);
    if (k < 1 || k > 6)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: fan-in k=%d outside 1..6", who, k);
    if (w_in <= 0 || w_out <= 0 || n_words < 0)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need w_in > 0, w_out > 0, n_words >= 0", who);
    if (n_words > ((int64_t)1 << 40))
        return fail(BITLOGIC_ERR_SHAPE, "%s: n_words too large", who);
    if (!aligned(in, 8) || !aligned(out, 8))
        return fail(BITLOGIC_ERR_ALIGN, "%s: bit buffers must be 8-byte aligned", who);
    if (!aligned(conn, 4) || !aligned(tables, 8))
        return fail(BITLOGIC_ERR_ALIGN, "%s: conn/tables misaligned", who);
    return BITLOGIC_OK;
}

int check_head(const uint64_t *bits, int32_t w, int64_t n, int32_t c, const int32_t *scores,
               const int32_t *argmax)
{
    if (!bits || (!scores && !argmax))
        return fail(BITLOGIC_ERR_NULL, "head: NULL bits, or both outputs NULL");
    if (w <= 0 || c <= 0 || n < 0)
        return fail(BITLOGIC_ERR_SHAPE, "head: need w > 0, c > 0, n >= 0");
    if (w % c != 0)
        return fail(BITLOGIC_ERR_SHAPE, "head: w=%d not a multiple of n_classes=%d", w, c);
    if (w / c > 65535)
        return fail(BITLOGIC_ERR_SHAPE, "head: group size %d > 65535", w / c);
    if (n > ((int64_t)1 << 40))
        return fail(BITLOGIC_ERR_SHAPE, "head: n_samples too large");
    if (!aligned(bits, 8) || (scores && !aligned(scores, 4)) || (argmax && !aligned(argmax, 4)))
        return fail(BITLOGIC_ERR_ALIGN, "head: misaligned buffer");
    return BITLOGIC_OK;
}

// Rows of class scores or logits: type, sizes and stride.
constexpr int64_t kMaxStride = 1 << 30;
constexpr int64_t kMaxRequestStride = (int64_t)1 << 40;

size_t logit_bytes(int32_t type)
{
    return type == BITLOGIC_LOGITS_I32 || type == BITLOGIC_LOGITS_F32 ? 4 : 2;
}

int check_rows(const char *who, int32_t type, int64_t n_rows, int32_t n_classes,
               int64_t row_stride)
{
    if (type < BITLOGIC_LOGITS_I32 || type > BITLOGIC_LOGITS_BF16)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: unknown element type %d", who, type);
    if (n_rows < 0 || n_rows > kMaxRows || n_classes < 1 || n_classes > bl::rows::kMaxClasses)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need 0 <= n_rows < 2^31, 1 <= n_classes <= 2^30",
                    who);
    if (row_stride < 0 || row_stride > kMaxStride)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need 0 <= row_stride <= 2^30", who);
    return BITLOGIC_OK;
}

// Bytes from a buffer's first element to behind its last one.
size_t span_bytes(int64_t n_rows, int64_t n_cols, int64_t stride, int32_t type)
{
    return (size_t)((n_rows - 1) * stride + n_cols) * logit_bytes(type);
}

bool overlaps(const void *a, size_t a_bytes, const void *b, size_t b_bytes)
{
    return (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

// Rows in memory: widths and strides in bytes (p NULL: not there).
struct Region {
    const char *name;
    const void *p;
    int64_t rows;
    size_t width, stride;
};

Region flat(const char *name, const void *p, size_t bytes) { return {name, p, 1, bytes, bytes}; }

// Rows of one stride may lie between each other's; others are apart where their ranges are.
bool overlaps(const Region &a, const Region &b)
{
    if (!a.p || !b.p || a.rows == 0 || b.rows == 0 ||
        !overlaps(a.p, (a.rows - 1) * a.stride + a.width, b.p, (b.rows - 1) * b.stride + b.width))
        return false;
    const size_t stride = a.stride;
    if (stride != b.stride || a.width > stride || b.width > stride)
        return true;
    const uintptr_t ap = (uintptr_t)a.p, bp = (uintptr_t)b.p;
    const size_t at = bp >= ap ? (bp - ap) % stride : (stride - (ap - bp) % stride) % stride;
    return at < a.width || at + b.width > stride;
}

// Outputs apart from each other and from what is read.
int check_apart(const char *who, std::initializer_list<Region> outputs,
                std::initializer_list<Region> inputs)
{
    for (const Region *o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Region *other = outputs.begin(); other != o; ++other)
            if (overlaps(*o, *other))
                return fail(BITLOGIC_ERR_SHAPE, "%s: %s overlaps %s", who, o->name, other->name);
        for (const Region &i : inputs)
            if (overlaps(*o, i))
                return fail(BITLOGIC_ERR_SHAPE, "%s: %s overlaps %s", who, o->name, i.name);
    }
    return BITLOGIC_OK;
}

int check_list(const char *who, int32_t k, float temperature)
{
    if (k < 1)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need k >= 1", who);
    if (k > BITLOGIC_TOP_MAX)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: k=%d > %d", who, k, BITLOGIC_TOP_MAX);
    if (!(temperature > 0.0f && temperature <= FLT_MAX))
        return fail(BITLOGIC_ERR_SHAPE, "%s: temperature %g is not positive and finite", who,
                    (double)temperature);
    return BITLOGIC_OK;
}

// BITLOGIC_UNFUSED_HEAD=1 in the environment runs the last layer and the head
// as separate kernels (for comparison; results are identical).
bool fused_head_enabled()
{
    const char *e = getenv("BITLOGIC_UNFUSED_HEAD");
    return !(e && e[0] == '1');
}

// BITLOGIC_JUMP_LAYER=0 keeps every stored layer on the per-lane slab kernel,
// =1 runs the node-per-wave kernel wherever it can (also where it is not the
// faster choice); unset, it runs where it is faster.  Results are identical.
enum JumpMode { kJumpOff, kJumpAuto, kJumpForced };
JumpMode jump_mode()
{
    const char *e = getenv("BITLOGIC_JUMP_LAYER");
    if (e && e[0] == '0')
        return kJumpOff;
    if (e && e[0] == '1')
        return kJumpForced;
    return kJumpAuto;
}

// bitlogic_forward keeps its encoded and intermediate bit tensors in the slab
// layout [Wp / S][rows][S] (S = kSlabWords, Wp = W rounded up to whole slabs),
// which bounds the LUT-layer gathers' per-XCD working set (see lut_layer.hip).
struct ForwardPlan {
    int64_t W;
    int64_t n_slabs;
    int32_t widest;
    size_t off_enc, off_a, off_b, off_head, total;
    bl::HeadPlan head;
    bool fused;            // last layer + head in one kernel
    uint64_t jump_mask;    // bit l: layer l runs on the node-per-wave kernel
    size_t off_rec;        // its per-node records (shared by those layers)
    bl::ColumnHeadPlan cols;   // cols.ok: the column kernels run the batch
    bl::ColumnNetwork net;     // net.ok: and a column's network runs in one block
};

bitlogic_network legacy_net(int32_t n_features, const uint8_t *thresholds, int32_t n_thresholds,
                            const bitlogic_layer *layers, int32_t n_layers, int32_t n_classes,
                            const int8_t *dsp_weights);

// Work of a forward by columns, in units of about 4 ps of the whole GPU: a
// wire, and a node of up to 4 or of 5 and 6 inputs.  The slab kernels take over
// at kColumnMaxCost, where 30 random networks (1000 to 57000 nodes a layer, 64
// to 33000 samples) crossed: columns against slabs 25.7 us : 29.7 at 2.7M,
// 16.3 : 22.2 at 1.2M, 38.2 : 64.7 at 0.9M, but 32.0 : 30.2 at 3.5M, 45.9 :
// 35.7 at 4.0M, 39.0 : 33.2 at 5.8M and 66.8 : 49.3 at 7.9M.
constexpr int64_t kColumnMaxCost = 3000000;
// The cost counts nodes, but a column's last kernel is a block of 1024 threads
// however few of them it has: networks of 16 to 256 nodes a layer crossed at 1200
// to 2000 columns far below that cost.  Stages by columns against slabs, 1024
// columns: 16 -> 16 nodes 14.7 us : 16.8, 100 -> 100 14.7 : 17.7, 784 -> 100 ->
// 100 26.1 : 27.2; 2048: 22.7 : 17.2, 23.8 : 22.5; 4096: 41 : 22, 43 : 33 (one
// block a column, without a bound: 96 and 73).  k_col_encode's grid has a column
// per block in y, of which there are at most 65535.
constexpr int64_t kColumnMaxColumns = 1024;
bool columns_pay(int64_t W, int64_t wires, const bitlogic_layer *layers, int32_t L)
{
    // every sum stays below kColumnMaxCost + 5 * 2^31 and the product is not taken
    // (sizes up to 2^40 samples and 2^31 rows a layer are planned for)
    int64_t per_column = wires;
    for (int32_t l = 0; l < L && per_column <= kColumnMaxCost; ++l)
        per_column += (int64_t)layers[l].w_out * (layers[l].k <= 4 ? 2 : 5);
    return W <= kColumnMaxColumns && W <= kColumnMaxCost / per_column;
}

int plan_forward(int64_t n, int32_t d, int32_t b, const bitlogic_layer *layers, int32_t L,
                 int32_t c, const uint8_t *const *pass_fanin, ForwardPlan *fp)
{
    if (!layers)
        return fail(BITLOGIC_ERR_NULL, "forward: NULL layer array");
    if (L < 1)
        return fail(BITLOGIC_ERR_SHAPE, "forward: need n_layers >= 1");
    if (n < 0 || d <= 0 || b <= 0 || b > 64 || c <= 0)
        return fail(BITLOGIC_ERR_SHAPE, "forward: need n >= 0, d > 0, 1 <= b <= 64, c > 0");
    if ((int64_t)d * b > kMaxRows)
        return fail(BITLOGIC_ERR_SHAPE, "forward: d * b exceeds int32");
    if (n > ((int64_t)1 << 40))
        return fail(BITLOGIC_ERR_SHAPE, "forward: n_samples too large");
    int32_t widest = 0;
    for (int32_t l = 0; l < L; ++l) {
        if (!layers[l].conn || !layers[l].tables)
            return fail(BITLOGIC_ERR_NULL, "forward: layer %d has a NULL pointer", l);
        if (layers[l].k < 1 || layers[l].k > 6)
            return fail(BITLOGIC_ERR_UNSUPPORTED, "forward: layer %d fan-in %d outside 1..6",
                        l, layers[l].k);
        if (layers[l].w_out <= 0)
            return fail(BITLOGIC_ERR_SHAPE, "forward: layer %d width %d", l, layers[l].w_out);
        if (!aligned(layers[l].conn, 4) || !aligned(layers[l].tables, 8))
            return fail(BITLOGIC_ERR_ALIGN, "forward: layer %d conn/tables misaligned", l);
        if (layers[l].w_out > widest)
            widest = layers[l].w_out;
    }
    const int32_t w_last = layers[L - 1].w_out;
    if (w_last % c != 0)
        return fail(BITLOGIC_ERR_SHAPE, "forward: last width %d not a multiple of %d classes",
                    w_last, c);
    if (w_last / c > 65535)
        return fail(BITLOGIC_ERR_SHAPE, "forward: group size %d > 65535", w_last / c);
    fp->W = words_of(n);
    fp->n_slabs = (fp->W + bl::kSlabWords - 1) / bl::kSlabWords;
    fp->widest = widest;
    const int64_t Wp = fp->n_slabs * bl::kSlabWords;
    const size_t enc = (size_t)d * b * Wp * sizeof(uint64_t);
    const size_t act = (size_t)widest * Wp * sizeof(uint64_t);
    // the last layer and the head run fused when the group size allows it
    const int32_t nb = bl::fused_head_nodes(w_last / c, c, fp->n_slabs);
    fp->fused = nb > 0 && fused_head_enabled();
    fp->head = fp->fused ? bl::plan_fused_head(w_last, n, c, nb) : bl::plan_head(w_last, n, c);
    // layer l writes activation buffer l % 2, except a last layer fused with
    // the head, which writes nothing: allocate only the buffers some layer writes
    const int32_t stored = fp->fused ? L - 1 : L;     // layers whose bits are stored
    const bool need_a = stored >= 1, need_b = stored >= 2;
    fp->off_enc = 0;
    fp->off_a = round_up(enc);
    fp->off_b = fp->off_a + (need_a ? round_up(act) : 0);
    fp->off_head = fp->off_b + (need_b ? round_up(act) : 0);
    // stored, unspecialized layers of fan-in 5 or 6 whose input slab pair
    // fits the L2 run with a node per wave (lut_jump.hip); they share one
    // record array, sized for the widest of them
    fp->jump_mask = 0;
    int32_t rec_w = 0;
    int32_t w_in = d * b;
    const JumpMode jm = jump_mode();
    for (int32_t l = 0; l < L; ++l) {
        const bool last_fused = fp->fused && l == L - 1;
        const bool spec = pass_fanin && pass_fanin[l];
        if (l < 64 && !last_fused && !spec && jm != kJumpOff &&
            bl::jump_layer_fits(w_in, layers[l].w_out, layers[l].k, fp->n_slabs,
                                jm == kJumpForced)) {
            fp->jump_mask |= 1ull << l;
            rec_w = std::max(rec_w, layers[l].w_out);
        }
        w_in = layers[l].w_out;
    }
    // small batches run by 64-sample columns, in the space of the slab layout's
    // tensors (a column tensor is never larger): the encoded bits and the
    // activations where the slab layout has them, counts that the caller does
    // not receive over the encoded bits, which layer 0 has consumed by then (room
    // for them there, 32 wires a class in whole slabs, is asked of every batch,
    // since the plan does not know the outputs).  Where a switch asks for other
    // kernels, or the encoder has more wires a feature than the column encoder's
    // waves hold, the slab kernels run.
    fp->cols.ok = fp->net.ok = false;
    if (L >= 2 && b <= 8 && fp->fused && jm == kJumpAuto &&
        (size_t)n * c * sizeof(int32_t) <= enc && columns_pay(fp->W, d * b, layers, L))
        fp->cols = bl::plan_column_head(layers[L - 2].w_out, w_last, c);
    if (fp->cols.ok && L <= bl::kColumnMaxLayers) {
        int32_t w[bl::kColumnMaxLayers], k[bl::kColumnMaxLayers];
        for (int32_t l = 0; l < L; ++l) {
            w[l] = layers[l].w_out;
            k[l] = layers[l].k;
        }
        fp->net = bl::plan_column_network(d, b, w, k, L, c, n);
    }
    fp->off_rec = fp->off_head + round_up(fp->head.ws_bytes);
    fp->total = fp->off_rec + (fp->jump_mask ? round_up(bl::jump_records_bytes(rec_w)) : 0);
    return BITLOGIC_OK;
}

}  // namespace

// ---- adapters: checks and layouts ----

static_assert(bl::adapt::kMaxGroups == BITLOGIC_MAX_ADAPTERS &&
              bl::adapt::kMaxRank == BITLOGIC_MAX_RANK, "the interface's limits");

namespace {

constexpr int64_t kMaxGroupedRows = (int64_t)1 << 27;   // a launch's lanes stay below 2^32
constexpr int64_t kMaxLoneRows = (int64_t)1 << 20;
constexpr int32_t kMaxWidth = 1 << 24;

int check_set(const char *who, const bitlogic_adapter_set *set, int64_t n_rows)
{
    if (!set)
        return fail(BITLOGIC_ERR_NULL, "%s: NULL adapter set", who);
    if (set->weight_type < BITLOGIC_LOGITS_F32 || set->weight_type > BITLOGIC_LOGITS_BF16)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: weights of type %d", who, set->weight_type);
    if (n_rows < 0 || n_rows > kMaxGroupedRows)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need 0 <= n_rows <= 2^27", who);
    if (set->n_adapters < 1 || set->rank < 1 || set->n_in < 1 || set->n_out < 1 ||
        set->n_in > kMaxWidth || set->n_out > kMaxWidth)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need n_adapters >= 1, rank >= 1, 1 <= n_in, n_out "
                    "<= 2^24", who);
    if (set->n_adapters > BITLOGIC_MAX_ADAPTERS || set->rank > BITLOGIC_MAX_RANK)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: %d adapters of rank %d, at most %d of rank %d",
                    who, set->n_adapters, set->rank, BITLOGIC_MAX_ADAPTERS, BITLOGIC_MAX_RANK);
    return BITLOGIC_OK;
}

// x's type, and whether x, base: the weights' type, or int32 beside float32 weights.
int check_beside(const char *who, const char *what, int32_t type, int32_t weight_type)
{
    if (type != weight_type &&
        !(type == BITLOGIC_LOGITS_I32 && weight_type == BITLOGIC_LOGITS_F32))
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: %s of type %d beside weights of type %d", who,
                    what, type, weight_type);
    return BITLOGIC_OK;
}

int check_stride(const char *who, const char *what, int64_t stride, int64_t least)
{
    if (stride < least || stride > kMaxStride)
        return fail(BITLOGIC_ERR_SHAPE, "%s: need %lld <= %s <= 2^30", who, (long long)least,
                    what);
    return BITLOGIC_OK;
}

// Rows by plan or by ids into a pass's arguments.
int take_rows(const char *who, bl::adapt::PassArgs &a, int64_t n_rows, int32_t groups,
              const int32_t *ids, const void *plan)
{
    if (!plan && !ids)
        return fail(BITLOGIC_ERR_NULL, "%s: neither a plan nor ids", who);
    if (!aligned(plan, 16) || !aligned(ids, 4))
        return fail(BITLOGIC_ERR_ALIGN, "%s: plan or ids misaligned", who);
    if (!plan && n_rows > kMaxLoneRows)
        return fail(BITLOGIC_ERR_SHAPE, "%s: more than 2^20 rows need a plan", who);
    a.groups = groups;
    a.n_rows = n_rows;
    if (plan) {
        const auto l = bl::adapt::group_layout(n_rows, groups);
        const char *p = static_cast<const char *>(plan);
        a.tiles = reinterpret_cast<const bl::adapt::Piece4 *>(p + l.tiles);
        a.order = reinterpret_cast<const int32_t *>(p + l.order);
        a.n_tiles = l.n_tiles;
    } else {
        a.ids = ids;
        a.n_tiles = n_rows;
    }
    return BITLOGIC_OK;
}

template <class F>
auto by_weight(int32_t type, F f)
{
    switch (type) {
    case BITLOGIC_LOGITS_F32: return f(std::integral_constant<int, bl::rows::kF32>());
    case BITLOGIC_LOGITS_F16: return f(std::integral_constant<int, bl::rows::kF16>());
    default: return f(std::integral_constant<int, bl::rows::kBf16>());
    }
}

bl::adapt::PassLayout layout_of(int32_t type, int64_t n_rows, int32_t groups, int32_t rank,
                                int32_t k, int32_t m, bool planned, bool back)
{
    const bool narrow = by_weight(type, [&](auto W) {
        return bl::adapt::fits_narrow<decltype(W)::value>(k, m, rank, back);
    });
    return bl::adapt::pass_layout(n_rows, groups, rank, k, (int32_t)logit_bytes(type), planned,
                                  narrow);
}

// A pass's form, and its workspace.
int take_parts(const char *who, bl::adapt::PassArgs &a, int32_t type, bool back, void *workspace,
               size_t workspace_bytes)
{
    const auto l = layout_of(type, a.n_rows, a.groups, a.rank, a.k, a.m, a.tiles != nullptr, back);
    a.splits = l.splits;
    if (!bl::adapt::fits_launches(a, (int32_t)logit_bytes(type), back))
        return fail(BITLOGIC_ERR_UNSUPPORTED, "%s: rows (or adapters) times columns too large for "
                    "one launch", who);
    if (l.splits == 1 && a.hidden) {
        a.partial = a.hidden;
        return BITLOGIC_OK;
    }
    if (l.bytes > 0 && (!workspace || workspace_bytes < l.bytes))
        return fail(BITLOGIC_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who,
                    workspace_bytes, l.bytes);
    if (l.bytes > 0 && !aligned(workspace, 16))
        return fail(BITLOGIC_ERR_ALIGN, "%s: workspace not 16-byte aligned", who);
    a.partial = static_cast<float *>(workspace);
    return BITLOGIC_OK;
}

struct BackwardLayout {
    size_t back, parts, parts_bytes, partial_down, partial_up, bytes;
    int cut;                            // of the plan's two
};

BackwardLayout backward_layout(const bitlogic_adapter_set &s, int64_t n_rows)
{
    const auto l = bl::adapt::group_layout(n_rows, s.n_adapters);
    const int32_t el = (int32_t)logit_bytes(s.weight_type);
    BackwardLayout b;
    // the small cut's chunks, unless the large one's make blocks enough (weights' gradients, us,
    // small and large: 65536 rows of 100 columns 30 and 56, 12289 of 7051 92 and 99, 2^18 of 512
    // 125 and 119)
    const int64_t columns = ((int64_t)s.n_in + s.n_out) * el / 256 + 1;
    b.cut = (n_rows / l.cut[1].rows + 1) * columns >= 768;
    b.back = 0;
    b.parts = round_up((size_t)n_rows * s.rank * 4);
    // a pass by plan or by ids, whichever takes more
    b.parts_bytes = 0;
    for (bool planned : {true, false})
        if (planned || n_rows <= kMaxLoneRows)
            b.parts_bytes = std::max(b.parts_bytes,
                                     layout_of(s.weight_type, n_rows, s.n_adapters, s.rank,
                                               s.n_out, s.n_in, planned, true).bytes);
    b.partial_down = b.parts + round_up(b.parts_bytes);
    const size_t slots = (size_t)l.cut[b.cut].n_slots * s.rank * 4;
    b.partial_up = b.partial_down + round_up(slots * s.n_in);
    b.bytes = b.partial_up + round_up(slots * s.n_out);
    return b;
}

}  // namespace

extern "C" {

int bitlogic_encode(const uint8_t *x, int64_t n_samples, int32_t n_features,
                    const uint8_t *thresholds, int32_t n_thresholds, uint64_t *bits_out,
                    void *stream)
{
    int st = check_encode(x, n_samples, n_features, thresholds, n_thresholds, bits_out);
    if (st != BITLOGIC_OK)
        return st;
    if (n_samples == 0)
        return ok();
    return hip_status(bl::launch_encode(x, n_samples, n_features, thresholds, n_thresholds,
                                        bits_out, bl::kLayoutRowMajor, words_of(n_samples),
                                        (hipStream_t)stream),
                      "encode launch");
}

int bitlogic_lut_layer(const uint64_t *bits_in, int32_t w_in, int64_t n_words,
                       const int32_t *conn, const uint64_t *tables, int32_t w_out, int32_t k,
                       uint64_t *bits_out, void *stream)
{
    int st = check_layer(bits_in, w_in, n_words, conn, tables, w_out, k, bits_out, "lut_layer");
    if (st != BITLOGIC_OK)
        return st;
    if (n_words == 0)
        return ok();
    return hip_status(bl::launch_lut_layer(bits_in, w_in, n_words, conn, tables, w_out, k,
                                           bits_out, (hipStream_t)stream),
                      "lut_layer launch");
}

size_t bitlogic_groupsum_head_workspace_bytes(int32_t w, int64_t n_samples, int32_t n_classes)
{
    if (w <= 0 || n_classes <= 0 || n_samples < 0 || w % n_classes != 0 ||
        w / n_classes > 65535 || n_samples > ((int64_t)1 << 40))
        return 0;
    return bl::plan_head(w, n_samples, n_classes).ws_bytes;
}

int bitlogic_groupsum_head(const uint64_t *bits, int32_t w, int64_t n_samples,
                           int32_t n_classes, int32_t *scores, int32_t *argmax,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    int st = check_head(bits, w, n_samples, n_classes, scores, argmax);
    if (st != BITLOGIC_OK)
        return st;
    const bl::HeadPlan plan = bl::plan_head(w, n_samples, n_classes);
    if (plan.ws_bytes > 0 && !workspace)
        return fail(BITLOGIC_ERR_NULL, "head: NULL workspace");
    if (workspace_bytes < plan.ws_bytes)
        return fail(BITLOGIC_ERR_WORKSPACE, "head: workspace %zu < %zu bytes", workspace_bytes,
                    plan.ws_bytes);
    if (workspace && !aligned(workspace, kWsAlign))
        return fail(BITLOGIC_ERR_ALIGN, "head: workspace not 256-byte aligned");
    if (n_samples == 0)
        return ok();
    return hip_status(bl::launch_head(bits, w, n_samples, n_classes, scores, argmax, nullptr,
                                      workspace, plan, bl::kLayoutRowMajor,
                                      (hipStream_t)stream),
                      "head launch");
}

size_t bitlogic_forward_workspace_bytes(int64_t n_samples, int32_t n_features,
                                        int32_t n_thresholds, const bitlogic_layer *layers,
                                        int32_t n_layers, int32_t n_classes)
{
    ForwardPlan fp;
    if (plan_forward(n_samples, n_features, n_thresholds, layers, n_layers, n_classes, nullptr,
                     &fp) != BITLOGIC_OK)
        return 0;
    return fp.total;
}

int bitlogic_forward_plan(int64_t n_samples, int32_t n_features, int32_t n_thresholds,
                          const bitlogic_layer *layers, int32_t n_layers, int32_t n_classes,
                          bitlogic_forward_info *info)
{
    // the descriptor bitlogic_forward builds; a placeholder stands in for the
    // threshold pointer, which planning never reads
    static const uint8_t kPlaceholder = 0;
    const bitlogic_network net =
        legacy_net(n_features, &kPlaceholder, n_thresholds, layers, n_layers, n_classes, nullptr);
    return bitlogic_network_plan(&net, n_samples, info);
}

}  // extern "C"

namespace {

// Checks of a network descriptor beyond the shapes that plan_forward checks.
int check_network(const bitlogic_network *net)
{
    if (!net)
        return fail(BITLOGIC_ERR_NULL, "network: NULL descriptor");
    if (net->encoder == BITLOGIC_ENCODER_THERMOMETER) {
        if (!net->thresholds)
            return fail(BITLOGIC_ERR_NULL, "network: thermometer needs thresholds");
    } else if (net->encoder == BITLOGIC_ENCODER_BINARY) {
        if (net->n_bits < 1 || net->n_bits > 8)
            return fail(BITLOGIC_ERR_UNSUPPORTED, "network: binary code of %d bits (1..8)",
                        net->n_bits);
    } else {
        return fail(BITLOGIC_ERR_UNSUPPORTED, "network: unknown encoder %d", net->encoder);
    }
    if (net->head == BITLOGIC_HEAD_GROUPED_DSP) {
        if (!net->head_weights)
            return fail(BITLOGIC_ERR_NULL, "network: quantized head needs weights");
        if (net->n_classes > kDspMaxClasses)
            return fail(BITLOGIC_ERR_UNSUPPORTED, "network: quantized head needs n_classes <= %d",
                        kDspMaxClasses);
    } else if (net->head != BITLOGIC_HEAD_GROUPSUM) {
        return fail(BITLOGIC_ERR_UNSUPPORTED, "network: unknown head %d", net->head);
    }
    return BITLOGIC_OK;
}

int plan_network(const bitlogic_network *net, int64_t n, ForwardPlan *fp)
{
    int st = check_network(net);
    if (st != BITLOGIC_OK)
        return st;
    st = plan_forward(n, net->n_features, net->n_bits, net->layers, net->n_layers,
                      net->n_classes, net->pass_fanin, fp);
    if (st != BITLOGIC_OK)
        return st;
    return BITLOGIC_OK;
}

// The forward of a small batch by 64-sample columns (columns.hip).  mark(i)
// records event i of the timed variant.
template <class Mark>
int forward_columns(const bitlogic_network *net, const ForwardPlan &fp, const uint8_t *x,
                    int64_t n, int32_t *scores, int32_t *argmax, uint64_t *enc,
                    uint64_t *const (&act)[2], hipStream_t s, bool timed, Mark mark)
{
    const bitlogic_layer *layers = net->layers;
    const int32_t L = net->n_layers, c = net->n_classes;
    const int kind = net->encoder == BITLOGIC_ENCODER_BINARY ? bl::kEncBinary
                                                             : bl::kEncThermometer;
    const bool dsp = net->head == BITLOGIC_HEAD_GROUPED_DSP;
    // the counts: the caller's scores, or scratch where they are not wanted
    int32_t *counts = !dsp && scores ? scores : reinterpret_cast<int32_t *>(enc);
    hipError_t e = mark(0);
    // one kernel for the whole network where a column fits a block; a timed
    // forward has stages to tell apart
    if (e == hipSuccess && !timed && fp.net.ok) {
        bl::ColumnNetwork cn = fp.net;
        for (int32_t l = 0; l < L; ++l) {
            cn.conn[l] = layers[l].conn;
            cn.tables[l] = layers[l].tables;
            cn.fanin[l] = net->pass_fanin ? net->pass_fanin[l] : nullptr;
        }
        e = bl::launch_column_network(x, n, net->n_features, net->thresholds, net->n_bits, kind,
                                      cn, c, !dsp && !scores ? nullptr : counts,
                                      dsp ? nullptr : argmax, s);
        if (e == hipSuccess && dsp)
            e = bl::launch_grouped_dsp(counts, n, c, net->head_weights, scores, argmax, s);
        return hip_status(e, "forward: network launch");
    }
    if (e == hipSuccess)
        e = bl::launch_column_encode(x, n, net->n_features, net->thresholds, net->n_bits, enc,
                                     kind, s);
    if (e == hipSuccess)
        e = mark(1);
    if (e != hipSuccess)
        return hip_status(e, "forward: encode launch");
    const uint64_t *cur = enc;
    int32_t w_in = net->n_features * net->n_bits;
    for (int32_t l = 0; l < L - 1; ++l) {
        e = bl::launch_column_layer(cur, w_in, (int32_t)fp.W, layers[l].conn, layers[l].tables,
                                    layers[l].w_out, layers[l].k, act[l & 1],
                                    net->pass_fanin ? net->pass_fanin[l] : nullptr, s);
        if (e == hipSuccess)
            e = mark(2 + l);
        if (e != hipSuccess)
            return fail(BITLOGIC_ERR_HIP, "forward: layer %d launch: %s", l, hipGetErrorString(e));
        cur = act[l & 1];
        w_in = layers[l].w_out;
    }
    e = bl::launch_column_head(cur, w_in, layers[L - 1].conn, layers[L - 1].tables,
                               layers[L - 1].w_out, layers[L - 1].k, c, n, fp.cols, counts,
                               dsp ? nullptr : argmax,
                               net->pass_fanin ? net->pass_fanin[L - 1] : nullptr, s);
    if (e == hipSuccess)
        e = mark(L + 1);
    if (e == hipSuccess && dsp)
        e = bl::launch_grouped_dsp(counts, n, c, net->head_weights, scores, argmax, s);
    if (e == hipSuccess)
        e = mark(L + 2);
    return hip_status(e, "forward: head launch");
}

int forward_impl(const bitlogic_network *net, const uint8_t *x, int64_t n_samples,
                 int32_t *scores, int32_t *argmax, void *workspace, size_t workspace_bytes,
                 void *stream, void *const *events, int32_t n_events)
{
    ForwardPlan fp;
    int st = plan_network(net, n_samples, &fp);
    if (st != BITLOGIC_OK)
        return st;
    if (!x || (!scores && !argmax))
        return fail(BITLOGIC_ERR_NULL, "forward: NULL pixels or both outputs NULL");
    if (!workspace)
        return fail(BITLOGIC_ERR_NULL, "forward: NULL workspace");
    if (workspace_bytes < fp.total)
        return fail(BITLOGIC_ERR_WORKSPACE, "forward: workspace %zu < %zu bytes",
                    workspace_bytes, fp.total);
    if (!aligned(workspace, kWsAlign))
        return fail(BITLOGIC_ERR_ALIGN, "forward: workspace not 256-byte aligned");
    if ((scores && !aligned(scores, 4)) || (argmax && !aligned(argmax, 4)))
        return fail(BITLOGIC_ERR_ALIGN, "forward: misaligned output");
    const int32_t n_layers = net->n_layers;
    if (events) {
        if (n_events != n_layers + 3)
            return fail(BITLOGIC_ERR_SHAPE, "forward_timed: need %d events, got %d",
                        n_layers + 3, n_events);
        for (int32_t i = 0; i < n_events; ++i)
            if (!events[i])
                return fail(BITLOGIC_ERR_NULL, "forward_timed: event %d is NULL", i);
    }
    if (n_samples == 0)
        return ok();

    const bitlogic_layer *layers = net->layers;
    const int32_t n_classes = net->n_classes;
    const int8_t *dsp = net->head == BITLOGIC_HEAD_GROUPED_DSP ? net->head_weights : nullptr;
    hipStream_t s = (hipStream_t)stream;
    auto mark = [&](int i) -> hipError_t {
        return events ? hipEventRecord((hipEvent_t)events[i], s) : hipSuccess;
    };
    char *ws = static_cast<char *>(workspace);
    uint64_t *enc = reinterpret_cast<uint64_t *>(ws + fp.off_enc);
    uint64_t *act[2] = {reinterpret_cast<uint64_t *>(ws + fp.off_a),
                        reinterpret_cast<uint64_t *>(ws + fp.off_b)};
    if (fp.cols.ok)
        return forward_columns(net, fp, x, n_samples, scores, argmax, enc, act, s,
                               events != nullptr, mark);
    hipError_t e = mark(0);
    if (e == hipSuccess)
        e = bl::launch_encode(x, n_samples, net->n_features, net->thresholds, net->n_bits, enc,
                              bl::kLayoutSlab, fp.n_slabs * bl::kSlabWords, s,
                              net->encoder == BITLOGIC_ENCODER_BINARY ? bl::kEncBinary
                                                                      : bl::kEncThermometer);
    if (e == hipSuccess)
        e = mark(1);
    if (e != hipSuccess)
        return hip_status(e, "forward: encode launch");
    const uint64_t *cur = enc;
    int32_t w_in = net->n_features * net->n_bits;
    uint64_t *planes = reinterpret_cast<uint64_t *>(ws + fp.off_head);
    uint32_t *rec = reinterpret_cast<uint32_t *>(ws + fp.off_rec);
    for (int32_t l = 0; l < n_layers; ++l) {
        const bool last_fused = fp.fused && l == n_layers - 1;
        uint64_t *dst = act[l & 1];
        const uint8_t *fanin = net->pass_fanin ? net->pass_fanin[l] : nullptr;
        if (last_fused)
            e = bl::launch_lut_slab_head(cur, w_in, fp.n_slabs, layers[l].conn, layers[l].tables,
                                         layers[l].w_out, layers[l].k, n_classes, fp.W, planes,
                                         fp.head.planes, s, fanin);
        else if ((fp.jump_mask >> l) & 1)
            e = bl::launch_jump_layer(cur, w_in, fp.n_slabs, layers[l].conn, layers[l].tables,
                                      layers[l].w_out, layers[l].k, dst, rec, s);
        else
            e = bl::launch_lut_layer_slab(cur, w_in, fp.n_slabs, layers[l].conn,
                                          layers[l].tables, layers[l].w_out, layers[l].k, dst, s,
                                          fanin);
        if (e == hipSuccess)
            e = mark(2 + l);
        if (e != hipSuccess)
            return fail(BITLOGIC_ERR_HIP, "forward: layer %d launch: %s", l, hipGetErrorString(e));
        cur = dst;
        w_in = layers[l].w_out;
    }
    if (fp.fused)
        e = bl::launch_head_finish(planes, n_samples, n_classes, scores, argmax, dsp, fp.head, s);
    else
        e = bl::launch_head(cur, w_in, n_samples, n_classes, scores, argmax, dsp, planes,
                            fp.head, bl::kLayoutSlab, s);
    if (e == hipSuccess)
        e = mark(n_layers + 2);
    return hip_status(e, "forward: head launch");
}

// The descriptor of the legacy entry points' arguments.
bitlogic_network legacy_net(int32_t n_features, const uint8_t *thresholds, int32_t n_thresholds,
                            const bitlogic_layer *layers, int32_t n_layers, int32_t n_classes,
                            const int8_t *dsp_weights)
{
    bitlogic_network net;
    net.n_features = n_features;
    net.encoder = BITLOGIC_ENCODER_THERMOMETER;
    net.n_bits = n_thresholds;
    net.thresholds = thresholds;
    net.layers = layers;
    net.n_layers = n_layers;
    net.n_classes = n_classes;
    net.head = dsp_weights ? BITLOGIC_HEAD_GROUPED_DSP : BITLOGIC_HEAD_GROUPSUM;
    net.head_weights = dsp_weights;
    net.pass_fanin = nullptr;
    return net;
}

}  // namespace

extern "C" {

int bitlogic_forward(const uint8_t *x, int64_t n_samples, int32_t n_features,
                     const uint8_t *thresholds, int32_t n_thresholds,
                     const bitlogic_layer *layers, int32_t n_layers, int32_t n_classes,
                     int32_t *scores, int32_t *argmax, void *workspace, size_t workspace_bytes,
                     void *stream)
{
    if (!thresholds)
        return fail(BITLOGIC_ERR_NULL, "forward: NULL thresholds");
    const bitlogic_network net =
        legacy_net(n_features, thresholds, n_thresholds, layers, n_layers, n_classes, nullptr);
    return forward_impl(&net, x, n_samples, scores, argmax, workspace, workspace_bytes, stream,
                        nullptr, 0);
}

int bitlogic_forward_grouped_dsp(const uint8_t *x, int64_t n_samples, int32_t n_features,
                                 const uint8_t *thresholds, int32_t n_thresholds,
                                 const bitlogic_layer *layers, int32_t n_layers,
                                 int32_t n_classes, const int8_t *weights, int32_t *logits,
                                 int32_t *argmax, void *workspace, size_t workspace_bytes,
                                 void *stream)
{
    if (!weights)
        return fail(BITLOGIC_ERR_NULL, "forward_grouped_dsp: NULL weights");
    if (!thresholds)
        return fail(BITLOGIC_ERR_NULL, "forward: NULL thresholds");
    const bitlogic_network net =
        legacy_net(n_features, thresholds, n_thresholds, layers, n_layers, n_classes, weights);
    return forward_impl(&net, x, n_samples, logits, argmax, workspace, workspace_bytes, stream,
                        nullptr, 0);
}

int bitlogic_grouped_dsp_head(const int32_t *counts, int64_t n_samples, int32_t n_classes,
                              const int8_t *weights, int32_t *logits, int32_t *argmax,
                              void *stream)
{
    if (!counts || !weights || (!logits && !argmax))
        return fail(BITLOGIC_ERR_NULL, "grouped_dsp_head: NULL counts/weights or both outputs");
    if (n_samples < 0 || n_classes < 1 || n_samples > ((int64_t)1 << 40))
        return fail(BITLOGIC_ERR_SHAPE, "grouped_dsp_head: need n_samples >= 0, n_classes >= 1");
    if (n_classes > kDspMaxClasses)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "grouped_dsp_head: n_classes %d > %d", n_classes,
                    kDspMaxClasses);
    if (!aligned(counts, 4) || (logits && !aligned(logits, 4)) || (argmax && !aligned(argmax, 4)))
        return fail(BITLOGIC_ERR_ALIGN, "grouped_dsp_head: misaligned buffer");
    if (n_samples == 0)
        return ok();
    return hip_status(bl::launch_grouped_dsp(counts, n_samples, n_classes, weights, logits, argmax,
                                             (hipStream_t)stream),
                      "grouped_dsp_head launch");
}

int bitlogic_forward_timed(const uint8_t *x, int64_t n_samples, int32_t n_features,
                           const uint8_t *thresholds, int32_t n_thresholds,
                           const bitlogic_layer *layers, int32_t n_layers, int32_t n_classes,
                           int32_t *scores, int32_t *argmax, void *workspace,
                           size_t workspace_bytes, void *stream, void *const *events,
                           int32_t n_events)
{
    if (!events)
        return fail(BITLOGIC_ERR_NULL, "forward_timed: NULL event array");
    if (!thresholds)
        return fail(BITLOGIC_ERR_NULL, "forward: NULL thresholds");
    const bitlogic_network net =
        legacy_net(n_features, thresholds, n_thresholds, layers, n_layers, n_classes, nullptr);
    return forward_impl(&net, x, n_samples, scores, argmax, workspace, workspace_bytes, stream,
                        events, n_events);
}

size_t bitlogic_network_workspace_bytes(const bitlogic_network *net, int64_t n_samples)
{
    ForwardPlan fp;
    if (plan_network(net, n_samples, &fp) != BITLOGIC_OK)
        return 0;
    return fp.total;
}

int bitlogic_network_plan(const bitlogic_network *net, int64_t n_samples,
                          bitlogic_forward_info *info)
{
    if (!info)
        return fail(BITLOGIC_ERR_NULL, "network_plan: NULL info");
    ForwardPlan fp;
    int st = plan_network(net, n_samples, &fp);
    if (st != BITLOGIC_OK)
        return st;
    info->workspace_bytes = fp.total;
    info->slab_words = bl::kSlabWords;
    info->fused_head = fp.fused ? 1 : 0;
    info->head_splits = fp.head.splits;
    info->head_planes = fp.head.planes;
    info->jump_layers = (uint32_t)(fp.jump_mask & 0xFFFFFFFFu);
    return ok();
}

int bitlogic_network_path(const bitlogic_network *net, int64_t n_samples, int32_t *path)
{
    if (!path)
        return fail(BITLOGIC_ERR_NULL, "network_path: NULL path");
    ForwardPlan fp;
    int st = plan_network(net, n_samples, &fp);
    if (st != BITLOGIC_OK)
        return st;
    *path = !fp.cols.ok ? BITLOGIC_PATH_SLAB
            : fp.net.ok ? BITLOGIC_PATH_BLOCK
                        : BITLOGIC_PATH_COLUMNS;
    return ok();
}

int bitlogic_network_forward(const bitlogic_network *net, const uint8_t *x, int64_t n_samples,
                             int32_t *out, int32_t *argmax, void *workspace,
                             size_t workspace_bytes, void *stream, void *const *events,
                             int32_t n_events)
{
    return forward_impl(net, x, n_samples, out, argmax, workspace, workspace_bytes, stream,
                        events, events ? n_events : 0);
}

}  // extern "C"

namespace {

constexpr int kMaxDevices = 64;
std::atomic<void *> g_scratch_ptr[kMaxDevices];
std::mutex g_scratch_mu;

// Device address of `scratch` on device dev (the current device), looked up
// on the first call for that device.
int scratch_address(int dev, void **ptr)
{
    void *p = g_scratch_ptr[dev].load(std::memory_order_acquire);
    if (!p) {
        std::lock_guard<std::mutex> lock(g_scratch_mu);
        p = g_scratch_ptr[dev].load(std::memory_order_relaxed);
        if (!p) {
            hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
            if (e != hipSuccess || !p)
                return fail(BITLOGIC_ERR_HIP, "forward_noalloc: scratch address on device %d: %s",
                            dev, hipGetErrorString(e));
            g_scratch_ptr[dev].store(p, std::memory_order_release);
        }
    }
    *ptr = p;
    return BITLOGIC_OK;
}

}  // namespace

extern "C" {

int bitlogic_network_forward_noalloc(const bitlogic_network *net, const uint8_t *x,
                                     int64_t n_samples, int32_t *out, int32_t *argmax,
                                     void *stream)
{
    // every argument check before the first HIP call
    ForwardPlan fp;
    int st = plan_network(net, n_samples, &fp);
    if (st != BITLOGIC_OK)
        return st;
    if (!x || (!out && !argmax))
        return fail(BITLOGIC_ERR_NULL, "forward_noalloc: NULL pixels or both outputs NULL");
    if ((out && !aligned(out, 4)) || (argmax && !aligned(argmax, 4)))
        return fail(BITLOGIC_ERR_ALIGN, "forward_noalloc: misaligned output");
    if (fp.total > (size_t)BITLOGIC_NOALLOC_SCRATCH_BYTES)
        return fail(BITLOGIC_ERR_WORKSPACE,
                    "forward_noalloc: %lld samples need %zu bytes of scratch, the static buffer "
                    "holds %zu (use bitlogic_network_forward with a workspace)",
                    (long long)n_samples, fp.total, (size_t)BITLOGIC_NOALLOC_SCRATCH_BYTES);
    if (n_samples == 0)
        return ok();
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return hip_status(e, "forward_noalloc: current device");
    if (dev < 0 || dev >= kMaxDevices)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "forward_noalloc: device %d beyond %d", dev,
                    kMaxDevices);
    if (stream) {
        hipDevice_t sdev = 0;
        e = hipStreamGetDevice((hipStream_t)stream, &sdev);
        if (e != hipSuccess)
            return hip_status(e, "forward_noalloc: stream device");
        if (sdev != dev)
            return fail(BITLOGIC_ERR_UNSUPPORTED,
                        "forward_noalloc: stream of device %d, current device %d", (int)sdev, dev);
    }
    void *ws = nullptr;
    st = scratch_address(dev, &ws);
    if (st != BITLOGIC_OK)
        return st;
    return forward_impl(net, x, n_samples, out, argmax, ws, BITLOGIC_NOALLOC_SCRATCH_BYTES,
                        stream, nullptr, 0);
}

int bitlogic_encode_binary(const uint8_t *x, int64_t n_samples, int32_t n_features,
                           int32_t n_bits, uint64_t *bits_out, void *stream)
{
    if (!x || !bits_out)
        return fail(BITLOGIC_ERR_NULL, "encode_binary: NULL pointer");
    if (n_samples < 0 || n_features <= 0 || n_bits < 1 || n_bits > 8)
        return fail(BITLOGIC_ERR_SHAPE, "encode_binary: need n >= 0, d > 0, 1 <= n_bits <= 8");
    if ((int64_t)n_features * n_bits > kMaxRows)
        return fail(BITLOGIC_ERR_SHAPE, "encode_binary: d * n_bits exceeds int32");
    if (!aligned(bits_out, 8))
        return fail(BITLOGIC_ERR_ALIGN, "encode_binary: bits_out not 8-byte aligned");
    if (n_samples == 0)
        return ok();
    return hip_status(bl::launch_encode(x, n_samples, n_features, nullptr, n_bits, bits_out,
                                        bl::kLayoutRowMajor, words_of(n_samples),
                                        (hipStream_t)stream, bl::kEncBinary),
                      "encode_binary launch");
}

int bitlogic_specialize_layer(const int32_t *conn, const uint64_t *tables, int32_t w_out,
                              int32_t k, int32_t w_in, int32_t *k_eff, int32_t *conn_out,
                              uint64_t *tables_out)
{
    if (!conn || !tables || !k_eff || !conn_out || !tables_out)
        return fail(BITLOGIC_ERR_NULL, "specialize_layer: NULL pointer");
    if (k < 1 || k > 6)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "specialize_layer: fan-in %d outside 1..6", k);
    if (w_out < 0 || w_in <= 0)
        return fail(BITLOGIC_ERR_SHAPE, "specialize_layer: need w_out >= 0, w_in > 0");
    for (int64_t q = 0; q < (int64_t)w_out * k; ++q)
        if (conn[q] < 0 || conn[q] >= w_in)
            return fail(BITLOGIC_ERR_SHAPE, "specialize_layer: connection %lld = %d outside [0, %d)",
                        (long long)q, conn[q], w_in);
    for (int32_t j = 0; j < w_out; ++j) {
        int32_t *co = conn_out + (int64_t)j * k;
        k_eff[j] = bl::specialize_node(conn + (int64_t)j * k, tables[j], k, co, &tables_out[j]);
        for (int i = k_eff[j]; i < k; ++i)
            co[i] = 0;
    }
    return ok();
}

int bitlogic_specialize_network(int32_t w_in, const int32_t *const *conn,
                                const uint64_t *const *tables, const int32_t *w_out,
                                const int32_t *k, int32_t n_layers, int32_t n_classes,
                                double min_gain, int32_t *k_out, int32_t *applied_out,
                                int32_t *const *conn_out, uint64_t *const *tables_out,
                                uint8_t *const *fanin_out, int32_t *const *order_out)
{
    if (!conn || !tables || !w_out || !k || !k_out || !applied_out || !conn_out || !tables_out ||
        !fanin_out)
        return fail(BITLOGIC_ERR_NULL, "specialize_network: NULL pointer");
    if (n_layers < 1 || w_in <= 0 || n_classes < 1)
        return fail(BITLOGIC_ERR_SHAPE, "specialize_network: need n_layers, w_in, n_classes > 0");
    int32_t wi = w_in;
    for (int32_t l = 0; l < n_layers; ++l) {
        if (!conn[l] || !tables[l] || !conn_out[l] || !tables_out[l] || !fanin_out[l] ||
            (order_out && !order_out[l]))
            return fail(BITLOGIC_ERR_NULL, "specialize_network: layer %d NULL pointer", l);
        if (k[l] < 1 || k[l] > 6)
            return fail(BITLOGIC_ERR_UNSUPPORTED, "specialize_network: layer %d fan-in %d", l,
                        k[l]);
        if (w_out[l] <= 0)
            return fail(BITLOGIC_ERR_SHAPE, "specialize_network: layer %d width %d", l, w_out[l]);
        for (int64_t q = 0; q < (int64_t)w_out[l] * k[l]; ++q)
            if (conn[l][q] < 0 || conn[l][q] >= wi)
                return fail(BITLOGIC_ERR_SHAPE,
                            "specialize_network: layer %d connection %lld = %d outside [0, %d)",
                            l, (long long)q, conn[l][q], wi);
        wi = w_out[l];
    }
    if (wi % n_classes != 0)
        return fail(BITLOGIC_ERR_SHAPE, "specialize_network: last width %d not a multiple of %d",
                    wi, n_classes);
    if (!(min_gain >= 0.0 && min_gain <= 1.0))
        return fail(BITLOGIC_ERR_SHAPE, "specialize_network: min_gain outside [0, 1]");
    bl::specialize_network(w_in, n_layers, w_out, k, conn, tables, n_classes, min_gain, k_out,
                           applied_out, conn_out, tables_out, fanin_out, order_out);
    return ok();
}

size_t bitlogic_fit_quantile_thresholds_workspace_bytes(int32_t n_groups)
{
    if (n_groups < 1 || n_groups > bl::kFitMaxGroups)
        return 0;
    return (size_t)n_groups * 256 * sizeof(uint64_t);
}

int bitlogic_fit_quantile_thresholds(const uint8_t *x, int64_t n_samples, int32_t n_features,
                                     int32_t n_thresholds, int32_t n_groups,
                                     uint8_t *thresholds_out, void *workspace,
                                     size_t workspace_bytes, void *stream)
{
    if (!x || !thresholds_out || !workspace)
        return fail(BITLOGIC_ERR_NULL, "fit_quantiles: NULL pointer");
    if (n_samples < 1 || n_features < 1 || n_thresholds < 1 || n_thresholds > 64)
        return fail(BITLOGIC_ERR_SHAPE, "fit_quantiles: need n >= 1, d >= 1, 1 <= b <= 64");
    if (n_groups < 1 || n_groups > bl::kFitMaxGroups || n_features % n_groups != 0)
        return fail(BITLOGIC_ERR_SHAPE, "fit_quantiles: %d groups of %d features", n_groups,
                    n_features);
    if (n_samples > ((int64_t)1 << 56) / n_features)
        return fail(BITLOGIC_ERR_SHAPE, "fit_quantiles: n * d exceeds 2^56");
    if (workspace_bytes < bitlogic_fit_quantile_thresholds_workspace_bytes(n_groups))
        return fail(BITLOGIC_ERR_WORKSPACE, "fit_quantiles: workspace too small");
    if (!aligned(workspace, 8))
        return fail(BITLOGIC_ERR_ALIGN, "fit_quantiles: workspace not 8-byte aligned");
    return hip_status(bl::launch_fit_quantiles(x, n_samples, n_features, n_thresholds, n_groups,
                                               thresholds_out,
                                               static_cast<uint64_t *>(workspace),
                                               (hipStream_t)stream),
                      "fit_quantiles launch");
}

const char *bitlogic_status_string(int status)
{
    switch (status) {
    case BITLOGIC_OK: return "ok";
    case BITLOGIC_ERR_NULL: return "a required pointer is NULL";
    case BITLOGIC_ERR_SHAPE: return "a size is out of range or inconsistent";
    case BITLOGIC_ERR_ALIGN: return "a buffer is not aligned as required";
    case BITLOGIC_ERR_UNSUPPORTED: return "unsupported parameter";
    case BITLOGIC_ERR_HIP: return "HIP runtime error";
    case BITLOGIC_ERR_WORKSPACE: return "workspace too small";
    default: return "unknown status";
    }
}

const char *bitlogic_last_error(void) { return g_last_error; }

int bitlogic_version(void) { return BITLOGIC_VERSION; }

// ---- rows of class scores or logits ----

static_assert(bl::rows::kI32 == BITLOGIC_LOGITS_I32 && bl::rows::kF32 == BITLOGIC_LOGITS_F32 &&
              bl::rows::kF16 == BITLOGIC_LOGITS_F16 && bl::rows::kBf16 == BITLOGIC_LOGITS_BF16,
              "the kernels' element types are the interface's");

int bitlogic_top_logits(const void *logits, int32_t type, int64_t n_rows, int32_t n_classes,
                        int64_t row_stride, int32_t k, float temperature, void *values,
                        int32_t *indices, float *log_norm, void *stream)
{
    if (int rc = check_rows("top_logits", type, n_rows, n_classes, row_stride))
        return rc;
    if (int rc = check_list("top_logits", k, temperature))
        return rc;
    if (n_rows == 0)
        return ok();
    if (!logits || !values || !indices)
        return fail(BITLOGIC_ERR_NULL, "top_logits: NULL pointer");
    if (!aligned(logits, logit_bytes(type)) || !aligned(values, logit_bytes(type)) ||
        !aligned(indices, 4) || !aligned(log_norm, 4))
        return fail(BITLOGIC_ERR_ALIGN, "top_logits: misaligned buffer");
    return hip_status(bl::launch_top_logits(logits, type, n_rows, n_classes, row_stride, k,
                                            bl::rows::inverse(temperature), values, indices,
                                            log_norm, (hipStream_t)stream),
                      "top_logits launch");
}

int bitlogic_distill(const void *logits, int32_t type, int64_t n_rows, int32_t n_classes,
                     int64_t row_stride, float temperature, const void *top_values,
                     int32_t top_type, const int32_t *top_indices, int32_t k,
                     const float *top_log_norm, float top_temperature,
                     const float *row_weight, float *loss, void *grad, int64_t grad_stride,
                     void *stream)
{
    if (int rc = check_rows("distill", type, n_rows, n_classes, row_stride))
        return rc;
    if (int rc = check_rows("distill", top_type, n_rows, n_classes, 0))
        return rc;
    if (int rc = check_list("distill", k, temperature))
        return rc;
    if (int rc = check_list("distill", k, top_temperature))
        return rc;
    if (grad && type == BITLOGIC_LOGITS_I32)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "distill: int32 scores have no gradient");
    if (grad && (grad_stride < n_classes || grad_stride > kMaxStride))
        return fail(BITLOGIC_ERR_SHAPE, "distill: need n_classes <= grad_stride <= 2^30");
    if (n_rows == 0)
        return ok();
    if (!logits || !top_values || !top_indices || (!loss && !grad))
        return fail(BITLOGIC_ERR_NULL, "distill: NULL input, or both outputs NULL");
    if (!aligned(logits, logit_bytes(type)) || !aligned(grad, logit_bytes(type)) ||
        !aligned(top_values, logit_bytes(top_type)) || !aligned(top_indices, 4) ||
        !aligned(top_log_norm, 4) || !aligned(row_weight, 4) || !aligned(loss, 4))
        return fail(BITLOGIC_ERR_ALIGN, "distill: misaligned buffer");
    return hip_status(bl::launch_distill(logits, type, n_rows, n_classes, row_stride,
                                         bl::rows::inverse(temperature), top_values, top_type,
                                         top_indices, k, top_log_norm,
                                         bl::rows::inverse(top_temperature), row_weight, loss,
                                         grad, grad_stride, (hipStream_t)stream),
                      "distill launch");
}

int bitlogic_sample(const void *logits, int32_t type, int64_t n_rows, int32_t n_classes,
                    int64_t row_stride, const float *noise, int64_t noise_stride,
                    const bitlogic_sampling *sampling, int32_t *token, float *log_prob,
                    void *stream)
{
    if (int rc = check_rows("sample", type, n_rows, n_classes, row_stride))
        return rc;
    if (!sampling)
        return fail(BITLOGIC_ERR_NULL, "sample: NULL sampling parameters");
    if (noise_stride < 0 || noise_stride > kMaxStride)
        return fail(BITLOGIC_ERR_SHAPE, "sample: need 0 <= noise_stride <= 2^30");
    const bitlogic_sampling &s = *sampling;
    if (!s.temperatures && !(s.temperature >= 0.0f && s.temperature <= FLT_MAX))
        return fail(BITLOGIC_ERR_SHAPE, "sample: temperature %g is not in [0, inf)",
                    (double)s.temperature);
    if (!s.top_ks && s.top_k < 0)
        return fail(BITLOGIC_ERR_SHAPE, "sample: top_k %d < 0", s.top_k);
    if (!s.top_ps && !(s.top_p >= 0.0f && s.top_p <= 1.0f))
        return fail(BITLOGIC_ERR_SHAPE, "sample: top_p %g is not in [0, 1]", (double)s.top_p);
    if (!s.min_ps && !(s.min_p >= 0.0f && s.min_p <= 1.0f))
        return fail(BITLOGIC_ERR_SHAPE, "sample: min_p %g is not in [0, 1]", (double)s.min_p);
    if (n_rows == 0)
        return ok();
    const bool greedy = !s.temperatures && s.temperature == 0.0f;
    if (!logits || !token || (!noise && !greedy))
        return fail(BITLOGIC_ERR_NULL, "sample: NULL pointer");
    if (!aligned(logits, logit_bytes(type)) || !aligned(noise, 4) || !aligned(token, 4) ||
        !aligned(log_prob, 4) || !aligned(s.temperatures, 4) || !aligned(s.top_ks, 4) ||
        !aligned(s.top_ps, 4) || !aligned(s.min_ps, 4))
        return fail(BITLOGIC_ERR_ALIGN, "sample: misaligned buffer");
    const bl::SampleParams sp = {s.temperature, s.top_p, s.min_p, s.top_k,
                                 s.temperatures, s.top_ps, s.min_ps, s.top_ks};
    return hip_status(bl::launch_sample(logits, type, n_rows, n_classes, row_stride, noise,
                                        noise_stride, sp, token, log_prob, (hipStream_t)stream),
                      "sample launch");
}

size_t bitlogic_verify_workspace_bytes(int64_t n_requests, int32_t n_drafted,
                                       int32_t n_classes)
{
    if (n_requests < 0 || n_drafted < 0 || n_requests > kMaxRows / ((int64_t)n_drafted + 1) ||
        n_classes < 1 || n_classes > bl::rows::kMaxClasses)
        return 0;
    return bl::verify_workspace_bytes(n_requests, n_drafted, n_classes);
}

int bitlogic_verify(const void *logits, int32_t type, int64_t n_requests, int32_t n_classes,
                    int64_t row_stride, int64_t request_stride, const bitlogic_drafts *drafts,
                    const float *noise, int64_t noise_stride, int32_t *accepted,
                    int32_t *token, float *log_prob, void *workspace, size_t workspace_bytes,
                    void *stream)
{
    if (int rc = check_rows("verify", type, n_requests, n_classes, row_stride))
        return rc;
    if (!drafts)
        return fail(BITLOGIC_ERR_NULL, "verify: NULL drafts");
    const bitlogic_drafts &d = *drafts;
    if (d.n_drafted < 0 || n_requests > kMaxRows / ((int64_t)d.n_drafted + 1))
        return fail(BITLOGIC_ERR_SHAPE, "verify: need n_drafted >= 0, n_requests * "
                    "(n_drafted + 1) < 2^31");
    if (request_stride < 0 || request_stride > kMaxRequestStride)
        return fail(BITLOGIC_ERR_SHAPE, "verify: need 0 <= request_stride <= 2^40");
    if (d.draft_logits) {
        if (int rc = check_rows("verify", d.draft_type, n_requests, n_classes,
                                d.draft_row_stride))
            return rc;
        if (d.draft_request_stride < 0 || d.draft_request_stride > kMaxRequestStride)
            return fail(BITLOGIC_ERR_SHAPE, "verify: need 0 <= draft_request_stride <= 2^40");
    }
    if (noise_stride < 0 || noise_stride > kMaxStride)
        return fail(BITLOGIC_ERR_SHAPE, "verify: need 0 <= noise_stride <= 2^30");
    if (!d.temperatures && !(d.temperature >= 0.0f && d.temperature <= FLT_MAX))
        return fail(BITLOGIC_ERR_SHAPE, "verify: temperature %g is not in [0, inf)",
                    (double)d.temperature);
    if (!d.draft_temperatures && !(d.draft_temperature >= 0.0f && d.draft_temperature <= FLT_MAX))
        return fail(BITLOGIC_ERR_SHAPE, "verify: draft_temperature %g is not in [0, inf)",
                    (double)d.draft_temperature);
    if (n_requests == 0)
        return ok();
    const bool greedy = !d.temperatures && d.temperature == 0.0f;
    if (!logits || !accepted || !token || (!noise && !greedy) ||
        (d.n_drafted > 0 && (!d.drafted || (!d.uniform && !greedy))))
        return fail(BITLOGIC_ERR_NULL, "verify: NULL pointer");
    if (!aligned(logits, logit_bytes(type)) ||
        (d.draft_logits && !aligned(d.draft_logits, logit_bytes(d.draft_type))) ||
        !aligned(d.drafted, 4) || !aligned(d.lengths, 4) || !aligned(d.uniform, 4) ||
        !aligned(d.temperatures, 4) || !aligned(d.draft_temperatures, 4) || !aligned(noise, 4) ||
        !aligned(accepted, 4) || !aligned(token, 4) || !aligned(log_prob, 4))
        return fail(BITLOGIC_ERR_ALIGN, "verify: misaligned buffer");
    const size_t need = bl::verify_workspace_bytes(n_requests, d.n_drafted, n_classes);
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(BITLOGIC_ERR_WORKSPACE, "verify: workspace of %zu bytes, %zu needed",
                    workspace_bytes, need);
    if (need > 0 && !aligned(workspace, 8))
        return fail(BITLOGIC_ERR_ALIGN, "verify: workspace not 8-byte aligned");
    const bl::VerifySide target = {logits, type, row_stride, request_stride, d.temperature,
                                   d.temperatures};
    const bl::VerifySide draft = {d.draft_logits, d.draft_logits ? d.draft_type : type,
                                  d.draft_row_stride, d.draft_request_stride,
                                  d.draft_temperature, d.draft_temperatures};
    return hip_status(bl::launch_verify(target, draft, n_requests, n_classes, d.n_drafted,
                                        d.drafted, d.lengths, d.uniform, noise, noise_stride,
                                        accepted, token, log_prob, workspace,
                                        (hipStream_t)stream),
                      "verify launch");
}

int bitlogic_dropout(const void *x, int32_t type, int64_t n_rows, int32_t n_cols,
                     int64_t row_stride, float p, uint64_t seed, uint64_t offset,
                     const uint64_t *offset_at, void *out, int64_t out_stride, void *stream)
{
    if (int rc = check_rows("dropout", type, n_rows, n_cols, row_stride))
        return rc;
    if (!(p >= 0.0f && p <= 1.0f))
        return fail(BITLOGIC_ERR_SHAPE, "dropout: p %g is not in [0, 1]", (double)p);
    if (out_stride < n_cols || out_stride > kMaxStride)
        return fail(BITLOGIC_ERR_SHAPE, "dropout: need n_cols <= out_stride <= 2^30");
    if (n_rows == 0)
        return ok();
    if (!x || !out)
        return fail(BITLOGIC_ERR_NULL, "dropout: NULL pointer");
    if (!aligned(x, logit_bytes(type)) || !aligned(out, logit_bytes(type)) ||
        !aligned(offset_at, 8))
        return fail(BITLOGIC_ERR_ALIGN, "dropout: misaligned buffer");
    if (overlaps(x, span_bytes(n_rows, n_cols, row_stride, type), out,
                 span_bytes(n_rows, n_cols, out_stride, type)) &&
        !(x == out && (row_stride == out_stride || n_rows == 1)))
        return fail(BITLOGIC_ERR_SHAPE, "dropout: out overlaps x without being x");
    const uint32_t border = (uint32_t)floor((double)p * 65536.0 + 0.5);
    return hip_status(bl::launch_dropout(x, type, n_rows, n_cols, row_stride, border, seed,
                                         offset, offset_at, out, out_stride,
                                         (hipStream_t)stream),
                      "dropout launch");
}

// ---- adapters ----

size_t bitlogic_group_rows_bytes(int64_t n_rows, int32_t n_groups)
{
    if (n_rows < 0 || n_rows > kMaxGroupedRows || n_groups < 1 ||
        n_groups > BITLOGIC_MAX_ADAPTERS)
        return 0;
    return bl::adapt::group_layout(n_rows, n_groups).bytes;
}

int bitlogic_group_rows(const int32_t *ids, int64_t n_rows, int32_t n_groups, void *plan,
                        size_t plan_bytes, void *stream)
{
    if (n_rows < 0 || n_rows > kMaxGroupedRows || n_groups < 1)
        return fail(BITLOGIC_ERR_SHAPE, "group_rows: need 0 <= n_rows <= 2^27, n_groups >= 1");
    if (n_groups > BITLOGIC_MAX_ADAPTERS)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "group_rows: %d groups > %d", n_groups,
                    BITLOGIC_MAX_ADAPTERS);
    if (n_rows == 0)
        return ok();
    if (!ids || !plan)
        return fail(BITLOGIC_ERR_NULL, "group_rows: NULL pointer");
    if (!aligned(ids, 4) || !aligned(plan, 16))
        return fail(BITLOGIC_ERR_ALIGN, "group_rows: ids or plan misaligned");
    if (plan_bytes < bitlogic_group_rows_bytes(n_rows, n_groups))
        return fail(BITLOGIC_ERR_WORKSPACE, "group_rows: plan of %zu bytes, %zu needed",
                    plan_bytes, bitlogic_group_rows_bytes(n_rows, n_groups));
    return hip_status(bl::launch_group_rows(ids, n_rows, n_groups, plan, (hipStream_t)stream),
                      "group_rows launch");
}

int bitlogic_adapters(const void *x, int32_t x_type, int64_t n_rows, int64_t x_stride,
                      const bitlogic_adapter_set *set, const int32_t *ids, const void *plan,
                      const void *base, int32_t base_type, int64_t base_stride,
                      float base_scale, void *out, int64_t out_stride, float *hidden,
                      void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "adapters";
    if (int rc = check_set(who, set, n_rows))
        return rc;
    const bitlogic_adapter_set &s = *set;
    if (int rc = check_beside(who, "x", x_type, s.weight_type))
        return rc;
    if (int rc = check_stride(who, "x_stride", x_stride, 0))
        return rc;
    if (base) {
        if (int rc = check_beside(who, "base", base_type, s.weight_type))
            return rc;
        if (int rc = check_stride(who, "base_stride", base_stride, 0))
            return rc;
    }
    if (out)
        if (int rc = check_stride(who, "out_stride", out_stride, s.n_out))
            return rc;
    if (n_rows == 0)
        return ok();
    if (!x || !s.down || !s.up || (!out && !hidden))
        return fail(BITLOGIC_ERR_NULL, "adapters: NULL input, or both outputs NULL");
    const size_t el = logit_bytes(s.weight_type);
    if (!aligned(x, el) || !aligned(s.down, el) || !aligned(s.up, el) || !aligned(base, el) ||
        !aligned(out, el) || !aligned(hidden, 4) || !aligned(s.scales, 4))
        return fail(BITLOGIC_ERR_ALIGN, "adapters: misaligned buffer");
    if (out) {
        const size_t out_span = span_bytes(n_rows, s.n_out, out_stride, s.weight_type);
        if (overlaps(x, span_bytes(n_rows, s.n_in, x_stride, s.weight_type), out, out_span))
            return fail(BITLOGIC_ERR_SHAPE, "adapters: out overlaps x");
        if (base &&
            overlaps(base, span_bytes(n_rows, s.n_out, base_stride, s.weight_type), out,
                     out_span) &&
            !(base == out && (base_stride == out_stride || n_rows == 1) &&
              base_type == s.weight_type))
            return fail(BITLOGIC_ERR_SHAPE, "adapters: out overlaps base without being base");
    }
    bl::adapt::PassArgs a = {};
    if (int rc = take_rows(who, a, n_rows, s.n_adapters, ids, plan))
        return rc;
    a.x = static_cast<const char *>(x);
    a.x_stride = x_stride * (int64_t)el;
    a.w1 = static_cast<const char *>(s.down);
    a.w2 = static_cast<const char *>(s.up);
    a.w1_step = (int64_t)s.rank * s.n_in * (int64_t)el;
    a.w2_step = (int64_t)s.rank * s.n_out * (int64_t)el;
    a.k = s.n_in;
    a.m = s.n_out;
    a.rank = s.rank;
    a.scales = s.scales;
    a.scale = s.scale;
    a.base = static_cast<const char *>(base);
    a.base_stride = base_stride * (int64_t)el;
    a.base_i32 = base_type == BITLOGIC_LOGITS_I32;
    a.base_scale = base_scale;
    a.out = static_cast<char *>(out);
    a.out_stride = out_stride * (int64_t)el;
    a.hidden = hidden;
    if (int rc = take_parts(who, a, s.weight_type, false, workspace, workspace_bytes))
        return rc;
    // (out beside x and base: above; a wide pass writes hidden before it reads base)
    const size_t rows = n_rows;
    if (int rc = check_apart(
            who, {{"hidden", hidden, n_rows, s.rank * 4ul, s.rank * 4ul}},
            {{"x", x, n_rows, s.n_in * el, x_stride * el},
             {"base", out ? base : nullptr, n_rows, s.n_out * el, base_stride * el},
             {"out", out, n_rows, s.n_out * el, out_stride * el},
             flat("down", s.down, a.w1_step * s.n_adapters),
             flat("up", out ? s.up : nullptr, a.w2_step * s.n_adapters),
             flat("ids", plan ? nullptr : ids, rows * 4),
             flat("plan", plan, bitlogic_group_rows_bytes(n_rows, s.n_adapters)),
             flat("scales", s.scales, s.n_adapters * 4ul)}))
        return rc;
    return hip_status(by_weight(s.weight_type, [&](auto W) {
        return bl::adapt::launch_pass<decltype(W)::value>(a, x_type == BITLOGIC_LOGITS_I32, false,
                                                          (hipStream_t)stream);
    }), "adapters launch");
}

size_t bitlogic_adapters_workspace_bytes(const bitlogic_adapter_set *set, int64_t n_rows,
                                         int32_t planned)
{
    if (check_set("adapters", set, n_rows) != BITLOGIC_OK || (!planned && n_rows > kMaxLoneRows))
        return 0;
    return layout_of(set->weight_type, n_rows, set->n_adapters, set->rank, set->n_in, set->n_out,
                     planned != 0, false).bytes;
}

size_t bitlogic_adapters_backward_workspace_bytes(const bitlogic_adapter_set *set,
                                                  int64_t n_rows)
{
    if (check_set("adapters_backward", set, n_rows) != BITLOGIC_OK)
        return 0;
    return backward_layout(*set, n_rows).bytes;
}

int bitlogic_adapters_backward(const void *grad, int64_t n_rows, int64_t grad_stride,
                               const void *x, int32_t x_type, int64_t x_stride,
                               const float *hidden, const bitlogic_adapter_set *set,
                               const int32_t *ids, const void *plan, void *grad_x,
                               int64_t grad_x_stride, void *grad_down, void *grad_up,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "adapters_backward";
    if (int rc = check_set(who, set, n_rows))
        return rc;
    const bitlogic_adapter_set &s = *set;
    if (int rc = check_beside(who, "x", x_type, s.weight_type))
        return rc;
    if (int rc = check_stride(who, "grad_stride", grad_stride, 0))
        return rc;
    if (int rc = check_stride(who, "x_stride", x_stride, 0))
        return rc;
    if (grad_x)
        if (int rc = check_stride(who, "grad_x_stride", grad_x_stride, s.n_in))
            return rc;
    const size_t el = logit_bytes(s.weight_type);
    const bool weights = grad_down || grad_up;
    if (!aligned(grad, el) || !aligned(x, el) || !aligned(hidden, 4) || !aligned(s.down, el) ||
        !aligned(s.up, el) || !aligned(s.scales, 4) || !aligned(grad_x, el) ||
        !aligned(grad_down, el) || !aligned(grad_up, el))
        return fail(BITLOGIC_ERR_ALIGN, "adapters_backward: misaligned buffer");
    if (!grad_x && !weights)
        return fail(BITLOGIC_ERR_NULL, "adapters_backward: all outputs NULL");
    bl::adapt::PassArgs a = {};
    if (n_rows > 0) {
        if (!grad || !s.up || (grad_x && !s.down) || (grad_down && !x) || (grad_up && !hidden))
            return fail(BITLOGIC_ERR_NULL, "adapters_backward: NULL input");
        if (weights && !plan)
            return fail(BITLOGIC_ERR_NULL, "adapters_backward: weights' gradients need a plan");
        if (int rc = take_rows(who, a, n_rows, s.n_adapters, ids, plan))
            return rc;
        const size_t need = bitlogic_adapters_backward_workspace_bytes(set, n_rows);
        if (!workspace || workspace_bytes < need)
            return fail(BITLOGIC_ERR_WORKSPACE, "adapters_backward: workspace of %zu bytes, %zu "
                        "needed", workspace_bytes, need);
        if (!aligned(workspace, 16))
            return fail(BITLOGIC_ERR_ALIGN, "adapters_backward: workspace not 16-byte aligned");
    }
    const auto l = bl::adapt::group_layout(n_rows, s.n_adapters);
    const BackwardLayout b = backward_layout(s, n_rows);
    char *ws = static_cast<char *>(workspace);
    float *back = reinterpret_cast<float *>(ws + b.back);
    bl::adapt::GradArgs g = {};
    const int32_t block = by_weight(s.weight_type, [](auto W) {
        return bl::adapt::grad_block<decltype(W)::value>();
    });
    if (weights) {
        const char *p = static_cast<const char *>(plan);
        g.rank = s.rank;
        g.groups = s.n_adapters;
        g.scales = s.scales;
        g.scale = s.scale;
        g.job[0].cols = s.n_in;
        g.job[1].cols = s.n_out;
        g.job[0].out = static_cast<char *>(grad_down);
        g.job[1].out = static_cast<char *>(grad_up);
        g.job[1].transposed = 1;
        if (n_rows > 0) {
            const auto &cut = l.cut[b.cut];
            g.chunks = reinterpret_cast<const bl::adapt::Piece4 *>(p + cut.chunks);
            g.order = reinterpret_cast<const int32_t *>(p + l.order);
            g.chunk_starts = reinterpret_cast<const int32_t *>(p + cut.starts);
            g.slot_starts = reinterpret_cast<const int32_t *>(p + cut.slots);
            g.n_chunks = cut.n;
            g.job[0].y = static_cast<const char *>(x);
            g.job[0].y_stride = x_stride * (int64_t)el;
            g.job[0].y_i32 = x_type == BITLOGIC_LOGITS_I32;
            g.job[0].blocks = grad_down ? (s.n_in + block - 1) / block : 0;
            g.job[0].h = back;
            g.job[0].partial = reinterpret_cast<float *>(ws + b.partial_down);
            g.job[1].y = static_cast<const char *>(grad);
            g.job[1].y_stride = grad_stride * (int64_t)el;
            g.job[1].blocks = grad_up ? (s.n_out + block - 1) / block : 0;
            g.job[1].h = hidden;
            g.job[1].partial = reinterpret_cast<float *>(ws + b.partial_up);
        }
        if (g.n_chunks * ((int64_t)g.job[0].blocks + g.job[1].blocks) >= 1 << 24)
            return fail(BITLOGIC_ERR_UNSUPPORTED, "adapters_backward: n_rows * (n_in + n_out) too "
                        "large for one launch");
    }
    if (n_rows > 0) {
        const size_t down_bytes = (size_t)s.n_adapters * s.rank * s.n_in * el,
                     up_bytes = (size_t)s.n_adapters * s.rank * s.n_out * el;
        if (int rc = check_apart(
                who,
                {{"grad_x", grad_x, n_rows, s.n_in * el, grad_x_stride * el},
                 flat("grad_down", grad_down, down_bytes), flat("grad_up", grad_up, up_bytes)},
                {{"grad", grad, n_rows, s.n_out * el, grad_stride * el},
                 {"x", grad_down ? x : nullptr, n_rows, s.n_in * el, x_stride * el},
                 flat("hidden", grad_up ? hidden : nullptr, (size_t)n_rows * s.rank * 4),
                 flat("down", grad_x ? s.down : nullptr, down_bytes),
                 flat("up", grad_x || grad_down ? s.up : nullptr, up_bytes),
                 flat("ids", plan ? nullptr : ids, (size_t)n_rows * 4),
                 flat("plan", plan, bitlogic_group_rows_bytes(n_rows, s.n_adapters)),
                 flat("scales", s.scales, s.n_adapters * 4ul)}))
            return rc;
    }
    if (n_rows > 0 && (grad_x || grad_down)) {
        a.x = static_cast<const char *>(grad);
        a.x_stride = grad_stride * (int64_t)el;
        a.w1 = static_cast<const char *>(s.up);
        a.w2 = static_cast<const char *>(s.down);
        a.w1_step = (int64_t)s.rank * s.n_out * (int64_t)el;
        a.w2_step = (int64_t)s.rank * s.n_in * (int64_t)el;
        a.k = s.n_out;
        a.m = s.n_in;
        a.rank = s.rank;
        a.scales = s.scales;
        a.scale = s.scale;
        a.out = static_cast<char *>(grad_x);
        a.out_stride = grad_x_stride * (int64_t)el;
        a.hidden = grad_down ? back : nullptr;
        if (int rc = take_parts(who, a, s.weight_type, true, ws + b.parts, b.parts_bytes))
            return rc;
        const hipError_t err = by_weight(s.weight_type, [&](auto W) {
            return bl::adapt::launch_pass<decltype(W)::value>(a, false, true,
                                                              (hipStream_t)stream);
        });
        if (err != hipSuccess)
            return hip_status(err, "adapters_backward launch");
    }
    if (!weights)
        return ok();
    return hip_status(by_weight(s.weight_type, [&](auto W) {
        return bl::adapt::launch_grads<decltype(W)::value>(g, (hipStream_t)stream);
    }), "adapters_backward launch");
}

int bitlogic_probe_valu(uint32_t *out, int32_t blocks, int32_t iters, uint32_t seed,
                        void *stream)
{
    if (!out)
        return fail(BITLOGIC_ERR_NULL, "probe_valu: NULL output");
    if (blocks < 1 || iters < 0)
        return fail(BITLOGIC_ERR_SHAPE, "probe_valu: need blocks >= 1, iters >= 0");
    if (!aligned(out, 4))
        return fail(BITLOGIC_ERR_ALIGN, "probe_valu: output not 4-byte aligned");
    return hip_status(bl::launch_probe_valu(out, blocks, iters, seed, (hipStream_t)stream),
                      "probe_valu launch");
}

int bitlogic_probe_valu_op(int32_t op, uint32_t *out, int32_t blocks, int32_t iters,
                           uint32_t seed, void *stream)
{
    if (op < BITLOGIC_PROBE_OP_MUX || op > BITLOGIC_PROBE_OP_BFE)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "probe_valu_op: unknown op %d", op);
    if (!out)
        return fail(BITLOGIC_ERR_NULL, "probe_valu_op: NULL output");
    if (blocks < 1 || iters < 1)
        return fail(BITLOGIC_ERR_SHAPE, "probe_valu_op: need blocks >= 1, iters >= 1");
    if (!aligned(out, 4))
        return fail(BITLOGIC_ERR_ALIGN, "probe_valu_op: output not 4-byte aligned");
    return hip_status(bl::launch_probe_valu_op(op, out, blocks, iters, seed, (hipStream_t)stream),
                      "probe_valu_op launch");
}

int bitlogic_probe_gather(const void *rows, int64_t n_rows, int32_t lanes_per_row,
                          int32_t valu_per_pass, int32_t blocks, int32_t passes,
                          int32_t waves_per_simd, uint32_t seed, uint32_t *out, void *sink,
                          void *stream)
{
    if (lanes_per_row != 4 && lanes_per_row != 8)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "probe_gather: lanes_per_row %d not 4 or 8",
                    lanes_per_row);
    if (valu_per_pass != 0 && valu_per_pass != 256 && valu_per_pass != 512 &&
        valu_per_pass != 768)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "probe_gather: valu_per_pass %d not 0, 256, 512 "
                    "or 768", valu_per_pass);
    if (!rows || !out)
        return fail(BITLOGIC_ERR_NULL, "probe_gather: NULL rows or output");
    if (n_rows < 1 || n_rows > 0xFFFFFFFFll || blocks < 1 || passes < 1 || waves_per_simd < 0 ||
        waves_per_simd > 8)
        return fail(BITLOGIC_ERR_SHAPE, "probe_gather: need 1 <= n_rows < 2^32, blocks >= 1, "
                    "passes >= 1, 0 <= waves_per_simd <= 8");
    if ((int64_t)blocks * passes * 64 * 6 > 0xFFFFFFFFll)
        return fail(BITLOGIC_ERR_SHAPE, "probe_gather: blocks * passes too large");
    if (!aligned(rows, 16) || !aligned(out, 4) || (sink && !aligned(sink, 16)))
        return fail(BITLOGIC_ERR_ALIGN, "probe_gather: rows and sink need 16-byte alignment");
    return hip_status(bl::launch_probe_gather(rows, n_rows, lanes_per_row, valu_per_pass, blocks,
                                              passes, waves_per_simd, seed, out, sink,
                                              (hipStream_t)stream),
                      "probe_gather launch");
}

int bitlogic_probe_hbm(int32_t mode, const void *in, void *out, int64_t n_bytes,
                       int32_t unroll, int32_t blocks, void *stream)
{
    if (mode != BITLOGIC_PROBE_HBM_COPY && mode != BITLOGIC_PROBE_HBM_READ &&
        mode != BITLOGIC_PROBE_HBM_WRITE)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "probe_hbm: unknown mode %d", mode);
    if (unroll != 1 && unroll != 2 && unroll != 4 && unroll != 8)
        return fail(BITLOGIC_ERR_UNSUPPORTED, "probe_hbm: unroll %d not 1, 2, 4 or 8", unroll);
    if (n_bytes < 0 || n_bytes % 16 != 0 || blocks < 0)
        return fail(BITLOGIC_ERR_SHAPE, "probe_hbm: n_bytes %lld not a multiple of 16, or "
                    "blocks < 0", (long long)n_bytes);
    const bool reads = mode != BITLOGIC_PROBE_HBM_WRITE;
    if (mode == BITLOGIC_PROBE_HBM_READ) {
        if (!out || (n_bytes > 0 && !in))
            return fail(BITLOGIC_ERR_NULL, "probe_hbm: NULL buffer");
        if ((in && !aligned(in, 16)) || !aligned(out, 16))
            return fail(BITLOGIC_ERR_ALIGN, "probe_hbm: buffers not 16-byte aligned");
        return hip_status(bl::launch_probe_hbm(bl::kHbmRead, in, out, n_bytes, unroll, blocks,
                                               (hipStream_t)stream),
                          "probe_hbm launch");
    }
    if (n_bytes == 0)
        return ok();
    if (!out || (reads && !in))
        return fail(BITLOGIC_ERR_NULL, "probe_hbm: NULL buffer");
    if (!aligned(out, 16) || (reads && !aligned(in, 16)))
        return fail(BITLOGIC_ERR_ALIGN, "probe_hbm: buffers not 16-byte aligned");
    if (reads) {
        const char *a = static_cast<const char *>(in), *b = static_cast<const char *>(out);
        if (a < b + n_bytes && b < a + n_bytes)
            return fail(BITLOGIC_ERR_SHAPE, "probe_hbm: buffers overlap");
    }
    return hip_status(bl::launch_probe_hbm(mode == BITLOGIC_PROBE_HBM_COPY ? bl::kHbmCopy
                                                                            : bl::kHbmWrite,
                                           in, out, n_bytes, unroll, blocks,
                                           (hipStream_t)stream),
                      "probe_hbm launch");
}

}  // extern "C"
