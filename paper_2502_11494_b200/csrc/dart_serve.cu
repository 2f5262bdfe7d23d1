// Host side of the entry points around the reduction: rows of queries and keys on their way to it, the cache of what it keeps,
// and the attention that reads the cache.  Argument checks and launches; nothing here allocates.
#include "../../include/dart.h"

#include <math.h>

#include <atomic>

#include <cuda.h>

#include "dart_attend.cuh"
#include "dart_attend_wide.cuh"
#include "dart_host.cuh"
#include "dart_rows.cuh"

namespace {

bool misaligned(const void *p, unsigned to) { return ((uintptr_t)p & (to - 1)) != 0; }

// Whether two sets of rows share a byte: n rows of `width` bytes, `stride` bytes apart.  Columns of one buffer do not.
bool rows_overlap(const void *a, long long na, long long sa, long long wa, const void *b, long long nb, long long sb, long long wb)
{
    if (!a || !b || na == 0 || nb == 0 || !overlaps(a, (size_t)((na - 1) * sa + wa), b, (size_t)((nb - 1) * sb + wb))) return false;
    if (sa != sb || sa <= 0) return true;
    const long long d = ((long long)((uintptr_t)b - (uintptr_t)a) % sa + sa) % sa;
    return d < wa || sa - d < wb;
}

int check_rope(const dart_rope *r, const int64_t *pos, int64_t pos_stride, int head_dim, int n_rows, bool need_pos)
{
    if (!r || r->rot_dim == 0) return DART_OK;
    if (!r->inv_freq || (need_pos && !pos)) return DART_ERR_NULL;
    if (r->rot_dim < 0 || r->rot_dim % 16 != 0 || r->rot_dim > head_dim || r->n_axes < 0 || r->n_axes > 3) return DART_ERR_BAD_SHAPE;
    if (r->n_axes > 1) {
        if (pos && pos_stride < n_rows) return DART_ERR_BAD_SHAPE;
        long long sum = 0;
        for (int a = 0; a < r->n_axes; ++a) {
            if (r->section[a] < 0) return DART_ERR_BAD_SHAPE;
            sum += r->section[a];
        }
        if (sum != r->rot_dim / 2) return DART_ERR_BAD_SHAPE;
    }
    if (misaligned(r->inv_freq, 4) || misaligned(pos, 8)) return DART_ERR_ALIGN;
    return DART_OK;
}

void set_rope(dart::rows::Params &p, const dart_rope *r, const int64_t *pos, int64_t pos_stride)
{
    p.half = 0;
    if (!r || r->rot_dim == 0) return;
    p.half = r->rot_dim / 2, p.interleaved = r->interleaved != 0;
    p.n_axes = r->n_axes > 1 ? r->n_axes : 1;
    p.sec0 = r->n_axes > 1 ? r->section[0] : p.half;
    p.sec01 = r->n_axes > 2 ? r->section[0] + r->section[1] : p.half; // (two axes: no pair turns by a third)
    p.inv_freq = r->inv_freq, p.pos = pos, p.pos_stride = pos_stride;
}

bool known_type(int dtype) { return dtype == DART_BF16 || dtype == DART_FP16; }
bool head_rows_ok(int heads, int D, long long stride, int n_rows) { return heads >= 0 && (n_rows <= 1 || stride >= (long long)heads * D) && stride % 8 == 0 && stride >= 0; }

// Few rows: one round of heads per block, a row's heads over several blocks.  Many rows: up to eight rows a block, so that a thread has
// several rounds to overlap and the rows' angles serve all heads (43264 rows of 64 heads of 128 at 1965 MHz: eight rounds 230 us, four
// 238, sixteen 230; blocks of 256 threads 242, of 64 229; 18832 rows of 32 heads: 60.1; 60.2, 61.2; 60.7, 60.0.  In long runs, under the power cap: 255 to 260).
template <typename T, bool kPaged>
int launch_rows(dart::rows::Params &p, cudaStream_t st)
{
    using namespace dart::rows;
    const int H = p.side[0].heads + p.side[1].heads;
    const int pairs = (p.D / 8 + 1) / 2, kh = pairs <= 4 ? 4 : pairs <= 8 ? 8 : 16;
    const int groups = kThreads / kh;
    const long long rounds = ((long long)p.n_rows * H + groups - 1) / groups; // of a block
    p.heads_per_block = H, p.rows_per_block = 1;
    if (rounds <= 148 * 8)
        p.heads_per_block = H < groups ? H : groups;
    else
        while (p.rows_per_block < kMaxRows && p.rows_per_block * H < 8 * groups) p.rows_per_block *= 2;
    const dim3 grid((unsigned)((p.n_rows - 1) / p.rows_per_block + 1), (unsigned)((H + p.heads_per_block - 1) / p.heads_per_block));
    if (grid.y > 65535u) return DART_ERR_BAD_SHAPE;
    cudaError_t e = kh == 4    ? launch_next(head_rows_kernel<T, 4, kPaged>, grid, kThreads, 0, st, p)
                    : kh == 8  ? launch_next(head_rows_kernel<T, 8, kPaged>, grid, kThreads, 0, st, p)
                               : launch_next(head_rows_kernel<T, 16, kPaged>, grid, kThreads, 0, st, p);
    const cudaError_t e2 = cudaGetLastError();
    return e == cudaSuccess && e2 == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

int check_cache(const dart_cache *c)
{
    if (!c || !c->k || !c->v) return DART_ERR_NULL;
    if (c->n_pages < 1 || c->n_heads < 1 || c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0 || c->page_size < 1) return DART_ERR_BAD_SHAPE;
    if (!known_type(c->dtype)) return DART_ERR_UNSUPPORTED;
    if (misaligned(c->k, 16) || misaligned(c->v, 16)) return DART_ERR_ALIGN;
    return DART_OK;
}

size_t cache_bytes(const dart_cache *c) { return (size_t)c->n_pages * c->n_heads * c->page_size * c->head_dim * 2; }

// ---- attention ---------------------------------------------------------------------------------------------------------------

// Warps that join a (row, head) pair, by how many pairs there are: sixteen, four, one; beyond kJoinMany a warp joins several
constexpr int kJoinOne = 256, kJoinFew = 4096, kJoinMany = 16384;

enum Form { NARROW, WIDE, PAIR };

struct Launch {
    bool prefix, own;
    Form form;
    int M, n_workers, max_items, n_seg;
    size_t item_base, items, open, ml, o; // places in the workspace
};
struct Layout {
    Launch launch[2];
    int n;
    size_t whole_o[2], whole_ml[2], status, bytes;
};

// Rows of a tile by how many rows a segment has on average (the host knows the sizes, not the lengths).  64 sequences of 300 to 600 tokens,
// 8 KV heads, in us: 8 rows each narrow 40, wide 51; 16 rows 35, 47; 32 rows 47, 49; 64 rows 74, 52; 128 rows wide 58, pairs 64; 192 rows 81, 74.
// A wide tile holds whole tokens, so that a copy can fetch its queries.
Form form_of(long long rows, long long segments, long long R)
{
    const long long avg = (rows + segments - 1) / segments, wide = dart::attend::kWideRows / R * R;
    return avg <= dart::attend::kNarrowM || wide == 0 ? NARROW : avg <= wide ? WIDE : PAIR;
}

int sm_count_of(int device)
{
    static std::atomic<int> known[64]; // zero: not asked yet
    if (device >= 0 && device < 64 && known[device].load(std::memory_order_relaxed)) return known[device].load(std::memory_order_relaxed);
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 148;
    }
    if (device >= 0 && device < 64) known[device].store(n, std::memory_order_relaxed);
    return n;
}

// The launches of a call and their places in the workspace: from the sizes alone, lengths are only known on the device.
Layout attend_layout(const dart_cache *c, const dart_attend_args *a, int sms)
{
    using namespace dart::attend;
    Layout L = {};
    const long long R = a->n_q_heads / c->n_heads;
    Form own = form_of(a->n_rows * R, a->n_seq, R);
    const Form shared = a->n_groups > 0 ? form_of(a->n_rows * R, a->n_groups, R) : own;
    // Few sequences go along with their prefixes: one launch instead of two (a prefix of 18432 tokens, 28 query heads, 4 KV heads: 16 sequences 43.0
    // -> 32.1 us, 32 sequences 44.2 -> 35.9; more sequences than workers are left to a
    // launch of their own, though this prefix, in tiles of 256 rows, would take 48 along in 48.1 instead of 51.5 us, 64 in 52.7 instead of 56.0).
    if (own == NARROW && shared != NARROW && (long long)a->n_seq * c->n_heads <= (shared == WIDE ? 2 : 1) * sms) own = shared;
    L.n = own == shared ? 1 : 2;
    L.launch[0].prefix = a->n_groups > 0, L.launch[0].own = own == shared, L.launch[0].form = shared;
    L.launch[1].own = true, L.launch[1].form = own;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    for (int i = 0; i < L.n; ++i) {
        Launch &l = L.launch[i];
        const int wide = (int)(kWideRows / R * R);
        l.M = l.form == NARROW ? kNarrowM : l.form == WIDE ? wide : 2 * wide;
        l.n_workers = sms * (l.form == NARROW ? kNarrowWarps : l.form == WIDE ? 2 : 1);
        l.n_seg = (l.prefix ? a->n_groups : 0) + (l.own ? a->n_seq : 0);
        const long long more = a->n_rows * R / l.M; // a segment of n rows has at most 1 + n / M tiles
        const long long items = c->n_heads * (l.n_seg + more * ((l.prefix ? 1 : 0) + (l.own ? 1 : 0)));
        l.max_items = items < 2147483647ll ? (int)items : 2147483647;
        l.item_base = take(sizeof(int) * ((size_t)l.n_seg + 1));
        l.items = take(sizeof(int2) * (size_t)l.max_items);
        l.open = take(sizeof(Open) * l.n_workers);
        l.ml = take(sizeof(float2) * 2 * l.n_workers * l.M);
        l.o = take(sizeof(float) * 2 * l.n_workers * (size_t)l.M * c->head_dim);
    }
    for (int k = 0; k < 2 && a->n_groups > 0; ++k) {
        L.whole_ml[k] = take(sizeof(float2) * (size_t)a->n_rows * a->n_q_heads);
        L.whole_o[k] = take(sizeof(float) * (size_t)a->n_rows * a->n_q_heads * c->head_dim);
    }
    L.status = take(16); // for callers without a status of their own
    L.bytes = at;
    return L;
}

int check_attend(const dart_cache *c, const dart_attend_args *a)
{
    int rc = check_cache(c);
    if (rc != DART_OK) return rc;
    if (!a) return DART_ERR_NULL;
    if (c->head_dim != 64 && c->head_dim != 128) return DART_ERR_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return DART_ERR_UNSUPPORTED;
    if (a->n_rows < 0 || a->n_seq < 1 || a->n_groups < 0 || a->n_q_heads < 1 || a->n_q_heads % c->n_heads != 0 || a->table_stride < 1 ||
        !(a->scale > 0.0f) || isinf(a->scale) || (!a->cu_q && a->n_rows != a->n_seq) || (a->n_groups > 0 && a->prefix_stride < 1) || a->wait_limit < 0)
        return DART_ERR_BAD_SHAPE;
    // row and token numbers, and a table row's tokens, are counted in 32 bits
    if ((long long)a->n_rows * a->n_q_heads > 2147483647ll / 2 || (long long)c->n_pages * c->n_heads * c->page_size > 2147483647ll - 1024 ||
        (long long)a->table_stride * c->page_size > 2147483647ll / 2 || (long long)a->prefix_stride * c->page_size > 2147483647ll / 2 ||
        ((long long)a->n_seq + a->n_groups) * c->n_heads > 2147483647ll / 4)
        return DART_ERR_BAD_SHAPE;
    if (a->n_rows == 0) return DART_OK;
    if (!a->q || !a->out || !a->table || !a->kv_len || (a->n_groups > 0 && (!a->cu_group || !a->prefix_table || !a->prefix_len))) return DART_ERR_NULL;
    if (!head_rows_ok(a->n_q_heads, c->head_dim, a->q_stride, a->n_rows) || !head_rows_ok(a->n_q_heads, c->head_dim, a->out_stride, a->n_rows))
        return DART_ERR_BAD_SHAPE;
    if (misaligned(a->q, 16) || misaligned(a->out, 16) || misaligned(a->lse, 4) || misaligned(a->cu_q, 4) || misaligned(a->table, 4) ||
        misaligned(a->kv_len, 4) || misaligned(a->cu_group, 4) || misaligned(a->prefix_table, 4) || misaligned(a->prefix_len, 4) || misaligned(a->status, 4))
        return DART_ERR_ALIGN;
    const size_t all = cache_bytes(c), row = 2 * (size_t)a->n_q_heads * c->head_dim;
    const size_t ob = (size_t)(a->n_rows - 1) * 2 * a->out_stride + row, lb = sizeof(float) * (size_t)a->n_rows * a->n_q_heads;
    if (overlaps(a->out, ob, c->k, all) || overlaps(a->out, ob, c->v, all) || overlaps(a->lse, lb, c->k, all) || overlaps(a->lse, lb, c->v, all) ||
        rows_overlap(a->out, a->n_rows, 2 * a->out_stride, row, a->q, a->n_rows, 2 * a->q_stride, row) || overlaps(a->lse, lb, a->out, ob) ||
        overlaps(a->lse, lb, a->q, (size_t)(a->n_rows - 1) * 2 * a->q_stride + row))
        return DART_ERR_ALIAS;
    return DART_OK;
}

dart::attend::Divisor divisor(int d)
{
    uint32_t s = 0;
    while ((1ull << s) < (unsigned)d) ++s;
    return {(uint32_t)(((1ull << (32 + s)) + d - 1) / (unsigned)d - (1ull << 32)), s};
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder()
{
    static const EncodeFn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
        return (EncodeFn)f;
    }();
    return fn;
}

// A cache as the rows of all its pages and heads; a box is a page (or 128 tokens of it) by 64 columns, swizzled.
bool encode_cache(CUtensorMap *tm, const dart_cache *c, void *base)
{
    const EncodeFn fn = encoder();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->n_pages * c->n_heads * c->page_size}, strides[1] = {(cuuint64_t)c->head_dim * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)(c->page_size < dart::attend::kWideTile ? c->page_size : dart::attend::kWideTile)}, one[2] = {1, 1};
    return fn(tm, c->dtype == DART_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dims, strides, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The queries as [rows][KV heads][query heads of each][columns]; a box is the tokens of a tile, one KV head, 64 columns, swizzled.
bool encode_queries(CUtensorMap *tm, const dart_cache *c, const dart_attend_args *a)
{
    const EncodeFn fn = encoder();
    if (!fn) return false;
    const cuuint64_t R = (cuuint64_t)(a->n_q_heads / c->n_heads), D = (cuuint64_t)c->head_dim;
    const cuuint64_t row = a->n_rows > 1 ? (cuuint64_t)a->q_stride : R * D * c->n_heads;
    const cuuint64_t dims[4] = {D, R, (cuuint64_t)c->n_heads, (cuuint64_t)a->n_rows}, strides[3] = {D * 2, R * D * 2, row * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)R, 1, (cuuint32_t)(dart::attend::kWideRows / R)}, one[4] = {1, 1, 1, 1};
    return fn(tm, c->dtype == DART_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void *>(a->q), dims, strides, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename K>
cudaError_t with_smem(K kernel, size_t smem)
{
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}

template <typename T, int D>
int launch_attend(const dart_cache *c, const dart_attend_args *a, char *ws, const Layout &L, int sms, cudaStream_t st)
{
    using namespace dart::attend;
    Params p = {};
    p.q = (const char *)a->q, p.out = (char *)a->out, p.lse = a->lse, p.q_stride = 2 * a->q_stride, p.out_stride = 2 * a->out_stride;
    p.k = (const char *)c->k, p.v = (const char *)c->v;
    p.n_rows = a->n_rows, p.Hq = a->n_q_heads, p.Hk = c->n_heads, p.R = a->n_q_heads / c->n_heads, p.n_seq = a->n_seq, p.n_groups = a->n_groups;
    p.n_pages = c->n_pages, p.by_R = divisor(p.R), p.by_Hk = divisor(p.Hk);
    while ((1 << p.page_shift) < c->page_size) ++p.page_shift;
    p.table_stride = a->table_stride, p.ptable_stride = a->prefix_stride;
    p.cu_q = a->cu_q, p.table = a->table, p.kv_len = a->kv_len, p.cu_group = a->cu_group, p.ptable = a->prefix_table, p.plen = a->prefix_len;
    p.scale_log2 = a->scale * 1.44269504088896340736f, p.status = a->status;
    for (int k = 0; k < 2; ++k) p.whole[k] = Whole{(float *)(ws + L.whole_o[k]), (float2 *)(ws + L.whole_ml[k])};
    JoinParams j = {};
    CUtensorMap tm_q, tm_k, tm_v;
    bool maps = false;
    for (int i = 0; i < L.n; ++i) {
        const Launch &l = L.launch[i];
        p.n_prefix = l.prefix ? a->n_groups : 0, p.n_own = l.own ? a->n_seq : 0;
        p.n_workers = l.n_workers, p.least = l.form == NARROW ? kNarrowLeast : 1, p.max_items = l.max_items;
        p.pieces = Pieces{(int *)(ws + l.item_base), (int2 *)(ws + l.items), (float *)(ws + l.o), (float2 *)(ws + l.ml), (Open *)(ws + l.open), l.M, l.n_workers, divisor(l.M)};
        for (int k = 0; k < 2; ++k)
            if (k ? l.own : l.prefix) j.from[k] = p.pieces, j.seg_off[k] = k ? p.n_prefix : 0, j.n_seg[k] = l.n_seg;
        cudaError_t e;
        if (l.form == NARROW) {
            const size_t smem = kNarrowRing * kNarrowWarps;
            e = with_smem(attend_narrow_kernel<T, D>, smem);
            if (e == cudaSuccess) e = launch_next(attend_narrow_kernel<T, D>, dim3(sms), kNarrowWarps * 32, smem, st, p);
        } else {
            if (!maps && (!encode_queries(&tm_q, c, a) || !encode_cache(&tm_k, c, c->k) || !encode_cache(&tm_v, c, c->v))) return DART_ERR_CUDA;
            maps = true;
            const auto kernel = l.form == PAIR ? attend_wide_kernel<T, D, true> : attend_wide_kernel<T, D, false>;
            const unsigned long long limit = (a->wait_limit > 0 ? (unsigned long long)a->wait_limit : 2000000ull) * 2100ull;
            e = with_smem(kernel, kWideSmem);
            if (e == cudaSuccess)
                e = launch_next(kernel, dim3(sms), kWideThreads, kWideSmem, st, tm_q, tm_k, tm_v, p, a->status ? (int *)a->status : (int *)(ws + L.status), limit,
                                a->test_withhold);
        }
        if (e != cudaSuccess) {
            cudaGetLastError();
            return DART_ERR_CUDA;
        }
    }
    j.p = p;
    const long long pairs = (long long)a->n_rows * a->n_q_heads;
    const int heads = pairs <= kJoinMany ? 1 : 4;
    const long long warps = a->n_rows * ((a->n_q_heads + heads - 1ll) / heads);
    const cudaError_t e = pairs <= kJoinOne    ? launch_next(attend_join_rows_kernel<T, D, 16>, dim3((unsigned)pairs), 512, 0, st, j, 1)
                          : pairs <= kJoinFew  ? launch_next(attend_join_rows_kernel<T, D, 4>, dim3((unsigned)pairs), 128, 0, st, j, 1)
                          : a->n_groups > 0 ? launch_next(attend_join_rows_kernel<T, D, 1>, dim3((unsigned)((warps + 3) / 4)), 128, 0, st, j, heads)
                                            : launch_next(attend_join_cut_kernel<T, D>, dim3((unsigned)j.from[1].n_workers, (unsigned)((j.from[1].M + kCutRows - 1) / kCutRows)), 256, 0, st, p, j.from[1]);
    const cudaError_t e2 = cudaGetLastError();
    return e == cudaSuccess && e2 == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

} // namespace

extern "C" {

int dart_norm_rope(const void *q, int64_t q_stride, int n_q_heads, const void *k, int64_t k_stride, int n_k_heads, int n_rows,
                   int head_dim, int dtype, const void *q_weight, const void *k_weight, float eps, const dart_rope *rope,
                   const int64_t *pos, int64_t pos_stride, void *q_out, int64_t qo_stride, void *k_out, int64_t ko_stride, int device, void *stream)
{
    if (n_rows < 0 || n_q_heads < 0 || n_k_heads < 0 || n_q_heads + (long long)n_k_heads < 1 || n_q_heads + (long long)n_k_heads > 65536 ||
        head_dim < 8 || head_dim > 256 || head_dim % 8 != 0 || !(eps >= 0.0f) || isinf(eps))
        return DART_ERR_BAD_SHAPE;
    if (!known_type(dtype)) return DART_ERR_UNSUPPORTED;
    if (n_rows == 0) return DART_OK;
    if ((n_q_heads && (!q || !q_out)) || (n_k_heads && (!k || !k_out))) return DART_ERR_NULL;
    if (!head_rows_ok(n_q_heads, head_dim, q_stride, n_rows) || !head_rows_ok(n_q_heads, head_dim, qo_stride, n_rows) ||
        !head_rows_ok(n_k_heads, head_dim, k_stride, n_rows) || !head_rows_ok(n_k_heads, head_dim, ko_stride, n_rows))
        return DART_ERR_BAD_SHAPE;
    int rc = check_rope(rope, pos, pos_stride, head_dim, n_rows, true);
    if (rc != DART_OK) return rc;
    if (!n_q_heads) q = q_out = nullptr, q_weight = nullptr;
    if (!n_k_heads) k = k_out = nullptr, k_weight = nullptr;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(q_out, 16) || misaligned(k_out, 16) || misaligned(q_weight, 16) || misaligned(k_weight, 16))
        return DART_ERR_ALIGN;
    const long long wq = 2ll * n_q_heads * head_dim, wk = 2ll * n_k_heads * head_dim;
    const bool q_in_place = q_out == q && qo_stride == q_stride, k_in_place = k_out == k && ko_stride == k_stride;
    if ((!q_in_place && rows_overlap(q_out, n_rows, 2 * qo_stride, wq, q, n_rows, 2 * q_stride, wq)) ||
        (!k_in_place && rows_overlap(k_out, n_rows, 2 * ko_stride, wk, k, n_rows, 2 * k_stride, wk)) ||
        rows_overlap(q_out, n_rows, 2 * qo_stride, wq, k, n_rows, 2 * k_stride, wk) ||
        rows_overlap(k_out, n_rows, 2 * ko_stride, wk, q, n_rows, 2 * q_stride, wq) ||
        rows_overlap(q_out, n_rows, 2 * qo_stride, wq, k_out, n_rows, 2 * ko_stride, wk))
        return DART_ERR_ALIAS;
    DeviceGuard g(device);
    if (!g.ok) return DART_ERR_CUDA;
    dart::rows::Params p = {};
    p.side[0] = {(const char *)q, (char *)q_out, (const char *)q_weight, 2 * q_stride, 2 * qo_stride, n_q_heads, true};
    p.side[1] = {(const char *)k, (char *)k_out, (const char *)k_weight, 2 * k_stride, 2 * ko_stride, n_k_heads, true};
    p.n_rows = n_rows, p.D = head_dim, p.eps = eps;
    set_rope(p, rope, pos, pos_stride);
    return dtype == DART_BF16 ? launch_rows<__nv_bfloat16, false>(p, (cudaStream_t)stream) : launch_rows<__half, false>(p, (cudaStream_t)stream);
}

int dart_cache_append(const dart_cache *cache, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int n_seq,
                      int n_rows, const int32_t *cu_rows, const int32_t *idx, int S, const int32_t *table, int table_stride,
                      const int32_t *start, const void *k_weight, float eps, const dart_rope *rope, const int64_t *pos, int64_t pos_stride,
                      int32_t *status, void *stream)
{
    int rc = check_cache(cache);
    if (rc != DART_OK) return rc;
    if (n_rows < 0 || n_seq < 1 || table_stride < 1 || (idx && S < 1) || (!cu_rows && n_rows % n_seq != 0) || !(eps >= 0.0f) || isinf(eps) ||
        cache->n_heads > 32768)
        return DART_ERR_BAD_SHAPE;
    if (n_rows == 0) return DART_OK;
    if (!k || !v || !table) return DART_ERR_NULL;
    const long long n_src = idx ? (long long)n_seq * S : n_rows;
    const int D = cache->head_dim, Hk = cache->n_heads;
    if (!head_rows_ok(Hk, D, k_stride, n_src > 1 ? 2 : 1) || !head_rows_ok(Hk, D, v_stride, n_src > 1 ? 2 : 1)) return DART_ERR_BAD_SHAPE;
    rc = check_rope(rope, pos, pos_stride, D, n_rows, false);
    if (rc != DART_OK) return rc;
    if (rope && rope->rot_dim && !pos && rope->n_axes > 1) return DART_ERR_NULL; // a slot is a position on one axis only
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_weight, 16) || misaligned(cu_rows, 4) || misaligned(idx, 4) || misaligned(table, 4) ||
        misaligned(start, 4) || misaligned(status, 4))
        return DART_ERR_ALIGN;
    const size_t all = cache_bytes(cache), row = 2 * (size_t)Hk * D;
    const size_t kb = (size_t)(n_src - 1) * 2 * k_stride + row, vb = (size_t)(n_src - 1) * 2 * v_stride + row;
    if (overlaps(cache->k, all, cache->v, all) || overlaps(cache->k, all, k, kb) || overlaps(cache->k, all, v, vb) || overlaps(cache->v, all, k, kb) ||
        overlaps(cache->v, all, v, vb))
        return DART_ERR_ALIAS;
    DeviceGuard g(cache->device);
    if (!g.ok) return DART_ERR_CUDA;
    dart::rows::Params p = {};
    p.side[0] = {(const char *)k, (char *)cache->k, (const char *)k_weight, 2 * k_stride, 0, Hk, true};
    p.side[1] = {(const char *)v, (char *)cache->v, nullptr, 2 * v_stride, 0, Hk, false};
    p.n_rows = n_rows, p.D = D, p.eps = eps;
    set_rope(p, rope, pos, pos_stride);
    p.n_seq = n_seq, p.per_seq = cu_rows ? 0 : n_rows / n_seq, p.S = S, p.table_stride = table_stride, p.page_size = cache->page_size;
    p.n_pages = cache->n_pages, p.cu = cu_rows, p.idx = idx, p.table = table, p.start = start, p.status = status;
    return cache->dtype == DART_BF16 ? launch_rows<__nv_bfloat16, true>(p, (cudaStream_t)stream) : launch_rows<__half, true>(p, (cudaStream_t)stream);
}

size_t dart_attend_workspace(const dart_cache *cache, const dart_attend_args *args)
{
    if (check_attend(cache, args) != DART_OK || args->n_rows == 0) return 0;
    return attend_layout(cache, args, sm_count_of(cache->device)).bytes;
}

int dart_attend(const dart_cache *cache, const dart_attend_args *args, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_attend(cache, args);
    if (rc != DART_OK) return rc;
    if (args->n_rows == 0) return DART_OK;
    if (!workspace) return DART_ERR_NULL;
    if (misaligned(workspace, 256)) return DART_ERR_ALIGN;
    const int sms = sm_count_of(cache->device);
    const Layout L = attend_layout(cache, args, sms);
    if (workspace_bytes < L.bytes) return DART_ERR_NOMEM;
    DeviceGuard g(cache->device);
    if (!g.ok) return DART_ERR_CUDA;
    char *ws = (char *)workspace;
    cudaStream_t st = (cudaStream_t)stream;
    if (cache->dtype == DART_BF16)
        return cache->head_dim == 128 ? launch_attend<__nv_bfloat16, 128>(cache, args, ws, L, sms, st) : launch_attend<__nv_bfloat16, 64>(cache, args, ws, L, sms, st);
    return cache->head_dim == 128 ? launch_attend<__half, 128>(cache, args, ws, L, sms, st) : launch_attend<__half, 64>(cache, args, ws, L, sms, st);
}

} // extern "C"
