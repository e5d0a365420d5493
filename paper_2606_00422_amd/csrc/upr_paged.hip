// Host side of the paged-cache operators: argument checks, frequency tables,
// and the launches of upr_rope_*, upr_paged_append and upr_paged_attention.
#include <algorithm>
#include <cmath>

#include "upr_paged_host.h"
#include "upr_profile.h"

namespace upr {

namespace {

constexpr int32_t kMaxRows = 1 << 30;
// (a launch has fewer than 2^32 threads: one user's work items have to fit)
constexpr int32_t kMaxCount = 1 << 22;
constexpr int64_t kMaxCountHeads = int64_t{1} << 27;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int elem(int dtype) { return dtype == UPR_F32 ? 4 : 2; }

upr_status check_dtype(int32_t dtype) {
    if (dtype != UPR_F32 && dtype != UPR_BF16)
        return report_error(UPR_ERR_DTYPE, "dtype %d is not UPR_F32 or UPR_BF16", dtype);
    return UPR_OK;
}

upr_status check_head_dim(int32_t D) {
    if (D != 32 && D != 64 && D != 128)
        return report_error(UPR_ERR_CONFIG, "head_dim %d not supported (32, 64 or 128)", D);
    return UPR_OK;
}

upr_status check_shape(const upr_attn_shape* sh) {
    if (!sh) return report_error(UPR_ERR_NULL, "shape is NULL");
    upr_status st = check_dtype(sh->dtype);
    if (st == UPR_OK) st = check_head_dim(sh->head_dim);
    if (st != UPR_OK) return st;
    if (sh->n_kv_heads < 1 || sh->n_heads < sh->n_kv_heads || sh->n_heads > 1024 ||
        sh->n_heads % sh->n_kv_heads != 0)
        return report_error(UPR_ERR_CONFIG, "%d heads over %d key/value heads: need 1 <= n_kv_heads <= n_heads <= "
                            "1024, n_heads a multiple of n_kv_heads", sh->n_heads, sh->n_kv_heads);
    return UPR_OK;
}

// One tensor of rows of `heads` heads (name for the message).
upr_status check_rows(const char* name, const void* p, int64_t ld, int heads, int D, int dtype) {
    if (!p) return report_error(UPR_ERR_NULL, "%s is NULL", name);
    if (!aligned16(p)) return report_error(UPR_ERR_LIMIT, "%s is not 16-byte aligned", name);
    if (ld < (int64_t)heads * D || ld > (int64_t{1} << 40) || ld * elem(dtype) % 16 != 0)
        return report_error(UPR_ERR_LIMIT, "leading dimension %lld of %s: need at least %d elements, a multiple of "
                            "16 bytes", (long long)ld, name, heads * D);
    return UPR_OK;
}

upr_status check_rope(const upr_rope* r, int head_dim) {
    if (r->rot_dim < 2 || r->rot_dim % 2 != 0 || r->rot_dim > 2 * UPR_ROPE_MAX_PAIRS || r->rot_dim > head_dim)
        return report_error(UPR_ERR_LIMIT, "rot_dim %d must be even, in [2, %d]", r->rot_dim, head_dim);
    if (r->layout != UPR_ROPE_HALF && r->layout != UPR_ROPE_INTERLEAVED)
        return report_error(UPR_ERR_LIMIT, "rope layout %d is not a upr_rope_layout value", r->layout);
    if (!std::isfinite(r->magnitude) || !std::isfinite((float)r->magnitude))
        return report_error(UPR_ERR_LIMIT, "rope magnitude is not a finite float");
    for (int i = 0; i < r->rot_dim / 2; ++i)
        if (!std::isfinite(r->freq[i]) || std::fabs(r->freq[i]) > 1e6)
            return report_error(UPR_ERR_LIMIT, "rope frequency %d is not finite or beyond 1e6", i);
    return UPR_OK;
}

}  // namespace

upr_status check_page_rows(int32_t page_rows) {
    if (page_rows < 16 || page_rows > 1024 || (page_rows & (page_rows - 1)) != 0)
        return report_error(UPR_ERR_LIMIT, "page_rows %d must be a power of two in [16, 1024]", page_rows);
    return UPR_OK;
}

upr_status check_paged_users(const upr_segments* seg, const char* name, const int32_t* rows_host, int32_t page_rows,
                             int32_t table_stride, int n_heads, bool part_of_cache, int64_t* total) {
    if (!seg) return report_error(UPR_ERR_NULL, "%s segments pointer is NULL", name);
    if (seg->num_users < 0) return report_error(UPR_ERR_OFFSETS, "%s num_users %d < 0", name, seg->num_users);
    if (!seg->offsets_host) return report_error(UPR_ERR_NULL, "%s offsets_host is NULL", name);
    const int32_t* o = seg->offsets_host;
    if (o[0] < 0) return report_error(UPR_ERR_OFFSETS, "%s offsets[0] = %d < 0", name, o[0]);
    if (seg->num_users > 0 && !rows_host) return report_error(UPR_ERR_NULL, "rows_host is NULL");
    for (int u = 0; u < seg->num_users; ++u) {
        if (o[u + 1] < o[u])
            return report_error(UPR_ERR_OFFSETS, "%s offsets decrease at user %d (%d -> %d)", name, u, o[u], o[u + 1]);
        const int32_t n = rows_host[u], c = o[u + 1] - o[u];
        if (n < 0 || (part_of_cache && n < c))
            return report_error(UPR_ERR_OFFSETS, "user %d has %d cached rows, %d of them new", u, n, c);
        if (n > kMaxRows) return report_error(UPR_ERR_LIMIT, "user %d has %d cached rows (at most %d)", u, n, kMaxRows);
        if (c > kMaxCount || (int64_t)c * n_heads > kMaxCountHeads)
            return report_error(UPR_ERR_LIMIT, "user %d has %d rows of %d heads (at most 2^22, and 2^27 with the heads)",
                                u, c, n_heads);
        if (c > 0 && ((int64_t)n + page_rows - 1) / page_rows > table_stride)
            return report_error(UPR_ERR_CAPACITY, "user %d has %d cached rows, its table %d pages of %d", u, n,
                                table_stride, page_rows);
    }
    *total = (int64_t)o[seg->num_users] - o[0];
    return UPR_OK;
}

upr_status check_paged_cache(const upr_paged_cache* c, bool pointers) {
    if (!c) return report_error(UPR_ERR_NULL, "cache is NULL");
    const upr_status st = check_page_rows(c->page_rows);
    if (st != UPR_OK) return st;
    if (c->n_pages < 0 || c->n_pages > 0x7fffffff)
        return report_error(UPR_ERR_LIMIT, "n_pages %lld outside [0, 2^31)", (long long)c->n_pages);
    if (c->table_stride < 0) return report_error(UPR_ERR_LIMIT, "table_stride %d < 0", c->table_stride);
    if (!pointers) return UPR_OK;
    if (c->n_pages > 0 && !c->data) return report_error(UPR_ERR_NULL, "cache data is NULL");
    if (!aligned16(c->data)) return report_error(UPR_ERR_LIMIT, "cache data is not 16-byte aligned");
    if (c->table_stride > 0 && !c->tables) return report_error(UPR_ERR_NULL, "cache tables is NULL");
    return UPR_OK;
}

upr_status check_attn_options(const upr_attn_options* o) {
    if (!o) return report_error(UPR_ERR_NULL, "options is NULL");
    // (in log2 units, and as the argument of the tanh, they have to be fp32 too)
    if (!(o->scale > 0.f) || !(o->scale < 1e30f))
        return report_error(UPR_ERR_LIMIT, "scale must be positive and below 1e30");
    if (!(o->softcap >= 0.f) || !(o->softcap < 1e30f) || (o->softcap > 0.f && !(o->scale / o->softcap < 1e30f)))
        return report_error(UPR_ERR_LIMIT, "softcap must be 0, or positive, below 1e30 and with scale / softcap below 1e30");
    if (o->window < 0) return report_error(UPR_ERR_LIMIT, "window %d < 0", o->window);
    if ((o->k_self == nullptr) != (o->v_self == nullptr))
        return report_error(UPR_ERR_NULL, "k_self and v_self must both be given or both be NULL");
    return UPR_OK;
}

PagedPool paged_pool(const upr_paged_cache& c, size_t plane_bytes, int plane) {
    int shift = 0;
    while ((1 << shift) < c.page_rows) ++shift;
    return PagedPool{static_cast<char*>(c.data) + plane_bytes * plane, c.tables, c.n_pages, c.table_stride,
                     c.page_rows, shift};
}

RopeArgs rope_args(const upr_rope* r) {
    RopeArgs a{};
    if (!r) return a;
    a.rot_dim = r->rot_dim;
    a.layout = r->layout;
    a.magnitude = (float)r->magnitude;
    for (int i = 0; i < r->rot_dim / 2; ++i) a.quarters[i] = r->freq[i] * (2.0 / M_PI);
    return a;
}

upr_status check_model_rope(const upr_rope* r, int head_dim) { return r ? check_rope(r, head_dim) : UPR_OK; }

// Cuts a call's users into launches of at most kPagedUsers and kMaxItems work
// items; `items` gives a user's items.  longest_first: in each launch, users with
// the most cached rows first (their items take longest).
template <typename Items, typename Launch>
static hipError_t each_launch(const upr_segments* seg, const int32_t* rows_host, bool longest_first,
                              const Items& items, const Launch& launch) {
    // (of at most 256 threads; the largest user that the checks let through has
    // 2^27 / 16 items, and for each of up to 1024 key/value heads a part of one)
    constexpr int64_t kMaxItems = (1 << 23) + 1024;
    const int32_t* const o = seg->offsets_host;
    struct Entry {
        int32_t user, items;
    };
    Entry e[kPagedUsers];
    int64_t total = 0;
    int n = 0;
    auto flush = [&]() {
        if (longest_first)
            std::sort(e, e + n, [&](const Entry& x, const Entry& y) {
                const int32_t a = rows_host[x.user], b = rows_host[y.user];
                return a != b ? a > b : x.user < y.user;
            });
        PagedUsers u;
        u.n = n;
        u.item0[0] = 0;
        for (int i = 0; i < n; ++i) {
            const int32_t w = e[i].user;
            u.user[i] = w;
            u.row0[i] = o[w];
            u.count[i] = o[w + 1] - o[w];
            u.rows[i] = rows_host[w];
            u.item0[i + 1] = u.item0[i] + e[i].items;
        }
        n = 0;
        total = 0;
        return launch(u);
    };
    for (int w = 0; w < seg->num_users; ++w) {
        const int32_t c = o[w + 1] - o[w];
        if (c == 0) continue;
        const int64_t m = items(c, rows_host[w]);
        if (n == kPagedUsers || (n > 0 && total + m > kMaxItems)) {
            const hipError_t st = flush();
            if (st != hipSuccess) return st;
        }
        e[n++] = Entry{w, (int32_t)m};
        total += m;
    }
    return n > 0 ? flush() : hipSuccess;
}

hipError_t paged_append(int dtype, const RopeArgs& rope, const AppendArgs& a, const PagedPool& pool,
                        const upr_segments* seg, const int32_t* rows_host, hipStream_t s) {
    const int batch = append_batch(dtype, rope, a, (int64_t)seg->offsets_host[seg->num_users] - seg->offsets_host[0]);
    const int per = append_rows(dtype, rope, a, batch);
    return each_launch(
        seg, rows_host, false, [&](int32_t c, int32_t) { return (int64_t)((c + per - 1) / per); },
        [&](const PagedUsers& u) { return launch_append(dtype, rope, a, batch, pool, u, s); });
}

// ---- the attention's plan

// Keys that a user's rows see between them.
static int64_t attn_keys(const AttnArgs& a, int64_t count, int32_t rows) {
    return rows - attn_first_key(a.k_self.p ? rows : rows - (int32_t)count, a.window);
}

static int64_t attn_user_items(const AttnArgs& a, int32_t count, int32_t rows) {
    const int64_t tiles = ((int64_t)count * (a.n_heads / a.n_kv_heads) + a.tile - 1) / a.tile;
    return tiles * a.n_kv_heads * attn_splits(rows, count, a.k_self.p != nullptr, a.window, a.chunk);
}

// Rows per tile.
//   16: no user has more rows (or fp32, whose matrix instructions take as long
//       per row in any tile).
//   128: the keys of a stage serve most rows; from 192 such items up, if the
//       tiles are at least half full.
//   32: the rest.  Four waves share an item's keys, so that it ends sooner (4.9
//       against 15 ns per key at head_dim 64, 8.0 against 22 at 128) and there
//       are four times as many.
// Measured, us, 128 / 32 rows: 4 users x 100-300 rows over 1000, 32/8 heads of
// 128 (224 items of 128 rows): 37 / 73; 1 x 1000 over 8000, 8 heads of 64 (64
// items): 132 / 47; 48 x 1-96 over 32-4096, window 1024 (384, a third full): 45 /
// 34.
static int attn_tile(int dtype, const AttnArgs& a, const upr_segments* seg) {
    const int32_t* const o = seg->offsets_host;
    const int64_t G = a.n_heads / a.n_kv_heads;
    int64_t most = 0, rows = 0, tiles = 0;
    for (int u = 0; u < seg->num_users; ++u) {
        const int64_t r = (o[u + 1] - o[u]) * G;
        most = std::max(most, r);
        rows += r;
        tiles += (r + 127) / 128;
    }
    if (most <= 16 || dtype == UPR_F32) return 16;
    return tiles * a.n_kv_heads >= 192 && rows >= tiles * 64 ? 128 : 32;
}

// Keys per part, 0 for no parts.  An unsplit call takes about as long as its
// longest item alone (tk per key) or as the device (256 CUs; cached bytes at
// 5.2 TB/s) takes for all of them, whichever is more.  Parts pay where the item
// is the longer by more than the join's launch; a part is then an eighth of the
// device's time.  Long bf16 calls of single rows of 128 values, whose workgroups have
// a CU's LDS to themselves, are cut as well until there are four per CU: nothing
// else covers a workgroup's start there.  Measured, us, unsplit / split:
// single rows, 8 heads of 64: one user over 1024 rows 9.3 / 9.6, 2048 13.3 /
// 9.9, 16384 70 / 17, 16 users over 2048 15 / 23; 32/8 heads of 128: 64 users over
// 512-16384 436 / 398.
static int attn_chunk(int dtype, const AttnArgs& a, const upr_segments* seg, const int32_t* rows_host) {
    const int32_t* const o = seg->offsets_host;
    const int G = a.n_heads / a.n_kv_heads, D = a.D;
    const double tk = 1e-3 * (dtype == UPR_F32 ? 3.0 + 0.142 * D
                              : a.tile == 16   ? 2.6 + 0.027 * D
                              : a.tile == 32   ? 1.8 + 0.048 * D
                                               : 8.0 + 0.11 * D);     // us
    double keys = 0, seen = 0, longest = 0;
    int64_t items = 0;
    for (int u = 0; u < seg->num_users; ++u) {
        const int64_t c = o[u + 1] - o[u];
        if (c == 0) continue;
        const int64_t n = attn_keys(a, c, rows_host[u]), t = (c * G + a.tile - 1) / a.tile * a.n_kv_heads;
        items += t;
        keys += (double)t * n;
        seen += (double)n * a.n_kv_heads;
        longest = std::max(longest, (double)n);
    }
    const double bytes = seen * 2 * D * elem(dtype);
    const double device = std::max({keys * tk / 256, bytes / 5.2e6, 2.0});
    const bool even = dtype == UPR_BF16 && a.tile == 16 && D == 128 && device > 60 && items < 4 * 256;
    if (longest * tk <= device + 4 && !even) return 0;
    double chunk = device / tk / 8;
    if (even) chunk = std::min(chunk, keys / (4 * 256));
    return (int)std::min<int64_t>(std::max<int64_t>(512, ((int64_t)chunk + 255) / 256 * 256), 1 << 30);
}

// Tile, parts and workspace of a call, from its lengths alone.  part_ml holds an
// offset until the workspace is known.
size_t plan_paged_attn(int dtype, AttnArgs* a, const upr_segments* seg, const int32_t* rows_host) {
    const int32_t* const o = seg->offsets_host;
    a->tile = attn_tile(dtype, *a, seg);
    a->chunk = attn_chunk(dtype, *a, seg, rows_host);
    if (a->chunk == 0) return 0;
    // (launches of a call follow one another and use the same records)
    bool any = false;
    int64_t here = 0, most = 0;
    int users = 0;
    for (int u = 0; u < seg->num_users; ++u) {
        const int32_t c = o[u + 1] - o[u];
        if (c == 0) continue;
        if (users == kPagedUsers) users = 0, here = 0;
        here += attn_user_items(*a, c, rows_host[u]);
        ++users;
        any |= attn_splits(rows_host[u], c, a->k_self.p != nullptr, a->window, a->chunk) > 1;
        most = std::max(most, here);
    }
    if (!any) {
        a->chunk = 0;
        return 0;
    }
    const size_t recs = (size_t)most * a->tile, sums = (recs * a->D * 4 + 255) / 256 * 256;
    a->part_ml = reinterpret_cast<float*>(sums);
    return sums + recs * 8;
}

hipError_t paged_attn(int dtype, AttnArgs a, const PagedPool& pool, const upr_segments* seg,
                      const int32_t* rows_host, void* ws, hipStream_t s) {
    const bool join = a.chunk > 0;
    if (join) {
        a.part_o = static_cast<float*>(ws);
        a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + reinterpret_cast<uintptr_t>(a.part_ml));
    }
    const int G = a.n_heads / a.n_kv_heads;
    return each_launch(
        seg, rows_host, true, [&](int32_t c, int32_t n) { return attn_user_items(a, c, n); },
        [&](const PagedUsers& u) {
            const hipError_t e = launch_paged_attn(dtype, a, pool, u, s);
            if (e != hipSuccess || !join) return e;
            JoinUsers j;
            j.users.n = 0;
            j.users.item0[0] = 0;
            for (int i = 0; i < u.n; ++i) {
                if (attn_splits(u.rows[i], u.count[i], a.k_self.p != nullptr, a.window, a.chunk) == 1) continue;
                const int k = j.users.n++;
                j.users.user[k] = u.user[i];
                j.users.row0[k] = u.row0[i];
                j.users.count[k] = u.count[i];
                j.users.rows[k] = u.rows[i];
                j.part0[k] = u.item0[i];
                // (at most the rows of the parts' records: no more than items * tile)
                const int64_t groups = ((int64_t)u.count[i] * G + kJoinRows - 1) / kJoinRows * a.n_kv_heads;
                j.users.item0[k + 1] = j.users.item0[k] + (int32_t)groups;
            }
            return j.users.n > 0 ? launch_paged_join(dtype, a, pool, j, s) : e;
        });
}

}  // namespace upr

using namespace upr;

// What the attention's plan depends on (no pointers but whether rows have
// their own keys).
static AttnArgs attn_args(const upr_attn_shape& sh, const upr_attn_options& o) {
    AttnArgs a{};
    a.n_heads = sh.n_heads;
    a.n_kv_heads = sh.n_kv_heads;
    a.D = sh.head_dim;
    a.k_self = RowsOf{o.k_self, o.self_ld};
    a.v_self = RowsOf{o.v_self, o.self_ld};
    a.c = (float)(o.scale * 1.4426950408889634);
    if (o.softcap > 0.f) {
        a.ct2 = (float)(2 * 1.4426950408889634 * (double)o.scale / o.softcap);
        a.cap2 = (float)(o.softcap * 1.4426950408889634);
    }
    a.slopes = o.slopes;
    a.window = o.window;
    return a;
}

extern "C" {

upr_status upr_rope_init(int32_t rot_dim, int32_t layout, double base, int32_t scaling, double factor,
                         double original_length, upr_rope* out) {
    if (!out) return report_error(UPR_ERR_NULL, "out is NULL");
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 2 * UPR_ROPE_MAX_PAIRS)
        return report_error(UPR_ERR_LIMIT, "rot_dim %d must be even, in [2, %d]", rot_dim, 2 * UPR_ROPE_MAX_PAIRS);
    if (layout != UPR_ROPE_HALF && layout != UPR_ROPE_INTERLEAVED)
        return report_error(UPR_ERR_LIMIT, "rope layout %d is not a upr_rope_layout value", layout);
    if (!(base > 1.0) || !std::isfinite(base)) return report_error(UPR_ERR_LIMIT, "base must be finite and above 1");
    if (scaling < UPR_ROPE_PLAIN || scaling > UPR_ROPE_BY_PARTS)
        return report_error(UPR_ERR_LIMIT, "rope scaling %d is not a upr_rope_scaling value", scaling);
    if (scaling != UPR_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
        return report_error(UPR_ERR_LIMIT, "factor must be finite and at least 1");
    if (scaling == UPR_ROPE_NTK && rot_dim < 4)
        return report_error(UPR_ERR_LIMIT, "the base change needs rot_dim >= 4");
    if (scaling == UPR_ROPE_BY_PARTS && (!(original_length > 0.0) || !std::isfinite(original_length)))
        return report_error(UPR_ERR_LIMIT, "original_length must be positive and finite");
    upr_rope r{};
    r.rot_dim = rot_dim;
    r.layout = layout;
    r.magnitude = scaling == UPR_ROPE_BY_PARTS ? 1.0 + 0.1 * std::log(factor) : 1.0;
    if (scaling == UPR_ROPE_NTK) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
    if (!std::isfinite(base)) return report_error(UPR_ERR_LIMIT, "base and factor overflow");
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot_dim);
        if (scaling == UPR_ROPE_LINEAR) f /= factor;
        if (scaling == UPR_ROPE_BY_PARTS) {
            const double turns = f * original_length / (2.0 * M_PI);
            const double keep = std::fmin(1.0, std::fmax(0.0, (turns - 1.0) / 31.0));
            f = f * keep + f / factor * (1.0 - keep);
        }
        r.freq[i] = f;
    }
    *out = r;
    return report_ok();
}

upr_status upr_rope_apply(const upr_rope* rope, int32_t dtype, int32_t heads, int32_t head_dim, const void* x,
                          int64_t x_ld, const int32_t* positions, int64_t rows, void* out, int64_t out_ld,
                          void* stream) {
    if (!rope) return report_error(UPR_ERR_NULL, "rope is NULL");
    upr_status st = check_dtype(dtype);
    if (st == UPR_OK) st = check_head_dim(head_dim);
    if (st == UPR_OK) st = check_rope(rope, head_dim);
    if (st != UPR_OK) return st;
    if (heads < 1 || heads > 2048) return report_error(UPR_ERR_LIMIT, "heads %d outside [1, 2048]", heads);
    if (rows < 0 || rows > 0x7fffffff)
        return report_error(UPR_ERR_LIMIT, "rows %lld outside [0, 2^31)", (long long)rows);
    if (rows == 0) return report_ok();
    st = check_rows("x", x, x_ld, heads, head_dim, dtype);
    if (st == UPR_OK) st = check_rows("out", out, out_ld, heads, head_dim, dtype);
    if (st != UPR_OK) return st;
    if (!positions) return report_error(UPR_ERR_NULL, "positions is NULL");
    if (x == out && x_ld != out_ld) return report_error(UPR_ERR_LIMIT, "in place, x_ld and out_ld must agree");
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    {
        ProfScope ps("rope", s);
        e = launch_rope(dtype, rope_args(rope), heads, head_dim, RowsOf{x, x_ld}, positions, rows, out, out_ld, s);
    }
    if (e != hipSuccess) return report_error(UPR_ERR_HIP, "rope launch failed: %s", hipGetErrorString(e));
    return report_ok();
}

upr_status upr_paged_append(const upr_attn_shape* shape, const upr_paged_cache* cache, const upr_segments* fresh,
                            const int32_t* rows_host, const upr_rope* rope, const void* k, int64_t k_ld,
                            const void* v, int64_t v_ld, const void* q, int64_t q_ld, void* q_out,
                            int64_t q_out_ld, void* stream) {
    upr_status st = check_shape(shape);
    if (st == UPR_OK) st = check_paged_cache(cache, false);
    int64_t rows = 0;
    if (st == UPR_OK)
        st = check_paged_users(fresh, "fresh", rows_host, cache->page_rows, cache->table_stride, shape->n_heads, true,
                               &rows);
    if (st == UPR_OK && rope) st = check_rope(rope, shape->head_dim);
    if (st != UPR_OK) return st;
    if ((q == nullptr) != (q_out == nullptr))
        return report_error(UPR_ERR_NULL, "q and q_out must both be given or both be NULL");
    if (rows == 0) return report_ok();
    const int D = shape->head_dim, dt = shape->dtype;
    st = check_paged_cache(cache, true);
    if (st == UPR_OK) st = check_rows("k", k, k_ld, shape->n_kv_heads, D, dt);
    if (st == UPR_OK) st = check_rows("v", v, v_ld, shape->n_kv_heads, D, dt);
    if (st == UPR_OK && q) st = check_rows("q", q, q_ld, shape->n_heads, D, dt);
    if (st == UPR_OK && q) st = check_rows("q_out", q_out, q_out_ld, shape->n_heads, D, dt);
    if (st != UPR_OK) return st;
    if (q && q == q_out && q_ld != q_out_ld)
        return report_error(UPR_ERR_LIMIT, "in place, q_ld and q_out_ld must agree");
    AppendArgs a{};
    a.n_heads = shape->n_heads;
    a.n_kv_heads = shape->n_kv_heads;
    a.D = D;
    a.k = RowsOf{k, k_ld};
    a.v = RowsOf{v, v_ld};
    a.q = RowsOf{q, q_ld};
    a.q_out = q_out;
    a.q_out_ld = q_out_ld;
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    {
        ProfScope ps("paged.append", s);
        e = paged_append(dt, rope_args(rope), a, paged_pool(*cache, 0, 0), fresh, rows_host, s);
    }
    if (e != hipSuccess) return report_error(UPR_ERR_HIP, "append launch failed: %s", hipGetErrorString(e));
    return report_ok();
}

size_t upr_paged_attention_workspace_bytes(const upr_attn_shape* shape, const upr_paged_cache* cache,
                                           const upr_segments* queries, const int32_t* rows_host,
                                           const upr_attn_options* options) {
    int64_t rows;
    if (check_shape(shape) != UPR_OK || check_paged_cache(cache, false) != UPR_OK ||
        check_attn_options(options) != UPR_OK ||
        check_paged_users(queries, "query", rows_host, cache->page_rows, cache->table_stride, shape->n_heads,
                          !options->k_self, &rows) != UPR_OK)
        return 0;
    AttnArgs a = attn_args(*shape, *options);
    return plan_paged_attn(shape->dtype, &a, queries, rows_host);
}

upr_status upr_paged_attention(const upr_attn_shape* shape, const upr_paged_cache* cache,
                               const upr_segments* queries, const int32_t* rows_host,
                               const upr_attn_options* options, const void* q, int64_t q_ld, void* out,
                               int64_t out_ld, void* ws, size_t ws_bytes, void* stream) {
    upr_status st = check_shape(shape);
    if (st == UPR_OK) st = check_paged_cache(cache, false);
    if (st == UPR_OK) st = check_attn_options(options);
    int64_t rows = 0;
    if (st == UPR_OK)
        st = check_paged_users(queries, "query", rows_host, cache->page_rows, cache->table_stride, shape->n_heads,
                               !options->k_self, &rows);
    if (st != UPR_OK) return st;
    if (rows == 0) return report_ok();
    const int D = shape->head_dim, dt = shape->dtype;
    st = check_paged_cache(cache, true);
    if (st == UPR_OK) st = check_rows("q", q, q_ld, shape->n_heads, D, dt);
    if (st == UPR_OK) st = check_rows("out", out, out_ld, shape->n_heads, D, dt);
    if (st == UPR_OK && options->k_self) {
        st = check_rows("k_self", options->k_self, options->self_ld, shape->n_kv_heads, D, dt);
        if (st == UPR_OK) st = check_rows("v_self", options->v_self, options->self_ld, shape->n_kv_heads, D, dt);
    }
    if (st != UPR_OK) return st;
    AttnArgs a = attn_args(*shape, *options);
    const size_t need = plan_paged_attn(dt, &a, queries, rows_host);
    if (need > 0) {
        if (!ws) return report_error(UPR_ERR_NULL, "workspace is NULL (%zu bytes needed)", need);
        if (ws_bytes < need)
            return report_error(UPR_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
        if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
            return report_error(UPR_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    }
    a.q = RowsOf{q, q_ld};
    a.out = out;
    a.out_ld = out_ld;
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    {
        ProfScope ps("paged.attention", s);
        e = paged_attn(dt, a, paged_pool(*cache, 0, 0), queries, rows_host, ws, s);
    }
    if (e != hipSuccess) return report_error(UPR_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
    return report_ok();
}

}  // extern "C"
