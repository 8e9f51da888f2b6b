// C-ABI layer of the paged 4-bit cache and of rotary positions: argument validation (host only, before any HIP call), launch
// planning, dispatch.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <atomic>

#include "../../include/kvev_test_hooks.h"
#include "api.hpp"
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

static bool aligned4(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static bool aligned4_or_null(const void *p) { return !p || aligned4(p); }
static bool whole16(const void *p) { return p && aligned16(p); }

// whether [p, p + n) and [q, q + m) share a byte
static bool overlap(const void *p, size_t n, const void *q, size_t m)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    return x < y + m && y < x + n;
}

static int check_pages(const kvev_shape *sh, const kvev_pages *pg, PageGeom *g)
{
    const int rc = check_shape(sh, false);
    if (rc) return rc;
    if (!pg || pg->n_pages < 1 || pg->max_pages < 1) return KVEV_ERR_INVALID_ARG;
    int shift = 0;
    while (shift < 9 && 1 << shift != pg->page) ++shift;
    if (shift < 4 || shift > 8) return KVEV_ERR_UNSUPPORTED;
    // positions are 31 bits, and so are the places of table entries and the sums of page counts
    if (((int64_t)pg->max_pages << shift) > INT32_MAX - 256) return KVEV_ERR_INVALID_ARG;
    if ((int64_t)sh->B * ((int64_t)pg->max_pages + 1) > INT32_MAX || (int64_t)sh->L * pg->n_pages > INT32_MAX) return KVEV_ERR_INVALID_ARG;
    *g = PageGeom{sh->L, sh->B, kv_heads(sh), sh->d, shift, pg->n_pages, pg->max_pages};
    return KVEV_OK;
}
static size_t elem(const kvev_shape *sh) { return sh->dtype == KVEV_F32 ? 4 : 2; }
static size_t pool_bytes(const PageGeom &g) { return (size_t)g.L * g.n_pages * page_bytes(g); }

// ---- attention over pages: planning ----
// A unit is 16 or 32 queries of a key-value head; its rows, in chunks of 64 for one wave each, are cut into runs of `run` chunks, a
// workgroup of 1, 4 or 8 waves each.  A batch row takes as many of a unit's nsplit workgroups as its own length pays for
// (decided on the device, where the lengths are).  shape->T, or the capacity if it is 0, says for which length the launch is made;
// results depend on it in the order of sums and the choice of form only.
//   * While runs of 8 chunks are no more than the compute units: 8 waves, a chunk each (us, 8 and 4 waves: 32 units x 300 tokens 7.3 and
//     8.0, x 1000 9.9 and 10.9, x 4091 11.2 and 11.8; 64 units x 2000 10.7 and 11.1; 8 units x 16000 13.8 and 15.3).  More runs,
//     or longer ones, are worse: 512 units x 400 tokens 13.1 and 9.9.  fp32, whose registers leave no room for more waves than
//     that, takes them up to one unit per compute unit (256 units x 2000 tokens 19.9 and 23.0).
//   * Many units of short rows: a wave each, which has no other wave to wait for and whose beginning others hide (2048 units x 320
//     tokens 19.5, with 4 waves 24.7; x 1000 49.3 and 53.7; 16384 x 320 116 and 156; but x 8192 383 and 358, and 512 units x
//     320 12.4 and 8.9).
//   * Else 4 waves, in runs that give every compute unit one, of 4 chunks at least; where such a run would be longer than 16 chunks, in
//     runs for four workgroups per compute unit, of 16 chunks at least: they hide each other's ends, and long rows of a ragged
//     batch are spread (32 x 16000 tokens 19.9 us, one workgroup per compute unit 22.0; 512 units of 64 ragged rows up to 8192
//     tokens 63, unsplit 72; 128 units of 16 ragged rows up to 12000 29 and 47).
// Units of 32 queries (bf16) convert a row once for all of them, but leave registers for two waves on a SIMD and half the units: they are
// taken where they are two per compute unit, or half as many with enough rows (units of 16 and 32, us; 32 queries to a key-value
// head: 512 heads x 200 tokens 13.3 and 11.2, x 4000 110 and 73; 256 x 300 9.2 and 10.4, x 1000 17.6 and 16.6, x 4000 54 and 42; 128 x
// 4000 33.8 and 28.2, of 16 ragged rows up to 8192 36.6 and 39.1; 32 x 4000 15.6 and 19.4).  Their runs give every compute unit two
// workgroups, all that it holds at once (four: 81 and 47 at 512 and 256 heads x 4000).
// Frames (page_frame.hip; bf16): units of 128 or, for more queries at d = 128, 256, two workgroups or one per compute unit, whichever
// takes less by the count of rounds (256 and 128, us: 128 heads x 292 queries x 4000 tokens 122 and 139, 512 x 292 x 600 101 and 78, 32 x
// 580 x 4000 72 and 62, 128 x 1024 x 8192 521 and 573).  At d = 64 the
// registers of 128 queries fit three times, which gives more than converting a row for 256 at once (16 x 8 heads x 1024 queries x 8192
// tokens 353 us, with 256 queries 386; one row of 4096 causal tokens 92 and 110).  Frames take calls with 48 queries
// or more to a key-value head (65 where units of 32 are taken: 128 heads x 64 queries x 8192 tokens 70 and 84, 512 x 64 x 600
// 32.3 and 29.4) and enough work (units of 16 queries x tokens; 4 query heads to a key-value head, units of 16 and frame, us):
// 128 x 128 x 600 23.7 and 22.1; 128 x 256 x 600 32.6 and 29.0; 8 x 1024 x 4000 45.7 and 38.6; but 8 x 1024 x 600 12.1 and 22.2, 8 x 256
// x 4000 19.9 and 34.4.
constexpr int kPageChunk = 64, kPageMaxSplit = 64, kFrameQueries = 48, kFrameRounds = 3;
constexpr int64_t kFrameWork = 1200000;
constexpr int64_t kPairWork = 2000, kPairMost = 64;
static std::atomic<int64_t> g_frame_work{kFrameWork};      // (kvev_debug_page_frame_work lowers it)
static std::atomic<int64_t> g_pair_units{0};               // (kvev_debug_page_pair_units: 0: by the rule)
struct PageAttnPlan { int queries, waves, qtiles, nsplit, run; int64_t units; size_t ticket_bytes, ws_bytes, ws_any; double time; };
static PageAttnPlan plan_page_form(const kvev_shape *sh, const PageGeom &g, int Tq, int64_t tokens, int queries)
{
    PageAttnPlan p{};
    const int64_t R = (int64_t)(sh->H / g.Hkv) * Tq, cus = device_compute_units(), cap = (int64_t)g.max_pages << g.page_shift;
    const bool frame = queries > 32;
    p.queries = queries;
    p.qtiles = (int)((R + p.queries - 1) / p.queries);
    p.units = (int64_t)g.L * g.B * g.Hkv * p.qtiles;
    const int64_t chunks = (tokens + kPageChunk - 1) / kPageChunk, slots = p.queries == 128 ? (g.d == 64 ? 3 : 2) * cus : cus;
    auto fill = [&](int64_t wgs) { return (chunks * p.units + wgs - 1) / wgs; };       // the run of which `wgs` workgroups take all
    int64_t run;
    if (frame) {
        p.waves = p.queries / 32;
        // as many runs as give the least time: rounds of workgroups, each run two tiles longer for its beginning and end, a tile of
        // 64 rows 2.2 us (d = 128; 2.4 for two workgroups of 128 queries), partials out and in at 4 TB/s and a launch
        const double tile = (queries == 128 ? 2.4 : 2.2) * g.d / 128, merge = 2.0 * p.queries * (g.d + 4) * sizeof(float) / 4e6;
        double least = 0;
        int64_t best = 1;
        for (int64_t n = 1; n <= std::min<int64_t>(kPageMaxSplit, (chunks + 3) / 4) && (n == 1 || p.units * n <= kFrameRounds * slots); ++n) {
            const double rounds = (double)((p.units * n + slots - 1) / slots);
            const double t = rounds * ((double)((chunks + n - 1) / n) + 2) * tile + (n > 1 ? 4 + merge * (double)(p.units * n) : 0.0);
            if (n == 1 || t < least) { least = t; best = n; }
        }
        run = (chunks + best - 1) / best;
        p.time = least;
    } else if (queries == 16 && (sh->dtype == KVEV_F32 ? p.units <= cus : p.units * ((chunks + 7) / 8) <= cus)) {
        p.waves = 8;
        const int64_t n = std::max<int64_t>(cus / p.units, 1);
        run = std::max<int64_t>((chunks + n - 1) / n, 8);
    } else if (p.units >= 6 * cus && chunks <= 32) {
        p.waves = 1;
        run = chunks;
    } else {
        p.waves = 4;
        run = std::max<int64_t>(fill(cus), 4);
        if (run > 16) run = std::max<int64_t>(fill((queries == 32 ? 2 : 4) * cus), 16);
    }
    run = std::min(std::max(run, (chunks + kPageMaxSplit - 1) / kPageMaxSplit), std::max<int64_t>(chunks, 1));
    p.run = (int)run;
    p.nsplit = (int)std::max<int64_t>(1, (chunks + run - 1) / run);
    // Tickets, then the partials of every run: 16 queries' outputs, maxima and sums, or the waves' of a frame as they hold them.
    // One ticket per unit of 16 queries that is split; four workgroups per compute unit bound their number, and room for as many
    // stands first whatever the call: the partials of one call then never lie where another one has its tickets.
    p.ticket_bytes = ((size_t)4 * cus * sizeof(int32_t) + 255) / 256 * 256;
    const size_t partial = (size_t)p.queries * (g.d + (frame ? 4 : 2)) * sizeof(float);
    p.ws_bytes = p.nsplit > 1 ? p.ticket_bytes + (size_t)p.units * p.nsplit * partial : 0;
    // enough for every length of row and for fewer queries: split units take the workgroups wanted (rounded up to the unit), and no
    // run is shorter than 4 chunks
    const int64_t wanted = frame ? kFrameRounds * slots : 4 * slots, units = std::min(p.units, wanted), most = (cap / kPageChunk + 4) / 4;
    p.ws_any = most > 1 ? p.ticket_bytes + (size_t)std::min({units * kPageMaxSplit, units + wanted, units * most}) * partial : 0;
    return p;
}
static PageAttnPlan plan_page_attn(const kvev_shape *sh, const PageGeom &g, int Tq, int64_t tokens)
{
    const int64_t R = (int64_t)(sh->H / g.Hkv) * Tq, cus = device_compute_units(), pairs = g_pair_units.load();
    PageAttnPlan best = plan_page_form(sh, g, Tq, tokens, 16);
    if (sh->dtype != KVEV_BF16 || R <= 16) return best;
    const int64_t work = best.units * tokens;
    size_t any = best.ws_any;                    // (the form depends on the length and the queries as well)
    const PageAttnPlan p = plan_page_form(sh, g, Tq, tokens, 32);
    any = std::max(any, p.ws_any);
    const bool pair = pairs > 0 ? p.units >= pairs : p.units >= 2 * cus || (2 * p.units >= cus && p.units * tokens >= kPairWork * cus);
    if (pair) best = p;
    if (R >= kFrameQueries) {
        PageAttnPlan f = plan_page_form(sh, g, Tq, tokens, 128);
        any = std::max(any, f.ws_any);
        if (R > 128 && g.d == 128) {
            const PageAttnPlan w = plan_page_form(sh, g, Tq, tokens, 256);
            any = std::max(any, w.ws_any);
            if (w.time <= f.time) f = w;
        }
        if (work >= g_frame_work.load() && !(pair && R <= kPairMost)) best = f;
    }
    best.ws_any = any;
    return best;
}
static bool page_queries_fit(const kvev_shape *sh, int Tq) { return (int64_t)sh->L * sh->B * sh->H * Tq <= (int64_t)1 << 26; }
static int64_t plan_tokens(const kvev_shape *sh, const PageGeom &g)
{
    const int64_t cap = (int64_t)g.max_pages << g.page_shift;
    return sh->T > 0 ? std::min<int64_t>(sh->T, cap) : cap;
}

static int check_tables(const PageGeom &, const void *table, const void *length, const void *refs)
{
    return aligned4(table) && aligned4(length) && aligned4(refs) ? KVEV_OK : KVEV_ERR_INVALID_ARG;
}

static int rows_common(const kvev_shape *sh, const kvev_pages *pg, const void *K, const void *V, int Tn, const int32_t *start, const int32_t *n_new,
                       const int32_t *table, void *pool, PageRowsArgs *a)
{
    memset(a, 0, sizeof *a);
    const int rc = check_pages(sh, pg, &a->g);
    if (rc) return rc;
    if (!whole16(K) || !whole16(V) || !whole16(pool) || !aligned4(table) || !aligned4(start) || !aligned4_or_null(n_new) || Tn < 0)
        return KVEV_ERR_INVALID_ARG;
    if ((int64_t)sh->L * sh->B * a->g.Hkv * Tn > (int64_t)1 << 30) return KVEV_ERR_INVALID_ARG;
    a->pool = static_cast<unsigned char *>(pool); a->table = table; a->start = start; a->n_new = n_new; a->Tn = Tn;
    return KVEV_OK;
}

}  // namespace kvev

using namespace kvev;

extern "C" {

int kvev_debug_page_frame_work(int64_t work)
{
    if (work < 0) return KVEV_ERR_INVALID_ARG;
    g_frame_work = work == 0 ? kFrameWork : work;
    return KVEV_OK;
}

int kvev_debug_page_pair_units(int64_t units)
{
    if (units < 0) return KVEV_ERR_INVALID_ARG;
    g_pair_units = units;
    return KVEV_OK;
}

int kvev_debug_page_form(const kvev_shape *sh, const kvev_pages *pg, int Tq, int *queries, int *waves, int *runs)
{
    PageGeom g;
    if (check_pages(sh, pg, &g) != KVEV_OK || Tq < 1 || !page_queries_fit(sh, Tq) || !queries || !waves || !runs) return KVEV_ERR_INVALID_ARG;
    const PageAttnPlan p = plan_page_attn(sh, g, Tq, plan_tokens(sh, g));
    *queries = p.queries;
    *waves = p.waves;
    *runs = p.nsplit;
    return KVEV_OK;
}

size_t kvev_page_pool_bytes(const kvev_shape *sh, const kvev_pages *pg)
{
    PageGeom g;
    return check_pages(sh, pg, &g) == KVEV_OK ? pool_bytes(g) : 0;
}

size_t kvev_page_workspace_bytes(int op, const kvev_shape *sh, const kvev_pages *pg, int n)
{
    PageGeom g;
    if (check_pages(sh, pg, &g) != KVEV_OK || n < 0) return 0;
    switch (op) {
    case KVEV_OP_PAGE_ATTENTION:
        return n == 0 || !page_queries_fit(sh, n) ? 0 : plan_page_attn(sh, g, n, plan_tokens(sh, g)).ws_any;
    case KVEV_OP_PAGES_RESERVE:
        return reserve_words(g) * 4;
    case KVEV_OP_PAGES_COMPACT:
        return compact_words(g) * 4;
    default:
        return 0;
    }
}

int kvev_rotary(const kvev_shape *sh, const kvev_rotary_axes *axes, const float *freq, const int32_t *pos, int Tq, const void *Q,
                const void *K, void *Q_out, void *K_out, int inverse, void *stream)
{
    const int rc = check_shape(sh, false);
    if (rc) return rc;
    if (!axes || axes->n_axes < 1 || axes->n_axes > 4 || Tq < 0 || (inverse != 0 && inverse != 1)) return KVEV_ERR_INVALID_ARG;
    RotaryArgs a;
    memset(&a, 0, sizeof a);
    int64_t pairs = 0;
    for (int x = 0; x < axes->n_axes; ++x) {
        if (axes->section[x] < 0) return KVEV_ERR_INVALID_ARG;
        pairs += axes->section[x];
        a.end[x] = (int)std::min<int64_t>(pairs, sh->d);
    }
    for (int x = axes->n_axes; x < 4; ++x) a.end[x] = a.end[axes->n_axes - 1];
    if (pairs < 1 || 2 * pairs > sh->d) return KVEV_ERR_INVALID_ARG;
    if (axes->layout != KVEV_ROTARY_HALVES && axes->layout != KVEV_ROTARY_PAIRS) return KVEV_ERR_UNSUPPORTED;
    if (!aligned4(freq) || !aligned4(pos) || (!Q && !K) || !Q != !Q_out || !K != !K_out) return KVEV_ERR_INVALID_ARG;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(Q_out) || !aligned16(K_out)) return KVEV_ERR_INVALID_ARG;
    if (Tq == 0) return KVEV_OK;
    const int Hkv = kv_heads(sh);
    if ((int64_t)sh->L * sh->B * sh->H * Tq > (int64_t)1 << 28 || (int64_t)axes->n_axes * sh->B * Tq > INT32_MAX) return KVEV_ERR_INVALID_ARG;
    // in place, or apart from everything else
    const size_t nq = Q ? (size_t)sh->L * sh->B * sh->H * Tq * sh->d * elem(sh) : 0, nk = K ? (size_t)sh->L * sh->B * Hkv * Tq * sh->d * elem(sh) : 0;
    if (Q && Q != Q_out && overlap(Q, nq, Q_out, nq)) return KVEV_ERR_INVALID_ARG;
    if (K && K != K_out && overlap(K, nk, K_out, nk)) return KVEV_ERR_INVALID_ARG;
    if (Q && K && (overlap(Q_out, nq, K_out, nk) || overlap(Q, nq, K_out, nk) || overlap(Q_out, nq, K, nk))) return KVEV_ERR_INVALID_ARG;
    a.Q = Q; a.K = K; a.Qo = Q_out; a.Ko = K_out; a.freq = freq; a.pos = pos;
    a.L = sh->L; a.B = sh->B; a.H = sh->H; a.Hkv = Hkv; a.d = sh->d; a.Tq = Tq; a.n_axes = axes->n_axes;
    a.pairs = (int)pairs; a.adjacent = axes->layout == KVEV_ROTARY_PAIRS; a.sign = inverse ? -1.f : 1.f;
    const hipError_t e = launch_rotary(a, sh->dtype, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_page_append(const kvev_shape *sh, const kvev_pages *pg, const void *K, const void *V, int Tn, const int32_t *start,
                     const int32_t *n_new, const int32_t *table, void *pool, void *stream)
{
    PageRowsArgs a;
    const int rc = rows_common(sh, pg, K, V, Tn, start, n_new, table, pool, &a);
    if (rc || Tn == 0) return rc;
    a.K = K; a.V = V;
    const hipError_t e = launch_page_append(a, sh->dtype, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_page_read(const kvev_shape *sh, const kvev_pages *pg, const void *pool, const int32_t *table, const int32_t *first,
                   const int32_t *n, int Tn, void *K, void *V, void *stream)
{
    PageRowsArgs a;
    const int rc = rows_common(sh, pg, K, V, Tn, first, n, table, const_cast<void *>(pool), &a);
    if (rc || Tn == 0) return rc;
    const size_t bytes = (size_t)sh->L * sh->B * a.g.Hkv * Tn * sh->d * elem(sh);
    if (overlap(K, bytes, V, bytes)) return KVEV_ERR_INVALID_ARG;
    a.Ko = K; a.Vo = V;
    const hipError_t e = launch_page_read(a, sh->dtype, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_page_attention(const kvev_shape *sh, const kvev_pages *pg, const void *Q, int Tq, const void *pool, const int32_t *table,
                        const int32_t *length, const int32_t *first, const int32_t *q_start, const void *Kc, const void *Vc,
                        const int32_t *count, int k_cap, void *O, void *ws, size_t ws_bytes, void *stream)
{
    PageAttnArgs a;
    memset(&a, 0, sizeof a);
    const int rc = check_pages(sh, pg, &a.g);
    if (rc) return rc;
    if (!whole16(Q) || !whole16(O) || !whole16(pool) || !aligned4(table) || !aligned4(length) || !aligned4_or_null(first) ||
        !aligned4_or_null(q_start) || Tq < 0 || k_cap < 0)
        return KVEV_ERR_INVALID_ARG;
    if (k_cap > 0 && (!whole16(Kc) || !whole16(Vc) || !aligned4(count))) return KVEV_ERR_INVALID_ARG;
    if ((int64_t)sh->L * sh->B * a.g.Hkv * k_cap > INT32_MAX) return KVEV_ERR_INVALID_ARG;
    if (Tq == 0) return KVEV_OK;
    if (!page_queries_fit(sh, Tq)) return KVEV_ERR_INVALID_ARG;
    const size_t q_bytes = (size_t)sh->L * sh->B * sh->H * Tq * sh->d * elem(sh);
    if (overlap(Q, q_bytes, O, q_bytes)) return KVEV_ERR_INVALID_ARG;
    const PageAttnPlan p = plan_page_attn(sh, a.g, Tq, plan_tokens(sh, a.g));
    if (p.ws_bytes > 0 && (!whole16(ws) || ws_bytes < p.ws_bytes)) return KVEV_ERR_WORKSPACE;
    a.Q = Q; a.O = O; a.pool = static_cast<const unsigned char *>(pool); a.table = table; a.length = length; a.first = first; a.q_start = q_start;
    if (k_cap > 0) { a.Kc = Kc; a.Vc = Vc; a.count = count; a.k_cap = k_cap; }
    a.G = sh->H / a.g.Hkv; a.Tq = Tq; a.nsplit = p.nsplit; a.qtiles = p.qtiles; a.run = p.run;
    if (p.nsplit > 1) {
        a.tickets = static_cast<int32_t *>(ws);
        a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + p.ticket_bytes);
    }
    a.stream = (size_t)sh->L * sh->B * a.g.Hkv * (size_t)plan_tokens(sh, a.g) * 17 * sh->d / 16 > attn_stream_bytes();
    a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)sh->d));
    const hipError_t e = p.queries <= 32 ? launch_page_attention(a, sh->dtype, p.queries, p.waves, static_cast<hipStream_t>(stream))
                                         : launch_page_frame(a, p.queries, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_pages_reserve(const kvev_shape *sh, const kvev_pages *pg, const int32_t *n_new, int32_t *table, int32_t *length, int32_t *refs,
                       void *pool, int32_t *start, int32_t *status, void *ws, size_t ws_bytes, void *stream)
{
    PagesArgs a;
    memset(&a, 0, sizeof a);
    int rc = check_pages(sh, pg, &a.g);
    if (rc) return rc;
    rc = check_tables(a.g, table, length, refs);
    if (rc) return rc;
    if (!aligned4(n_new) || !aligned4(start) || !aligned4(status) || !whole16(pool)) return KVEV_ERR_INVALID_ARG;
    const size_t row_bytes = (size_t)sh->B * 4;
    if (overlap(n_new, row_bytes, length, row_bytes) || overlap(start, row_bytes, length, row_bytes) || overlap(start, row_bytes, n_new, row_bytes))
        return KVEV_ERR_INVALID_ARG;
    if (!whole16(ws) || ws_bytes < reserve_words(a.g) * 4) return KVEV_ERR_WORKSPACE;
    a.n_new = n_new; a.table = table; a.length = length; a.refs = refs; a.pool = static_cast<unsigned char *>(pool);
    a.start = start; a.status = status; a.ws = static_cast<int32_t *>(ws);
    const hipError_t e = launch_pages_reserve(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_pages_fork(const kvev_shape *sh, const kvev_pages *pg, const int32_t *src, const int32_t *dst, int n, int32_t *table,
                    int32_t *length, int32_t *refs, int32_t *status, void *stream)
{
    PagesArgs a;
    memset(&a, 0, sizeof a);
    int rc = check_pages(sh, pg, &a.g);
    if (rc) return rc;
    rc = check_tables(a.g, table, length, refs);
    if (rc) return rc;
    if (n < 0 || n > sh->B || !aligned4(status) || !aligned4(src) || !aligned4(dst)) return KVEV_ERR_INVALID_ARG;
    if (n == 0) return KVEV_OK;
    a.src = src; a.dst = dst; a.n = n; a.table = table; a.length = length; a.refs = refs; a.status = status;
    const hipError_t e = launch_pages_fork(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_pages_trim(const kvev_shape *sh, const kvev_pages *pg, const int32_t *rows, int n, const int32_t *first, const int32_t *keep,
                    int32_t *table, int32_t *length, int32_t *refs, void *stream)
{
    PagesArgs a;
    memset(&a, 0, sizeof a);
    int rc = check_pages(sh, pg, &a.g);
    if (rc) return rc;
    rc = check_tables(a.g, table, length, refs);
    if (rc) return rc;
    if (n < 0 || n > sh->B || !aligned4_or_null(rows) || !aligned4_or_null(first) || !aligned4_or_null(keep)) return KVEV_ERR_INVALID_ARG;
    if (n == 0) return KVEV_OK;
    a.src = rows; a.n = n; a.first = first; a.keep = keep; a.table = table; a.length = length; a.refs = refs;
    const hipError_t e = launch_pages_trim(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_pages_copy(const kvev_shape *sh, const kvev_pages *pg, void *pool, const int32_t *src, const int32_t *dst, int n,
                    int32_t *status, void *stream)
{
    PagesArgs a;
    memset(&a, 0, sizeof a);
    const int rc = check_pages(sh, pg, &a.g);
    if (rc) return rc;
    if (n < 0 || n > pg->n_pages || !whole16(pool) || !aligned4(src) || !aligned4(dst) || !aligned4(status)) return KVEV_ERR_INVALID_ARG;
    if (n == 0) return KVEV_OK;
    a.pool = static_cast<unsigned char *>(pool); a.src = src; a.dst = dst; a.n = n; a.status = status;
    const hipError_t e = launch_pages_copy(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

int kvev_pages_compact(const kvev_shape *sh, const kvev_pages *pg, const void *pool, const int32_t *table, const int32_t *refs,
                       const kvev_pages *to, void *to_pool, int32_t *to_table, int32_t *to_refs, int32_t *status, void *ws,
                       size_t ws_bytes, void *stream)
{
    PagesArgs a;
    PageGeom t;
    memset(&a, 0, sizeof a);
    int rc = check_pages(sh, pg, &a.g);
    if (!rc) rc = check_pages(sh, to, &t);
    if (rc) return rc;
    if (t.page_shift != a.g.page_shift || t.max_pages != a.g.max_pages) return KVEV_ERR_INVALID_ARG;
    if (!whole16(pool) || !whole16(to_pool) || !aligned4(table) || !aligned4(refs) || !aligned4(to_table) || !aligned4(to_refs) || !aligned4(status))
        return KVEV_ERR_INVALID_ARG;
    const size_t cells = (size_t)a.g.B * a.g.max_pages * 4;
    if (overlap(pool, pool_bytes(a.g), to_pool, pool_bytes(t)) || overlap(refs, (size_t)a.g.n_pages * 4, to_refs, (size_t)t.n_pages * 4) ||
        (table != to_table && overlap(table, cells, to_table, cells)))
        return KVEV_ERR_INVALID_ARG;
    if (!whole16(ws) || ws_bytes < compact_words(a.g) * 4) return KVEV_ERR_WORKSPACE;
    a.pool = static_cast<unsigned char *>(const_cast<void *>(pool)); a.table = const_cast<int32_t *>(table); a.refs = const_cast<int32_t *>(refs);
    a.to_pool = static_cast<unsigned char *>(to_pool); a.to_table = to_table; a.to_refs = to_refs; a.to_pages = t.n_pages;
    a.status = status; a.ws = static_cast<int32_t *>(ws);
    a.stream = std::min(pool_bytes(a.g), pool_bytes(t)) > attn_stream_bytes();
    const hipError_t e = launch_pages_compact(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? KVEV_OK : hip_fail(e);
}

}  // extern "C"
