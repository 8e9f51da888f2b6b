// Attention of a frame of queries over a paged 4-bit cache (bf16; the same work as page_attention.hip, for more queries to a
// key-value head).
//
// With many queries the products bound it, and what a row costs to convert has to be paid once for all of them.  A workgroup takes
// 32 queries per wave (4 or 8 waves) of one key-value head and walks the rows in tiles of 64: the codes of a tile are in registers
// one tile ahead, 16 tokens a wave; they go through the hardware conversion into LDS as bf16 while the tile before is computed, into
// the other of two slots, and one barrier per tile hands them over.  The products are the ones of the frame kernels over raw
// caches: v_mfma_f32_32x32x16_bf16, transposed (S^T = K Q^T, O^T = V^T P^T), so that the weights stay in their lanes; values by
// the transposing LDS load; weights of a step made under the products of the one before.
// The weights enter the second product rounded to bf16 (the output is rounded to no more bits, and their terms' second half would cost as
// many matrix instructions again); the normaliser sums the rounded ones, two to an instruction.
// Measured (d = 128): 16 rows x 8 heads x 1024 queries over 8192 tokens, 541 GFLOP, 511 - 552 us = 980 - 1058 TFLOP/s, where the library's bf16
// product of 8192^3 reaches 1231.  Matrix and vector work take 45 % of a SIMD's clocks each and hardly overlap: that bounds it.
// Tried and dropped: raised wave priority around the products (no difference); half of the waves staging behind their products (553 for
// 527 us); the two waves of a SIMD half a tile apart, one making scores while the other makes weights (611 for 541); the next
// tile converted between the products (533 for 519).
#include "kernels.hpp"
#include "pages.hpp"
#include <atomic>
#include <utility>

namespace kvev {

#ifdef __HIP_DEVICE_COMPILE__
// Rows lie unpadded in LDS; piece c (16 bytes) of a row is put at c ^ swizzle(row).  Keys: 16 lanes that read or write one piece of 16
// rows touch every bank once.  Values: so do 16 lanes that write one piece of 16 rows, and 32 lanes that read four pieces of four
// rows (transposing loads).
template <int D> __device__ __forceinline__ int swizzle_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D> __device__ __forceinline__ int swizzle_v(int row)
{
    return D == 128 ? 4 * (row & 3) + ((row >> 2) & 3) : 4 * ((row >> 1) & 1) + ((row >> 2) & 3);
}
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8_t;

// The rows of a unit: the store's in tiles of 64, then the pages' from the tile of `first` up to the last token that some of its
// queries sees; and the run of tiles that each of `active` workgroups takes.
struct FrameRows {
    int len, first, kept;
    int lim_any;                  // the last token that some of the unit's queries see
    int sc, base0, tiles;         // tiles of the store, first token of the pages' tiles, all tiles
    int per, active;
};
__device__ __forceinline__ FrameRows frame_rows(const PageAttnArgs &a, int b, int s, int qt, int queries)
{
    FrameRows w;
    const int R = a.G * a.Tq;
    w.len = min(max(a.length[b], 0), a.g.max_pages << a.g.page_shift);
    w.first = a.first ? min(max(a.first[b], 0), w.len) : 0;
    w.kept = a.count ? min(max(a.count[s], 0), a.k_cap) : 0;
    w.lim_any = w.len - 1;
    if (a.q_start) {
        const int64_t at = a.q_start[b];
        const int q0 = qt * queries, q1 = min(q0 + queries, R) - 1;
        const bool one = q0 / a.Tq == q1 / a.Tq;           // (queries of one head)
        w.lim_any = (int)min<int64_t>(w.lim_any, at + (one ? q1 % a.Tq : a.Tq - 1));
    }
    w.sc = (w.kept + 63) >> 6;
    w.base0 = w.first & ~63;
    w.tiles = w.sc + ((max(w.lim_any + 1, w.base0) - w.base0 + 63) >> 6);
    w.per = max(a.run, (w.tiles + a.nsplit - 1) / a.nsplit);
    w.active = max(1, (w.tiles + w.per - 1) / w.per);
    return w;
}

// Which of a key-value head's query tiles stands x-th in the order of workgroups.  Tokens that see only those before them have rows
// in proportion to their place: the tiles of late tokens come first, of all heads, so that the short ones fill what the long ones
// leave (one row x 4096 tokens, 8 heads of 4: 270 us in ascending order, 177 us).  The tiles that begin in head g are
// ceil(g Tq / queries) and on: floor(Tq / queries) of them, or one more.
__device__ __forceinline__ int frame_tile(const PageAttnArgs &a, int x, int queries)
{
    if (!a.q_start) return x;
    const int base = a.Tq / queries;
    int extra = 0, longer = -1;
    for (int g = 0; g < a.G; ++g) {
        const int begin = (int)(((int64_t)g * a.Tq + queries - 1) / queries), end = (int)(((int64_t)(g + 1) * a.Tq + queries - 1) / queries);
        if (end - begin > base) {
            if (extra == x) longer = end - 1;
            ++extra;
        }
    }
    if (x < extra) return longer;
    x -= extra;
    const int k = base - 1 - x / a.G, g = x % a.G;
    return (int)(((int64_t)g * a.Tq + queries - 1) / queries) + k;
}

// lane (n, hh) holds d = 32 dt + 8 q + 4 hh + 0 .. 3 of its query in registers 4 q .. 4 q + 3 of o[dt]
template <int DT> __device__ __forceinline__ void store_frame(bf16_t *O, const f32x16_t (&o)[DT], float L)
{
    const float inv = 1.0f / L;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint2 w;
            w.x = pack_bf16x2(o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv);
            w.y = pack_bf16x2(o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv);
            if (L == 0.f) w = make_uint2(0u, 0u);          // (no rows)
            *reinterpret_cast<uint2 *>(O + dt * 32 + 8 * q) = w;
        }
}
#endif

// floats of a wave's partial: o in pieces of 16 bytes per lane, then maximum and sum
constexpr int frame_part(int d) { return 64 * (d / 2 + 2); }

template <int D, int NWV>
__global__ __launch_bounds__(64 * NWV, NWV == 4 ? 2 : 1) void page_frame_kernel(PageAttnArgs a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int KS = D / 16, DT = D / 32, BM = 32 * NWV, RB = 2 * D, TB = 64 * RB, NB = D / 32, RING = 6;
    constexpr int NP = D / 32;                   // 16-byte pieces of a lane's quarter of a row
    constexpr bool BOTH = NWV == 4;              // a wave takes the keys and the values of 16 tokens, or one of the two
    extern __shared__ __align__(1024) unsigned char smem_frame[];
    lds_byte_t *lds = (lds_byte_t *)smem_frame;  // [2 slots][keys, values][64 rows]
    __shared__ uint64_t s_nan[2][4];             // blocks of values that are NaN: bit (token % 16) + 16 * quarter of a row

    const PageGeom &g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5, n16 = lane & 15, gr = lane >> 4;
    // an XCD takes a contiguous run of units: the query tiles of a key-value head meet in its L2
    uint32_t id = blockIdx.x;
    if (gridDim.x % 8 == 0) id = (id % 8) * (gridDim.x / 8) + id / 8;
    const int units = (int)(gridDim.x / (uint32_t)a.nsplit), split = (int)(id / (uint32_t)units), unit = (int)(id % (uint32_t)units);
    const int qt = frame_tile(a, unit % a.qtiles, BM), s = unit / a.qtiles, h = s % g.Hkv, lb = s / g.Hkv, b = lb % g.B, l = lb / g.B;
    const int R = a.G * a.Tq;

    // this lane's query (rows s R .. s R + R - 1 of Q and O are those of the key-value head)
    const int qrow = qt * BM + wave * 32 + n, rc = min(qrow, R - 1), tq = rc % a.Tq;
    const size_t orow = (size_t)s * R + rc;
    bf16x8_t qf[KS];
    const bf16_t *Qp = static_cast<const bf16_t *>(a.Q) + orow * D + hh * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t *>(Qp + ks * 16);

    const FrameRows w = frame_rows(a, b, s, qt, BM);
    if (split >= w.active) return;
    const int len = w.len, first = w.first, kept = w.kept, sc = w.sc, base0 = w.base0;
    const int lim = a.q_start ? (int)min<int64_t>(len - 1, (int64_t)a.q_start[b] + tq) : len - 1;      // the last token that this lane's query sees
    int lim_all = len - 1, lim_any = len - 1;                                  // ... and that all, and some, of this wave's see
    if (a.q_start) {
        const int q0 = min(qt * BM + wave * 32, R - 1), q1 = min(q0 + 31, R - 1);
        const bool one = q0 / a.Tq == q1 / a.Tq;
        const int64_t at = a.q_start[b];
        lim_all = (int)min<int64_t>(lim_all, at + (one ? q0 % a.Tq : 0));
        lim_any = (int)min<int64_t>(lim_any, at + (one ? q1 % a.Tq : a.Tq - 1));
    }
    const int t0 = split * w.per, t1 = min(w.tiles, t0 + w.per);

    // ---- tiles into LDS ----
    const size_t block = block_bytes(g);
    const unsigned char *pool = a.pool + ((size_t)l * g.n_pages * g.Hkv + h) * block;
    const int32_t *table = a.table + (size_t)b * g.max_pages;
    // lane 4 j + i holds the page of group i of tile f0 + j (j < 16; -1: none)
    int f0 = -16, pv = -1;
    auto lookup = [&](int t) __attribute__((always_inline)) {
        f0 = t;
        const uint32_t pi = ((uint32_t)base0 + (uint32_t)(t - sc) * 64u + (uint32_t)lane * 16u) >> g.page_shift;
        const int e = table[min(pi, (uint32_t)g.max_pages - 1u)];
        pv = pi < (uint32_t)g.max_pages && (uint32_t)e < (uint32_t)g.n_pages ? e : -1;
    };
    typedef typename std::conditional<D == 128, u32x4_t, u32x2_t>::type codes_t;
    const int group = wave & 3;                  // of a tile: the 16 tokens that this wave brings
    const uint32_t at_codes = (uint32_t)(n16 * (D / 2) + gr * (D / 8)), at_scale = (uint32_t)(n16 * NB + gr * NB / 4) * 2;
    codes_t c0 = {}, c1 = {};                    // keys (or what this wave has of the two), values
    uint32_t scale = 0;
    uint32_t gone_next = 0, gone = 0;            // groups of the tile in flight, and of the one in LDS, that have no page
    auto fetch = [&](int t) __attribute__((always_inline)) {
        if (t < sc || t >= t1) return;
        if (t >= f0 + 16 || t < f0) lookup(t);
        gone_next = (uint32_t)(__ballot(pv < 0) >> ((t - f0) * 4)) & 15u;
        const int page = max(__builtin_amdgcn_readlane(pv, (t - f0) * 4 + group), 0);
        const uint32_t in = (uint32_t)(base0 + (t - sc) * 64 + 16 * group) & ((1u << g.page_shift) - 1u);
        const unsigned char *p = pool + (size_t)(uint32_t)page * (uint32_t)g.Hkv * block + (size_t)(in >> 4) * group_bytes(D);
        if (BOTH || wave < 4) c0 = *reinterpret_cast<const codes_t *>(p + at_codes);
        else c0 = *reinterpret_cast<const codes_t *>(p + 8 * D + at_codes);
        if (BOTH) c1 = *reinterpret_cast<const codes_t *>(p + 8 * D + at_codes);
        scale = *reinterpret_cast<const uint16_t *>(p + 16 * D + at_scale);
    };
    const int row = group * 16 + n16;            // this lane's row of a tile
    auto put_piece = [&](int slot, bool v, int p, bf16x8_t x) __attribute__((always_inline)) {
        const int at = (p ^ (v ? swizzle_v<D>(row) : swizzle_k<D>(row))) << 4;
        *(lds_bf16x8_t *)(lds + slot * 2 * TB + (v ? TB : 0) + row * RB + at) = x;
    };
    auto put = [&](int t, int slot) __attribute__((always_inline)) {
        if (t >= t1) return;
        const bool keys = BOTH || wave < 4, values = BOTH || wave >= 4;
        if (t < sc) {
            const int j = t * 64 + row;
            const size_t off = ((size_t)s * a.k_cap + min(j, kept - 1)) * D + gr * (D / 4);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const bf16x8_t zero = __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
                if (keys) put_piece(slot, false, gr * NP + p, *reinterpret_cast<const bf16x8_t *>(static_cast<const bf16_t *>(a.Kc) + off + p * 8));
                if (values) {
                    const bf16x8_t x = *reinterpret_cast<const bf16x8_t *>(static_cast<const bf16_t *>(a.Vc) + off + p * 8);
                    put_piece(slot, true, gr * NP + p, j < kept ? x : zero);
                }
            }
            if (values && lane == 0) s_nan[slot][group] = 0;
            return;
        }
        if (keys) {
            const float f = __uint_as_float(scale << 23);
#pragma unroll
            for (int p = 0; p < NP; ++p) put_piece(slot, false, gr * NP + p, unpack8(c0[p], f));
        }
        if (values) {
            // what lies in no page, before `first` or behind the length may hold anything, and blocks that are NaN would reach every
            // query: zeros in their place
            codes_t c = BOTH ? c1 : c0;
            const int tok = base0 + (t - sc) * 64 + row;
            const bool hold = !(gone_next >> group & 1) && tok >= first && tok < len, bad = hold && scale >= kNanScale << 8;
            const uint64_t mask = __ballot(bad);
            float f = __uint_as_float(scale << 15);
            if (!hold || bad) { c = codes_t{}; f = 1.0f; }
#pragma unroll
            for (int p = 0; p < NP; ++p) put_piece(slot, true, gr * NP + p, unpack8(c[p], f));
            if (lane == 0) s_nan[slot][group] = mask;
        }
    };

    // ---- fragments out of LDS: see the frame kernels over raw caches ----
    const int k_rd = n * RB + ((hh ^ swizzle_k<D>(n)) << 4);                    // ^ (ks << 5)
    const int v_row = 4 * hh + (n16 >> 2), v_piece = 2 * (gr & 1) + ((n16 >> 1) & 1);
    const int v_lo = TB + v_row * RB + ((v_piece ^ swizzle_v<D>(v_row)) << 4) + 8 * (n16 & 1);             // ^ (dt << 6)
    const int v_hi = TB + (v_row + 8) * RB + ((v_piece ^ swizzle_v<D>(v_row + 8)) << 4) + 8 * (n16 & 1);
    const float c = a.scale_log2e;
    const bool busy = qt * BM + wave * 32 < R;   // this wave has queries
    float m = -INFINITY, lsum = 0.f;
    uint32_t nan_blocks = 0;
    f32x16_t o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;

    fetch(t0);
    put(t0, 0);
    gone = gone_next;
    fetch(t0 + 1);
    for (int t = t0; t < t1; ++t) {
        const int slot = (t - t0) & 1;
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        __builtin_amdgcn_s_barrier();            // the tile is there for all waves, and nobody reads the one before
        asm volatile("" : : : "memory");
        const uint32_t gone_now = gone;
        put(t + 1, slot ^ 1);
        gone = gone_next;
        fetch(t + 2);
        const bool stored = t < sc;
        const int tok = base0 + (t - sc) * 64;
        if (!busy || (!stored && tok > lim_any)) continue;
        const lds_byte_t *tile = lds + slot * 2 * TB;
        const bool full = stored ? t * 64 + 64 <= kept : gone_now == 0 && tok >= first && tok + 64 <= len && tok + 63 <= lim_all;

        f32x16_t st[2];
        bf16x8_t ring[RING];
        auto read_k = [&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            ring[i % RING] = *(const lds_bf16x8_t *)(tile + (k_rd ^ ((i / 2) << 5)) + (i % 2) * 32 * RB);
        };
        auto read_v = [&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, sx = i / DT, dt = i % DT;
            const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)(tile + (v_lo ^ (dt << 6)) + 16 * sx * RB));
            const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)(tile + (v_hi ^ (dt << 6)) + 16 * sx * RB));
            ring[i % RING] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        static_for<RING>(read_k);
        __builtin_amdgcn_sched_barrier(0);
        static_for<2 * KS>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, ks = i / 2, kb = i % 2;
            const f32x16_t zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            st[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % RING], qf[ks], ks == 0 ? zero : st[kb], 0, 0, 0);
            if constexpr (i + RING < 2 * KS) read_k(std::integral_constant<int, i + RING>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        static_for<RING>(read_v);
        const uint64_t marked = s_nan[slot][lane & 3];
        __builtin_amdgcn_sched_barrier(0);
        // register r of block kb is row 32 kb + 8 (r / 4) + 4 hh + r % 4 of the tile
        if (!full) {
            // rows lo .. hi of the tile are seen
            const int lo = stored ? 0 : max(first - tok, 0), hi = stored ? kept - 1 - t * 64 : min(lim - tok, 63);
            const uint32_t from = hi < lo ? 0x40000000u : (uint32_t)(lo - 4 * hh), span = hi < lo ? 0u : (uint32_t)(hi - lo);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[kb][r] = (uint32_t)(32 * kb + 8 * (r >> 2) + (r & 3)) - from > span ? -INFINITY : st[kb][r];
            if (gone_now != 0 && !stored) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (gone_now >> (2 * kb + (r >> 3)) & 1) st[kb][r] = -INFINITY;
            }
        }
        float mx = max3(st[0][0], st[0][1], st[1][0]), my = max3(st[0][2], st[0][3], st[1][1]);
#pragma unroll
        for (int r = 2; r < 16; r += 2) {
            mx = max3(mx, st[1][r], st[1][r + 1]);
            if (r > 2) my = max3(my, st[0][r], st[0][r + 1]);
        }
        mx = fmaxf(mx, my);
        my = mx;
        swap32(mx, my);
        mx = fmaxf(m, fmaxf(mx, my) * c);
        if (__any(mx > m + kSlack)) {
            const float alpha = __builtin_amdgcn_exp2f(m - (mx == -INFINITY ? 0.f : mx));
            m = mx;
            lsum *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float cc = c;
        if (__any(fabsf(ref) > 0x1p20f)) {       // (see page_attention.hip)
            cc = 1.0f;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[kb][r] *= c;
        }
        uint32_t pw[2][4];
        float p_even = 0.f;
        auto weights = [&](auto sxc, auto ec) __attribute__((always_inline)) {          // of rows 2 e, 2 e + 1 of step sx
            constexpr int sx = decltype(sxc)::value, e = decltype(ec)::value;
            const float p0 = __builtin_amdgcn_exp2f(fmaf(st[sx >> 1][8 * (sx & 1) + 2 * e], cc, -ref));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(st[sx >> 1][8 * (sx & 1) + 2 * e + 1], cc, -ref));
            pw[sx & 1][e] = pack_bf16x2(p0, p1);
            (e & 1 ? p_even : lsum) = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pw[sx & 1][e]), __builtin_bit_cast(bf16x2_t, 0x3F803F80u), e & 1 ? p_even : lsum, false);
        };
        static_for<4>([&](auto ec) __attribute__((always_inline)) { weights(std::integral_constant<int, 0>{}, ec); });
        static_for<4 * DT>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, sx = i / DT, dt = i % DT;
            const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, make_uint4(pw[sx & 1][0], pw[sx & 1][1], pw[sx & 1][2], pw[sx & 1][3]));
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % RING], pb, o[dt], 0, 0, 0);
            if constexpr (i + RING < 4 * DT) read_v(std::integral_constant<int, i + RING>{});
            if constexpr (sx < 3)
                static_for<4 / DT>([&](auto kc) __attribute__((always_inline)) {
                    weights(std::integral_constant<int, (sx + 1) & 3>{}, std::integral_constant<int, dt * (4 / DT) + decltype(kc)::value>{});
                });
            __builtin_amdgcn_sched_barrier(0);
        });
        lsum += p_even;
        if (__any(marked != 0)) {                // (rare)
            for (int i = 0; i < 4; ++i)
                for (uint64_t bad = s_nan[slot][i]; bad; bad &= bad - 1) {
                    const int x = __builtin_ctzll(bad);
                    if (tok + 16 * i + (x & 15) <= lim) nan_blocks |= 1u << ((x >> 4) * NB / 4);
                }
        }
    }
    if (nan_blocks) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            if (nan_blocks >> dt & 1)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] = NAN;
    }

    float lo = lsum;
    swap32(lsum, lo);
    const float L = lsum + lo;
    if (w.active == 1) {
        if (qrow < R) store_frame<DT>(static_cast<bf16_t *>(a.O) + orow * D + 4 * hh, o, L);
        return;
    }
    float *part = a.part + (((size_t)unit * a.nsplit + split) * NWV + wave) * frame_part(D);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            reinterpret_cast<f32x4_t *>(part)[(dt * 4 + q) * 64 + lane] = f32x4_t{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]};
    reinterpret_cast<float2 *>(part + 64 * (D / 2))[lane] = make_float2(m, L);
#endif
}

// The partials of a unit's runs, added up in their order; a wave takes what one wave of page_frame_kernel left in `dt`.  A launch of
// its own, with the chip to itself: a unit's last workgroup would have 66 KiB and more of every other one to read.
template <int D, int NWV>
__global__ __launch_bounds__(256) void page_frame_merge_kernel(PageAttnArgs a, int waves)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int DT = D / 32;
    const PageGeom &g = a.g;
    const int lane = threadIdx.x & 63, n = lane & 31, hh = lane >> 5;
    const int x = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (x >= waves) return;
    const int dt = x % DT, wave = x / DT % NWV, unit = x / (DT * NWV);
    const int qt = frame_tile(a, unit % a.qtiles, 32 * NWV), s = unit / a.qtiles, b = s / g.Hkv % g.B, R = a.G * a.Tq;
    const int qrow = qt * 32 * NWV + wave * 32 + n;
    if (qt * 32 * NWV + wave * 32 >= R) return;
    const FrameRows w = frame_rows(a, b, s, qt, 32 * NWV);
    if (w.active == 1) return;
    const size_t step = (size_t)NWV * frame_part(D);
    const float *part = a.part + ((size_t)unit * a.nsplit * NWV + wave) * frame_part(D);
    float M = -INFINITY, L = 0.f;
    for (int i = 0; i < w.active; ++i) M = fmaxf(M, reinterpret_cast<const float2 *>(part + i * step + 64 * (D / 2))[lane].x);
    const float ref = M == -INFINITY ? 0.f : M;
    f32x16_t o[1];
#pragma unroll
    for (int r = 0; r < 16; ++r) o[0][r] = 0.f;
#pragma unroll 2
    for (int i = 0; i < w.active; ++i) {
        const float2 ml = reinterpret_cast<const float2 *>(part + i * step + 64 * (D / 2))[lane];
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        L += ml.y * f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4_t v = reinterpret_cast<const f32x4_t *>(part + i * step)[(dt * 4 + q) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[0][4 * q + e] += v[e] * f;
        }
    }
    if (qrow < R) store_frame<1>(static_cast<bf16_t *>(a.O) + ((size_t)s * R + qrow) * D + dt * 32 + 4 * hh, o, L);
#endif
}

template <int D, int NWV> static hipError_t launch_frame_as(const PageAttnArgs &a, hipStream_t st)
{
    constexpr int lds = 2 * 2 * 64 * 2 * D;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = allow_lds(page_frame_kernel<D, NWV>, lds, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((page_frame_kernel<D, NWV>), dim3((unsigned)((int64_t)a.g.L * a.g.B * a.g.Hkv * a.qtiles * a.nsplit)), dim3(64 * NWV), lds, st, a);
    if (a.nsplit > 1) {
        const int waves = a.g.L * a.g.B * a.g.Hkv * a.qtiles * NWV * (D / 32);
        hipLaunchKernelGGL((page_frame_merge_kernel<D, NWV>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, a, waves);
    }
    return hipGetLastError();
}

hipError_t launch_page_frame(const PageAttnArgs &a, int queries, hipStream_t st)
{
    if (a.g.d == 64) return launch_frame_as<64, 4>(a, st);
    return queries == 256 ? launch_frame_as<128, 8>(a, st) : launch_frame_as<128, 4>(a, st);
}

}  // namespace kvev
