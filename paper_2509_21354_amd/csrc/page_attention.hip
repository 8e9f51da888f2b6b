// Attention over a paged 4-bit cache: Eq. 1 of the paper for every batch row over the kept summaries of a compact store (in the
// storage type) and the tokens [first, length) of its pages.
//
// With keys and values in 4 bits a row of d = 128 is 68 bytes, and a compute unit has to take one of them every 5 clocks to keep
// up with the memory: too many elements for the vector unit even for a single query.  Both products therefore run on the matrix
// cores (v_mfma_f32_16x16x32_bf16) at any number of queries, transposed as in the frame kernels so that the softmax weights stay
// in their lanes:
//   S^T = K Q^T   A = 16 tokens, B = 16 queries.  Lane (row l % 16, block l / 16) loads a contiguous quarter of its token's
//                 codes, which lies in one block of 32 and so has one scale, and the hardware conversion gives bf16 with the
//                 scale in it, exactly.  (The contraction index may be permuted freely: step kk of the product takes elements
//                 8 kk .. 8 kk + 7 of every lane's quarter, and the queries are loaded the same way.)
//   O^T = V^T P^T A = V^T through LDS: values converted as above go to a wave's own 32 rows and come back by the transposing
//                 load; B = the weights where the first product left them.
// A wave takes chunks of 64 rows; the waves of a workgroup (1, 4 or 8) take chunks in turn and meet in LDS at the end, the workgroups
// that share a unit's rows meet in scratch (partials, a ticket, the last one to arrive merges in split order).  A unit has one or
// two such tiles of 16 queries (QT): with two, converting and staging a row is paid once for both (512 heads x 32 queries x 4000
// tokens 110 and 73 us).
// What bounds it (d = 128, bf16): 32 layers x 8 rows x 8 heads x 8192 tokens, 2.29 GB, 358 - 378 us = 6.0 - 6.4 TB/s with the vector unit 51 %
// and the matrix cores 26 % busy, a reader without arithmetic reaches 7.2; 64 x 8 heads of ragged rows up to 8192 60 - 63 us = 4.6 - 4.8 TB/s (the
// ends of rows, the join); 32 heads x 4091 tokens 11 us (launch and a chain of five round trips: length and table, codes, partials,
// ticket, partials again).  Four waves on a SIMD spill (629 us).  Tried and dropped, no gain: prefetching without branches, a peeled last
// chunk, store rows asked for ahead; equal shares of all chunks for as many workgroups as fit (410).
// fp32: the queries enter as three bf16 terms of 8 bits, the weights likewise, rows of the store too (of the products of terms those
// are left out that come to 2^-24 of the whole product, see cut3).  bf16: the weights enter as two terms.
//
// Values that are not finite: a block of the cache that held one has the scale byte 255 and reads as NaN.  Such keys make their
// token's scores NaN, which a query that must not see the token replaces.  Values would reach every query of the tile as 0 * NaN,
// so blocks of values marked 255 enter the product as zeros, and the outputs of the queries that do see the token are set to NaN
// at the end.
// Summaries of the store are seen by every query, so a NaN among them may go through the products.  An infinity may not: an operand that
// is cut into terms multiplies it term by term, and a term that is zero, or of the other sign, makes a NaN of what should be an
// infinity.  A wave whose sums are NaN behind its rows of the store takes these rows again, with what is not finite apart: zeros in its place in the
// products of all terms, then a product of its own with the other operand's first term, which has the operand's sign.
#include "kernels.hpp"
#include "pages.hpp"
#include <atomic>
#include <utility>

namespace kvev {

#ifdef __HIP_DEVICE_COMPILE__
__device__ __forceinline__ void store_device(float *p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float load_device(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// fp32 values as three bf16 terms, each the rounded rest of those before: their sum is the value.  The rest of a value of
// magnitude 1 to 2 is below 2^-8 behind the first term and at most 2^-17 behind the second, so of a product of two such values the terms that
// are left out (second times third, third times third) come to less than 2^-24 (1 + 2^-9), with either sign.  (Terms cut off instead
// of rounded have the value's sign: what was left out added up, to as much as 2^-21.)  A value that is not finite has NaN among its terms.
__device__ __forceinline__ void cut3(const float (&x)[8], bf16x8_t (&t)[3])
{
    const float most = __uint_as_float(0x7F7F7FFFu);             // rounded to bf16 the values above would be infinite
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[0][i] = pack_bf16x2(__builtin_amdgcn_fmed3f(x[2 * i], -most, most), __builtin_amdgcn_fmed3f(x[2 * i + 1], -most, most));
        float r[2] = {x[2 * i], x[2 * i + 1]};
#pragma unroll
        for (int k = 1; k < 3; ++k) {
            r[0] -= __uint_as_float(w[k - 1][i] << 16);
            r[1] -= __uint_as_float(w[k - 1][i] & 0xFFFF0000u);
            w[k][i] = pack_bf16x2(r[0], r[1]);
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) t[k] = __builtin_bit_cast(bf16x8_t, make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]));
}

// weights as N bf16 terms: rounded, then what the rounding left
template <int N> __device__ __forceinline__ void cut_weights(const float (&p)[8], bf16x8_t (&t)[N])
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = p[e];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack_bf16x2(r[2 * i], r[2 * i + 1]);
            r[2 * i] -= __uint_as_float(w[i] << 16);
            r[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
        }
        t[k] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

template <typename T> struct Terms;
template <> struct Terms<bf16_t> {
    static constexpr int Q = 1, P = 2;
    struct Raw { bf16x8_t v; };                  // 8 elements as they lie in memory
    static __device__ __forceinline__ void load(const bf16_t *p, Raw &r) { r.v = *reinterpret_cast<const bf16x8_t *>(p); }
    static __device__ __forceinline__ void cut(const Raw &r, bf16x8_t (&t)[1]) { t[0] = r.v; }
    // what is not finite, with zeros in the other places; `r` keeps the rest
    static __device__ __forceinline__ bf16x8_t take_infinite(Raw &r)
    {
        const u32x4_t w = __builtin_bit_cast(u32x4_t, r.v);
        u32x4_t far;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = (w[i] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u, hi = (w[i] & kInfBits) == kInfBits ? 0xFFFF0000u : 0u;
            far[i] = w[i] & (lo | hi);
        }
        r.v = __builtin_bit_cast(bf16x8_t, w ^ far);
        return __builtin_bit_cast(bf16x8_t, far);
    }
};
template <> struct Terms<float> {
    static constexpr int Q = 3, P = 3;
    struct Raw { float v[8]; };
    static __device__ __forceinline__ void load(const float *p, Raw &r) { VecLoad<float, 8>::run(p, r.v); }
    static __device__ __forceinline__ void cut(const Raw &r, bf16x8_t (&t)[3]) { cut3(r.v, t); }
    static __device__ __forceinline__ bf16x8_t take_infinite(Raw &r)
    {
        float far[8];
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool finite = (__float_as_uint(r.v[e]) & kInfBits) != kInfBits;
            far[e] = finite ? 0.f : r.v[e];
            r.v[e] = finite ? r.v[e] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(far[2 * i], far[2 * i + 1]);
        return __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
    }
};

// where in a group's keys or values lane (token n, quarter gr) finds its codes
template <int D> __device__ __forceinline__ int lane_offset(int n, int gr) { return n * (D / 2) + gr * (D / 8); }
template <int D> struct Codes;            // a lane's quarter of a token's codes
template <> struct Codes<128> { typedef u32x4_t type; };
template <> struct Codes<64> { typedef u32x2_t type; };
// from a base that is the same in all lanes
template <bool STREAM, typename V> __device__ __forceinline__ V load_codes(const unsigned char *base, uint32_t offset)
{
    const V *p = reinterpret_cast<const V *>(base + offset);
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}
#endif

// A wave's staging rows: 32 tokens, unpadded.  Piece p (16 bytes) of token t lies at p ^ turn(t): the 16-byte writes of 16 tokens'
// piece p and the transposing reads of 8 tokens' neighbouring pieces then touch every bank once.
template <int D> __device__ __forceinline__ int turn_of(int t)
{
    return D == 128 ? (t & 7) << 1 | (t >> 3 & 1) : (t >> 1 & 3) << 1 | (t >> 3 & 1);
}

// bytes of LDS of a wave: its staging rows, then its outputs
template <int D> constexpr int wave_lds() { return 32 * D * 2 > 16 * (D + 4) * 4 ? 32 * D * 2 : 16 * (D + 4) * 4; }

template <typename T, int D, int NW, bool STREAM, int QT>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 && NW < 8 && QT == 1 ? 3 : 2) void page_attention_kernel(PageAttnArgs a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int NQ = Terms<T>::Q, NP = Terms<T>::P, KS = D / 32, DT = D / 16, NB = D / 32;
    constexpr int OP = D + 4;                    // pitch of the waves' outputs
    constexpr int STAGE = 32 * D * 2;
    extern __shared__ __align__(256) unsigned char s_mem[];
    // maxima and sums of the waves; of the 16 rows of threads in the last merge
    __shared__ float s_m[NW][16], s_l[NW][16];

    const PageGeom &g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, gr = lane >> 4;
    // (workgroups go round-robin over the 8 XCDs: with the runs of a unit side by side, those that short rows of the batch do not
    // take would leave some XCDs idle)
    const int units = (int)(gridDim.x / (uint32_t)a.nsplit), split = (int)(blockIdx.x / (uint32_t)units), unit = (int)(blockIdx.x % (uint32_t)units);
    const int qt = unit % a.qtiles, s = unit / a.qtiles, h = s % g.Hkv, lb = s / g.Hkv, b = lb % g.B, l = lb / g.B;
    const int R = a.G * a.Tq, cap = g.max_pages << g.page_shift;

    // this lane's queries (rows s R .. s R + R - 1 of Q and O are those of the key-value head)
    bf16x8_t qf[QT][KS][NQ];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const size_t row = (size_t)s * R + min((qt * QT + u) * 16 + n, R - 1);
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
            typename Terms<T>::Raw raw;
            Terms<T>::load(static_cast<const T *>(a.Q) + row * D + gr * (D / 4) + kk * 8, raw);
            Terms<T>::cut(raw, qf[u][kk]);
        }
    }

    // Lane 4 j + i holds the table's entry for group i of this wave's chunk j (of 16; its chunks lie NW apart): asked for before the length is there, as if
    // the rows were the pages' from the beginning on and the run as long as planned, which they are most of the time.
    const int32_t *table = a.table + (size_t)b * g.max_pages;
    const uint32_t ahead = (uint32_t)((lane >> 2) * (64 * NW) + (lane & 3) * 16);
    auto entry = [&](uint32_t t) __attribute__((always_inline)) { return table[min((t + ahead) >> g.page_shift, (uint32_t)g.max_pages - 1u)]; };
    const uint32_t guess = ((uint32_t)split * (uint32_t)a.run + (uint32_t)wave) * 64u;
    int pv = entry(guess);

    // the rows of this unit in chunks of 64: the store's, then the pages' from the chunk of `first` on
    const int len = min(max(a.length[b], 0), cap), first = a.first ? min(max(a.first[b], 0), len) : 0;
    const int kept = a.count ? min(max(a.count[s], 0), a.k_cap) : 0;
    const int sc = (kept + 63) >> 6, base0 = first & ~63, pc = (len - base0 + 63) >> 6, chunks = sc + pc;
    const int per = max(a.run, (chunks + a.nsplit - 1) / a.nsplit), active = max(1, (chunks + per - 1) / per);
    if (split >= active) return;
    const int c0 = split * per, c1 = min(chunks, c0 + per);

    int lim[QT], lim_all = len - 1;              // the last token that this lane's queries see, and that all of the unit's see
#pragma unroll
    for (int u = 0; u < QT; ++u) lim[u] = len - 1;
    if (a.q_start) {
        const int64_t at = a.q_start[b];
        const int q0 = qt * QT * 16, q1 = min(q0 + QT * 16, R) - 1;
#pragma unroll
        for (int u = 0; u < QT; ++u) lim[u] = (int)min<int64_t>(lim[u], at + min(q0 + u * 16 + n, R - 1) % a.Tq);
        // (a unit whose queries are the ends of two heads and the beginning of a third has token 0 among them)
        lim_all = (int)min<int64_t>(lim_all, at + (q0 / a.Tq == q1 / a.Tq ? q0 % a.Tq : 0));
    }

    float m[QT], lsum[QT];                       // scaled running maximum and this lane's part of the sum, of query n of each tile
    f32x4_t o[QT][DT];
    uint32_t nan_blocks[QT];                     // blocks of d whose values are NaN in a token that the query sees
    auto reset = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            m[u] = -INFINITY;
            lsum[u] = 0.f;
            nan_blocks[u] = 0;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[u][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    };
    reset();

    // staging: lane (n, gr) writes pieces gr * KS + kk of tokens n and 16 + n; it reads, of tokens 4 gr + n / 4 and 16 further on, piece
    // 2 dt + (n & 3) / 2, half n & 1
    unsigned char *s_v = s_mem + wave * STAGE;
    unsigned char *put[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) put[kk] = s_v + n * (2 * D) + (((gr * KS + kk) ^ turn_of<D>(n)) << 4);
    const int row = 4 * gr + (n >> 2);
    const uint32_t get = (uint32_t)(row * (2 * D) + ((((n & 3) >> 1) ^ turn_of<D>(row)) << 4) + (n & 1) * 8);

    const float c = a.scale_log2e;
    const size_t block = block_bytes(g);
    const unsigned char *pool = a.pool + ((size_t)l * g.n_pages * g.Hkv + h) * block;

    // the weights of a chunk from its scores (hidden ones: -inf), and the running state
    auto soft = [&](int u, f32x4_t (&st)[4], bf16x8_t (&pb)[2][NP]) __attribute__((always_inline)) {
        float mx = max3(st[0][0], st[0][1], st[0][2]);
        mx = max3(mx, st[0][3], st[1][0]);
#pragma unroll
        for (int i = 5; i < 15; i += 2) mx = max3(mx, st[i / 4][i % 4], st[(i + 1) / 4][(i + 1) % 4]);
        mx = rows_max(fmaxf(mx, st[3][3])) * c;
        const float m_new = fmaxf(m[u], mx);
        if (__any(m_new > m[u] + kSlack)) {
            const float alpha = __builtin_amdgcn_exp2f(m[u] - (m_new == -INFINITY ? 0.f : m_new));
            lsum[u] *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[u][dt][e] *= alpha;
            m[u] = m_new;
        }
        const float ref = m[u] == -INFINITY ? 0.f : m[u];
        // (The multiply-add leaves the rounding of the maximum's product in every weight, a factor that the normaliser shares.
        // Where it is no longer near 1, the products are rounded first.)
        float cc = c;
        if (__any(fabsf(ref) > 0x1p20f)) {
            cc = 1.0f;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) st[kt][e] *= c;
        }
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(st[2 * h2 + (e >> 2)][e & 3], cc, -ref));
                lsum[u] += p[e];
            }
            cut_weights<NP>(p, pb[h2]);
        }
    };
    // the 32 staged rows are this wave's alone, and its LDS accesses keep their order: only the compiler is held
    auto hold = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    // O^T += V^T P^T over them: one term of the values, with the weights' terms that matter (all but the last `skip`)
    auto values = [&](const bf16x8_t (&pb)[QT][2][NP], int h2, int skip) __attribute__((always_inline)) {
        hold();
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            unsigned char *src = s_v + (get ^ (uint32_t)(dt << 5));
            const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)src);
            const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)(src + 16 * 2 * D));
            const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int k = NP - 1; k >= 0; --k)
                    if (k + skip < NP) o[u][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[u][h2][k], o[u][dt], 0, 0, 0);
        }
        hold();
    };

    // ---- rows of the store ----
    // (fp32: cutting a row into terms is most of the work, so half chunks without rows are passed over and values are read once for all
    // terms: 16 summaries of 2 x 4 heads x 33 queries and 320 tokens take 6.6 us, as do the tokens alone; they added 3.5 without)
    // (APART: what is not finite by itself)
    int ch;
    auto store_rows = [&](auto apart) __attribute__((always_inline)) {
        constexpr bool APART = decltype(apart)::value;
        for (ch = c0 + wave; ch < min(sc, c1); ch += NW) {
            f32x4_t st[QT][4];
            bf16x8_t pb[QT][2][NP];
            const T *Kc = static_cast<const T *>(a.Kc) + (size_t)s * a.k_cap * D, *Vc = static_cast<const T *>(a.Vc) + (size_t)s * a.k_cap * D;
            const int here = kept - ch * 64;         // rows of this chunk (1 and more)
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
                for (int u = 0; u < QT; ++u) st[u][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (NQ == 1 || kt / 2 * 32 < here) {
#pragma unroll
                    for (int kk = 0; kk < KS; ++kk) {
                        typename Terms<T>::Raw raw;
                        bf16x8_t kf[NQ];
                        if constexpr (APART) __builtin_amdgcn_sched_barrier(0);      // (or the loads of all pieces take registers)
                        Terms<T>::load(Kc + (size_t)min(ch * 64 + kt * 16 + n, kept - 1) * D + gr * (D / 4) + kk * 8, raw);
                        bf16x8_t far;
                        if constexpr (APART) far = Terms<T>::take_infinite(raw);
                        Terms<T>::cut(raw, kf);
#pragma unroll
                        for (int u = 0; u < QT; ++u)
#pragma unroll
                            for (int x = NQ - 1; x >= 0; --x)
#pragma unroll
                                for (int y = NQ - 1 - x; y >= 0; --y) st[u][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[x], qf[u][kk][y], st[u][kt], 0, 0, 0);
                        if constexpr (APART) {
#pragma unroll
                            for (int u = 0; u < QT; ++u) st[u][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(far, qf[u][kk][0], st[u][kt], 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (kt * 16 + 4 * gr + e >= here) st[u][kt][e] = -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < QT; ++u) soft(u, st[u], pb[u]);
#pragma unroll
            for (int h2 = 0; h2 < 2; ++h2) {
                if (NQ > 1 && h2 * 32 >= here) break;
                typename Terms<T>::Raw raw[2][KS];
                auto load = [&](int i, int kk) __attribute__((always_inline)) {
                    Terms<T>::load(Vc + (size_t)min(ch * 64 + h2 * 32 + i * 16 + n, kept - 1) * D + gr * (D / 4) + kk * 8, raw[i][kk]);
                };
                if (NQ > 1 && !APART) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int kk = 0; kk < KS; ++kk) load(i, kk);
                }
#pragma unroll
                for (int x = NQ - 1; x >= 0; --x) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int kk = 0; kk < KS; ++kk) {
                            bf16x8_t vf[NQ];
                            if constexpr (APART) __builtin_amdgcn_sched_barrier(0);
                            if (NQ == 1 || APART) load(i, kk);
                            if constexpr (APART) Terms<T>::take_infinite(raw[i][kk]);
                            Terms<T>::cut(raw[i][kk], vf);
                            if (h2 * 32 + i * 16 + n >= here) vf[x] = __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
                            *reinterpret_cast<bf16x8_t *>(put[kk] + i * 16 * 2 * D) = vf[x];
                        }
                    values(pb, h2, x);
                }
                if constexpr (APART) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int kk = 0; kk < KS; ++kk) {
                            __builtin_amdgcn_sched_barrier(0);
                            load(i, kk);
                            bf16x8_t far = Terms<T>::take_infinite(raw[i][kk]);
                            if (h2 * 32 + i * 16 + n >= here) far = __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
                            *reinterpret_cast<bf16x8_t *>(put[kk] + i * 16 * 2 * D) = far;
                        }
                    values(pb, h2, NP - 1);
                }
            }
        }
    };
    store_rows(std::false_type{});
    if (c0 + wave < min(sc, c1)) {
        float sum = 0.f;                         // (NaN if one of them is, or two are infinite)
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            sum += lsum[u];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) sum += (o[u][dt][0] + o[u][dt][1]) + (o[u][dt][2] + o[u][dt][3]);
        }
        if (__any(sum != sum)) {                 // (rare)
            reset();
            store_rows(std::true_type{});
        }
    }

    // ---- tokens of the pages ----
    const int tok = base0 + (ch - sc) * 64;      // the first of this wave's chunks
    const int mine = ch < c1 ? (c1 - ch + NW - 1) / NW : 0;
    if ((uint32_t)tok != guess) pv = entry((uint32_t)tok);
    // the pages of chunks j0 .. j0 + 15 from their entries; -1: none
    auto checked = [&](int e, int j0) __attribute__((always_inline)) {
        const uint32_t pi = ((uint32_t)tok + (uint32_t)j0 * (64u * NW) + ahead) >> g.page_shift;
        return j0 + (lane >> 2) < mine && pi < (uint32_t)g.max_pages && (uint32_t)e < (uint32_t)g.n_pages ? e : -1;
    };
    typedef typename Codes<D>::type codes_t;
    const uint32_t at_codes = (uint32_t)lane_offset<D>(n, gr), at_scale = (uint32_t)(n * NB + gr * NB / 4) * 2;
    codes_t kc[4], vc[4];
    uint32_t sk[4], sv[4];                       // scale bytes: of the key, of the value in the byte above
    const unsigned char *vbase[4];
    pv = checked(pv, 0);
    int pv_next = entry((uint32_t)tok + 16u * (64u * NW));
    auto fetch_keys = [&](int j) __attribute__((always_inline)) {
        const int t0 = tok + j * (64 * NW);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int page = max(__builtin_amdgcn_readlane(pv, (j & 15) * 4 + i), 0);
            const uint32_t in = (uint32_t)(t0 + 16 * i) & ((1u << g.page_shift) - 1u);
            const unsigned char *p = pool + (size_t)(uint32_t)page * (uint32_t)g.Hkv * block + (size_t)(in >> 4) * group_bytes(D);
            vbase[i] = p + 8 * D;
            kc[i] = load_codes<STREAM, codes_t>(p, at_codes);
            sk[i] = load_codes<STREAM, uint16_t>(p + 16 * D, at_scale);
        }
    };
    auto fetch_values = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { vc[i] = load_codes<STREAM, codes_t>(vbase[i], at_codes); sv[i] = sk[i]; }
    };
    if (mine > 0) {
        fetch_keys(0);
        fetch_values();
    }
    for (int j = 0; j < mine; ++j) {
        const int t0 = tok + j * (64 * NW);
        const uint64_t none = __ballot(pv < 0);
        const uint32_t gone = (uint32_t)(none >> ((j & 15) * 4)) & 15u;       // groups without a page
        const bool full = gone == 0 && t0 >= first && t0 + 64 <= len && t0 + 63 <= lim_all;
        // (what lies in no page, before `first` or behind the length may hold anything: its scores are replaced, its values are zeros)
        if (!full) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((gone >> i & 1) || t0 + 16 * i + n < first || t0 + 16 * i + n >= len) { vc[i] = codes_t{}; sv[i] = 127u << 8; }
        }
        f32x4_t st[QT][4];
        bf16x8_t pb[QT][2][NP];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int u = 0; u < QT; ++u) st[u][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                const bf16x8_t kf = unpack8(kc[kt][kk], __uint_as_float(sk[kt] << 23));
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int y = NQ - 1; y >= 0; --y) st[u][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[u][kk][y], st[u][kt], 0, 0, 0);
            }
        }
        if (j + 1 < mine) {
            if ((j + 1) % 16 == 0) {
                pv = checked(pv_next, j + 1);
                pv_next = entry((uint32_t)tok + (uint32_t)(j + 17) * (64u * NW));
            }
            fetch_keys(j + 1);
        }
        if (!full) {
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = t0 + 16 * kt + 4 * gr + e;
                        if ((gone >> kt & 1) || t < first || t > lim[u]) st[u][kt][e] = -INFINITY;
                    }
        }
#pragma unroll
        for (int u = 0; u < QT; ++u) soft(u, st[u], pb[u]);
        if (__any(max(max(sv[0], sv[1]), max(sv[2], sv[3])) >= kNanScale << 8)) {       // (rare)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint64_t bad = __ballot(sv[i] >= kNanScale << 8);
                while (bad) {
                    const int x = __builtin_ctzll(bad);
                    bad &= bad - 1;
#pragma unroll
                    for (int u = 0; u < QT; ++u)
                        if (t0 + 16 * i + (x & 15) <= lim[u]) nan_blocks[u] |= 1u << ((x >> 4) * NB / 4);
                }
                if (sv[i] >= kNanScale << 8) { vc[i] = codes_t{}; sv[i] = 127u << 8; }
            }
        }
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int kk = 0; kk < KS; ++kk)
                    *reinterpret_cast<bf16x8_t *>(put[kk] + i * 16 * 2 * D) = unpack8(vc[2 * h2 + i][kk], __uint_as_float(sv[2 * h2 + i] << 15));
            if (h2 == 1 && j + 1 < mine) fetch_values();
            values(pb, h2, 0);
        }
    }
#pragma unroll
    for (int u = 0; u < QT; ++u)
        if (nan_blocks[u]) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                if (nan_blocks[u] >> (dt / 2) & 1) o[u][dt] = f32x4_t{NAN, NAN, NAN, NAN};
        }

    // ---- the waves meet, a tile of 16 queries at a time ----
    float *s_o = reinterpret_cast<float *>(s_mem);               // (the staging rows become the waves' outputs)
    constexpr int TPQ = 4 * NW, EPT = D / TPQ;   // threads per query, and their elements, TPQ apart
    const int oq = tid / TPQ, oe = tid % TPQ;
    const int q_first = qt * QT * 16;
    auto store_out = [&](int q, const float (&acc)[EPT], float L) __attribute__((always_inline)) {
        T *O = static_cast<T *>(a.O) + ((size_t)s * R + q_first + q) * D;
        const float inv = 1.0f / L;                              // (no rows: 0 below; a NaN stays one)
#pragma unroll
        for (int e = 0; e < EPT; ++e) Storage<T>::store(O + oe + TPQ * e, L == 0.f ? 0.f : acc[e] * inv);
    };
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        __syncthreads();
        const float lw = rows_sum(lsum[u]);
        if (gr == 0) { s_m[wave][n] = m[u]; s_l[wave][n] = lw; }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t *>(s_o + (wave * 16 + n) * OP + dt * 16 + 4 * gr) = o[u][dt];
        __syncthreads();
        float M = s_m[0][oq];
#pragma unroll
        for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][oq]);
        const float Mr = M == -INFINITY ? 0.f : M;
        float L = 0.f, acc[EPT] = {};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][oq] - Mr);
            L += s_l[w][oq] * f;
#pragma unroll
            for (int e = 0; e < EPT; ++e) acc[e] += s_o[(w * 16 + oq) * OP + oe + TPQ * e] * f;
        }
        const int q = u * 16 + oq;
        if (q_first + q >= R) continue;
        if (active == 1) {
            store_out(q, acc, L);
            continue;
        }
        float *part = a.part + (((size_t)unit * a.nsplit + split) * (16 * QT) + q) * (D + 2);
#pragma unroll
        for (int e = 0; e < EPT; ++e) store_device(part + oe + TPQ * e, acc[e]);
        if (oe == 0) { store_device(part + D, M); store_device(part + D + 1, L); }
    }
    if (active == 1) return;
    // ---- the workgroups meet: as in decode attention ----
    __shared__ int s_last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // this wave's stores have completed
    __syncthreads();
    if (tid == 0) s_last = __hip_atomic_fetch_add(a.tickets + unit, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == active - 1;
    __syncthreads();
    if (!s_last) return;
    if (tid == 0) __hip_atomic_store(a.tickets + unit, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // Few queries leave most of the 16 rows of threads idle: those take partials side by side (row q + Q k: partials k, k + 16 / Q, ...
    // of query q), which are added up in LDS in that order.
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int live = min(16, R - q_first - u * 16);
        if (live <= 0) return;
        int lq = 0;
        while (1 << lq < live) ++lq;
        const int Q = 1 << lq, q = oq & (Q - 1), k0 = oq >> lq, kn = 16 >> lq;
        float L = 0.f, M = -INFINITY, acc[EPT] = {};
        if (q < live) {
            const float *part = a.part + ((size_t)unit * a.nsplit * (16 * QT) + u * 16 + q) * (D + 2);
#pragma unroll 2
            for (int x = k0; x < active; x += kn) {
                const float *pp = part + (size_t)x * (16 * QT) * (D + 2);
                const float px = load_device(pp + D), pl = load_device(pp + D + 1);
                float v[EPT];
#pragma unroll
                for (int e = 0; e < EPT; ++e) v[e] = load_device(pp + oe + TPQ * e);
                const float Mn = fmaxf(M, px), ref = Mn == -INFINITY ? 0.f : Mn, f0 = __builtin_amdgcn_exp2f(M - ref), f1 = __builtin_amdgcn_exp2f(px - ref);
                L = L * f0 + pl * f1;
#pragma unroll
                for (int e = 0; e < EPT; ++e) acc[e] = acc[e] * f0 + v[e] * f1;
                M = Mn;
            }
        }
        if (kn > 1) {
            // (the reads of s_o and s_m before lie behind the barriers of the ticket: only the unit's last tile has few queries)
            float *mm = &s_m[0][0], *ll = &s_l[0][0];
            if (oe == 0) { mm[oq] = M; ll[oq] = L; }
#pragma unroll
            for (int e = 0; e < EPT; ++e) s_o[oq * OP + oe + TPQ * e] = acc[e];
            __syncthreads();
            if (k0 != 0) return;
            M = -INFINITY;
            for (int k = 0; k < kn; ++k) M = fmaxf(M, mm[q + Q * k]);
            const float ref = M == -INFINITY ? 0.f : M;
            L = 0.f;
#pragma unroll
            for (int e = 0; e < EPT; ++e) acc[e] = 0.f;
            for (int k = 0; k < kn; ++k) {
                const float f = __builtin_amdgcn_exp2f(mm[q + Q * k] - ref);
                L += ll[q + Q * k] * f;
#pragma unroll
                for (int e = 0; e < EPT; ++e) acc[e] += s_o[(q + Q * k) * OP + oe + TPQ * e] * f;
            }
        }
        if (q < live) store_out(u * 16 + q, acc, L);
    }
#endif
}

template <typename T, int D, int NW, bool STREAM, int QT> static hipError_t launch_waves(const PageAttnArgs &a, hipStream_t st)
{
    constexpr int lds = NW * wave_lds<D>();
    if (lds > 64 * 1024 - 2048) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_lds(page_attention_kernel<T, D, NW, STREAM, QT>, lds, done);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)((int64_t)a.g.L * a.g.B * a.g.Hkv * a.qtiles * a.nsplit));
    hipLaunchKernelGGL((page_attention_kernel<T, D, NW, STREAM, QT>), grid, dim3(64 * NW), lds, st, a);
    return hipGetLastError();
}
template <typename T, int D, bool STREAM, int QT> static hipError_t launch_stream(const PageAttnArgs &a, int waves, hipStream_t st)
{
    if (waves == 1) return launch_waves<T, D, 1, STREAM, QT>(a, st);
    if constexpr (QT == 1) {
        if (waves == 8) return launch_waves<T, D, 8, STREAM, QT>(a, st);
    }
    return launch_waves<T, D, 4, STREAM, QT>(a, st);
}
template <typename T, int QT> static hipError_t launch_type(const PageAttnArgs &a, int waves, hipStream_t st)
{
    if (a.g.d == 128) return a.stream ? launch_stream<T, 128, true, QT>(a, waves, st) : launch_stream<T, 128, false, QT>(a, waves, st);
    return a.stream ? launch_stream<T, 64, true, QT>(a, waves, st) : launch_stream<T, 64, false, QT>(a, waves, st);
}

hipError_t launch_page_attention(const PageAttnArgs &a, int dtype, int queries, int waves, hipStream_t st)
{
    if (dtype == KVEV_F32) return launch_type<float, 1>(a, waves, st);
    return queries == 32 ? launch_type<bf16_t, 2>(a, waves, st) : launch_type<bf16_t, 1>(a, waves, st);
}

}  // namespace kvev
