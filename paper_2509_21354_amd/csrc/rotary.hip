// Rotary positions of tokens that have several coordinates (time, height, width): pair j of a head's elements is turned by the
// angle pos[axis of j] * freq[j].
//
// The angle is taken in double: a 31-bit position times a 24-bit frequency is 55 bits, and the turns that are thrown away are
// most of them for far tokens.  What is left of a turn goes to sine and cosine in fp32 (an error of 2^-25 turns).  They depend on
// the token and not on the head, so a thread makes those of its pairs once and takes them through the heads of its slice;
// queries and keys of one call are one list of heads.  Bytes bound it, sine and cosine where a token has few heads: 64 rows x 256
// tokens x (32 + 8) heads, bf16, d = 128: 65 - 71 us, 4.7 - 5.2 TB/s in and out, what a copy of that size reaches.  Where the pairs are
// no multiple of a piece, halves pay for the ends of pieces (4 x 1000 x 64 heads, 61 pairs: 31 us, as neighbouring pairs 23; with
// ends element by element 51).  Tried and dropped: non-temporal accesses (no difference).
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

// Pieces of up to 16 bytes (W elements), wherever they begin: memory takes such accesses at any element.  A piece of n < W elements
// is read whole where the tensor goes on behind it (`end`), and written in 8, 4 and 2 bytes.
template <typename T, int W> __device__ __forceinline__ void get_piece(const T *p, int n, const T *end, float (&o)[W])
{
    if (n >= W || end - p >= W) {
        u32x4_t w;
        __builtin_memcpy(&w, p, 16);
#pragma unroll
        for (int i = 0; i < W; ++i) o[i] = sizeof(T) == 4 ? __uint_as_float(w[i % 4]) : __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        return;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = i < n ? Storage<T>::load(p + i) : 0.f;
}
template <typename T, int W> __device__ __forceinline__ void put_piece(T *p, int n, const float (&o)[W])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(o[i]) : pack_bf16x2(o[(2 * i) % W], o[(2 * i + 1) % W]);
    if (n >= W) {
        u32x4_t v = {w[0], w[1], w[2], w[3]};
        __builtin_memcpy(p, &v, 16);
        hold_store_data(v);
        return;
    }
    constexpr int PW = 4 / (int)sizeof(T);       // elements of a word
    const int words = n / PW;
    if (words & 2) {
        const uint2 v = make_uint2(w[0], w[1]);
        __builtin_memcpy(p, &v, 8);
    }
    if (words & 1) {
        const uint32_t v = words & 2 ? w[2] : w[0];
        __builtin_memcpy(p + (words & 2) * PW, &v, 4);
    }
    if (PW == 2 && (n & 1)) {
        const uint32_t v = words & 2 ? (words & 1 ? w[3] : w[2]) : (words & 1 ? w[1] : w[0]);
        const uint16_t lo = (uint16_t)v;
        __builtin_memcpy(p + words * PW, &lo, 2);
    }
}

// A slot of a head is a piece.  Halves (ADJ false): up to W pairs, at j and at pairs + j, then the elements behind the turned ones, up
// to the next multiple of W and on in whole pieces.  Adjacent: W elements of the head, W / 2 pairs, those from `pairs` on as they are.
template <int W> __host__ __device__ inline int tail_pieces_at(int pairs) { return 2 * pairs / W * W; }

template <typename T, bool ADJ>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int slots, int tb, int ttiles, int slices)
{
    constexpr int W = 16 / (int)sizeof(T), NP = ADJ ? W / 2 : W;
    uint32_t blk = blockIdx.x;
    const int slice = (int)(blk % (uint32_t)slices); blk /= (uint32_t)slices;
    const int tt = (int)(blk % (uint32_t)ttiles), b = (int)(blk / (uint32_t)ttiles);
    const int slot = threadIdx.x % slots, rest = threadIdx.x / slots, t = tt * tb + rest % tb, hg = rest / tb, hgs = 256 / (slots * tb);
    if (hg >= hgs || t >= a.Tq) return;

    const int j0 = slot * NP, turned = (a.pairs + NP - 1) / NP;  // first pair; slots that have pairs
    const bool turn = slot < turned;
    const int whole = tail_pieces_at<W>(a.pairs), tail = whole + (slot - turned) * W;
    const int e0 = ADJ ? slot * W : turn ? j0 : max(tail, 2 * a.pairs);
    const int n = ADJ ? W : turn ? min(W, a.pairs - j0) : tail + W - e0;
    float cs[NP], sn[NP];
    if (turn) {
        int at[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) at[x] = x < a.n_axes ? a.pos[((size_t)x * a.B + b) * a.Tq + t] : 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int j = min(j0 + i, a.pairs - 1);
            const int p = j < a.end[0] ? at[0] : j < a.end[1] ? at[1] : j < a.end[2] ? at[2] : at[3];
            const double turns = (double)p * (double)a.freq[j] * 0.15915494309189533577;      // 1 / (2 pi)
            sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
            sn[i] *= a.sign;
        }
    }
    // the heads of this slice: queries' L * H, then keys' L * H_kv (of one batch row)
    const int nq = a.Q ? a.L * a.H : 0, nk = a.K ? a.L * a.Hkv : 0, heads = nq + nk;
    const int h0 = (int)((int64_t)heads * slice / slices), h1 = (int)((int64_t)heads * (slice + 1) / slices);
    for (int r = h0 + hg; r < h1; r += hgs) {
        const bool q = r < nq;
        const int k = q ? r : r - nq, H = q ? a.H : a.Hkv, l = k / H, h = k - l * H;
        const size_t off = ((((size_t)l * a.B + b) * H + h) * a.Tq + t) * a.d + e0;
        const T *x = static_cast<const T *>(q ? a.Q : a.K) + off;
        T *y = static_cast<T *>(q ? a.Qo : a.Ko) + off;
        const T *end = static_cast<const T *>(q ? a.Q : a.K) + (size_t)a.L * a.B * H * a.Tq * a.d;
        float u[W], v[W];
        get_piece<T, W>(x, n, end, u);
        if (!turn) {
            put_piece<T, W>(y, n, u);
            continue;
        }
        float p[W];
        if constexpr (ADJ) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const bool in = j0 + i < a.pairs;                // (the others may be anything, and stay as they are)
                p[2 * i] = in ? u[2 * i] * cs[i] - u[2 * i + 1] * sn[i] : u[2 * i];
                p[2 * i + 1] = in ? u[2 * i] * sn[i] + u[2 * i + 1] * cs[i] : u[2 * i + 1];
            }
            put_piece<T, W>(y, n, p);
        } else {
            get_piece<T, W>(x + a.pairs, n, end, v);
            float m[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                p[i] = u[i] * cs[i] - v[i] * sn[i];
                m[i] = u[i] * sn[i] + v[i] * cs[i];
            }
            put_piece<T, W>(y, n, p);
            put_piece<T, W>(y + a.pairs, n, m);
        }
    }
}

template <typename T>
static hipError_t launch_rotary_as(const RotaryArgs &a, hipStream_t st)
{
    constexpr int W = 16 / (int)sizeof(T);
    const int slots = a.adjacent ? a.d / W : (a.pairs + W - 1) / W + (a.d - tail_pieces_at<W>(a.pairs)) / W;        // (at most 33)
    // a workgroup takes up to 32 tokens; what is left of its threads takes heads side by side
    int tb = 1;
    while (tb < 32 && tb < a.Tq && tb * 2 * slots <= 256) tb *= 2;
    const int ttiles = (a.Tq + tb - 1) / tb, hgs = 256 / (slots * tb);
    const int64_t heads = (a.Q ? (int64_t)a.L * a.H : 0) + (a.K ? (int64_t)a.L * a.Hkv : 0);
    // slices of the heads: enough workgroups for the chip (and for a token's sines and cosines to be made seldom), and no more than
    // one pass each
    int64_t slices = (heads + hgs - 1) / hgs;
    const int64_t want = (2048 + (int64_t)a.B * ttiles - 1) / ((int64_t)a.B * ttiles);
    slices = slices < want ? slices : want;
    if (slices < 1) slices = 1;
    const int64_t blocks = (int64_t)a.B * ttiles * slices;
    const dim3 grid((unsigned)blocks), block(256);
    if (a.adjacent) hipLaunchKernelGGL((rotary_kernel<T, true>), grid, block, 0, st, a, slots, tb, ttiles, (int)slices);
    else hipLaunchKernelGGL((rotary_kernel<T, false>), grid, block, 0, st, a, slots, tb, ttiles, (int)slices);
    return hipGetLastError();
}

hipError_t launch_rotary(const RotaryArgs &a, int dtype, hipStream_t st)
{
    return dtype == KVEV_F32 ? launch_rotary_as<float>(a, st) : launch_rotary_as<bf16_t>(a, st);
}

}  // namespace kvev
