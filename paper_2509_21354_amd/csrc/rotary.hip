// Rotary positions of tokens that have several coordinates (time, height, width): pair j of a head's elements is turned by the
// angle pos[axis of j] * freq[j].
//
// The angle is taken in double: a 31-bit position times a 24-bit frequency is 55 bits, and the turns that are thrown away are
// most of them for far tokens.  What is left of a turn, half of one at most, goes to sine and cosine in fp32 (rounded by 2^-26 of a turn at most,
// 9.4e-8 of the angle).  They depend on
// the token and not on the head, so a thread makes those of its pairs once and takes them through the heads of its slice;
// queries and keys of one call are one list of heads.  Bytes bound it, sine and cosine where a token has few heads: 64 rows x 256
// tokens x (32 + 8) heads, bf16, d = 128: 65 - 71 us, 4.7 - 5.2 TB/s in and out, what a copy of that size reaches.  Where the pairs of
// halves are no multiple of a piece: 4 x 1000 x 64 heads, 61 pairs 28.6 us (neighbouring pairs 23.5); 14 layers x 919 x 64 heads, 17 pairs
// 102 us, 4.1 TB/s.  (Written from where each half begins, with ends in 8, 4 and 2 bytes: 31 and 138; element by element 51 and 204;
// reads behind branches: 66 and 365.)  Tried and dropped: non-temporal accesses (no difference).
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

// A piece of 16 bytes (W elements), wherever it begins: memory takes such accesses at any element.
template <typename T, int W> __device__ __forceinline__ void get_piece(const T *p, float (&o)[W])
{
    u32x4_t w;
    __builtin_memcpy(&w, p, 16);
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = sizeof(T) == 4 ? __uint_as_float(w[i % 4]) : __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}
template <typename T, int W> __device__ __forceinline__ void put_piece(T *p, const float (&o)[W])
{
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(o[i]) : pack_bf16x2(o[(2 * i) % W], o[(2 * i + 1) % W]);
    __builtin_memcpy(p, &w, 16);
    hold_store_data(w);
}

// A slot of a head is a piece.
//   kWhole     halves whose pairs are whole pieces: W pairs, at j and at pairs + j; then the elements behind the turned ones
//   kAdjacent  neighbours: W elements, W / 2 pairs, those from `pairs` on as they are
//   kAny       halves of any number of pairs: W elements of the output, aligned, from the same of the input and those `pairs` further on
//              and back.  A head's slots lie in one wave, which has read all of it before it writes: it may be turned in place
enum { kWhole, kAdjacent, kAny };
template <typename T, int MODE>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int slots, int tb, int ttiles, int slices)
{
    constexpr int W = 16 / (int)sizeof(T), NP = MODE == kAdjacent ? W / 2 : W;
    uint32_t blk = blockIdx.x;
    const int slice = (int)(blk % (uint32_t)slices); blk /= (uint32_t)slices;
    const int tt = (int)(blk % (uint32_t)ttiles), b = (int)(blk / (uint32_t)ttiles);
    const int slot = threadIdx.x % slots, rest = threadIdx.x / slots, t = tt * tb + rest % tb, hg = rest / tb, hgs = 256 / (slots * tb);
    if (hg >= hgs || t >= a.Tq) return;

    const int P = a.pairs, j0 = slot * NP;       // first pair (kAny: first element)
    const bool turn = j0 < (MODE == kAny ? 2 * P : P);
    const int e0 = MODE == kWhole && !turn ? 2 * P + (j0 - P) : slot * W;
    float cs[NP], sn[NP];
    if (turn) {
        int at[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) at[x] = x < a.n_axes ? a.pos[((size_t)x * a.B + b) * a.Tq + t] : 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const bool second = MODE == kAny && j0 + i >= P;     // (of the pair's elements)
            const int j = min(j0 + i - (second ? P : 0), P - 1);
            const int p = j < a.end[0] ? at[0] : j < a.end[1] ? at[1] : j < a.end[2] ? at[2] : at[3];
            const double turns = (double)p * (double)a.freq[j] * 0.15915494309189533577;      // 1 / (2 pi)
            sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
            sn[i] *= MODE == kAny && !second ? -a.sign : a.sign;
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
        float u[W], v[W], p[W];
        if constexpr (MODE == kAny) {
            // the other elements of the pairs: P further on for elements below P, P back for those from there on (both, where the piece
            // holds P); not read whole where that would pass the tensor's ends
            const size_t all = (size_t)a.L * a.B * H * a.Tq * a.d;
            const bool on = e0 < P, back = turn && e0 + W > P, on_all = all - off >= (size_t)(P + W), back_all = off >= (size_t)P;
            float w[W];
            get_piece<T, W>(x, u);
            get_piece<T, W>(on && on_all ? x + P : x, v);
            get_piece<T, W>(back && back_all ? x - P : x, w);
            if (on && !on_all) {
#pragma unroll
                for (int i = 0; i < W; ++i) v[i] = e0 + i < P ? Storage<T>::load(x + P + i) : 0.f;
            }
            if (back && !back_all) {
#pragma unroll
                for (int i = 0; i < W; ++i) w[i] = e0 + i >= P ? Storage<T>::load(x + i - P) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int e = e0 + i;
                p[i] = e < 2 * P ? u[i] * cs[i] + (e < P ? v[i] : w[i]) * sn[i] : u[i];
            }
            asm volatile("" ::: "memory");      // (every lane has read)
            __builtin_amdgcn_wave_barrier();
            put_piece<T, W>(y, p);
            continue;
        }
        get_piece<T, W>(x, u);
        if (!turn) {
            put_piece<T, W>(y, u);
        } else if constexpr (MODE == kAdjacent) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const bool in = j0 + i < P;                      // (the others may be anything, and stay as they are)
                p[2 * i] = in ? u[2 * i] * cs[i] - u[2 * i + 1] * sn[i] : u[2 * i];
                p[2 * i + 1] = in ? u[2 * i] * sn[i] + u[2 * i + 1] * cs[i] : u[2 * i + 1];
            }
            put_piece<T, W>(y, p);
        } else {
            get_piece<T, W>(x + P, v);
            float m[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                p[i] = u[i] * cs[i] - v[i] * sn[i];
                m[i] = u[i] * sn[i] + v[i] * cs[i];
            }
            put_piece<T, W>(y, p);
            put_piece<T, W>(y + P, m);
        }
    }
}

template <typename T, int MODE>
static hipError_t launch_rotary_mode(const RotaryArgs &a, int slots, hipStream_t st)
{
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
    hipLaunchKernelGGL((rotary_kernel<T, MODE>), dim3((unsigned)blocks), dim3(256), 0, st, a, slots, tb, ttiles, (int)slices);
    return hipGetLastError();
}
template <typename T> static hipError_t launch_rotary_as(const RotaryArgs &a, hipStream_t st)
{
    constexpr int W = 16 / (int)sizeof(T);       // (slots: 8, 16 or 32, fewer for whole halves)
    if (a.adjacent) return launch_rotary_mode<T, kAdjacent>(a, a.d / W, st);
    return a.pairs % W ? launch_rotary_mode<T, kAny>(a, a.d / W, st) : launch_rotary_mode<T, kWhole>(a, a.d / W - a.pairs / W, st);
}

hipError_t launch_rotary(const RotaryArgs &a, int dtype, hipStream_t st)
{
    return dtype == KVEV_F32 ? launch_rotary_as<float>(a, st) : launch_rotary_as<bf16_t>(a, st);
}

}  // namespace kvev
