// Rotary positions of tokens that have several coordinates (time, height, width): pair j of a head's elements is turned by the
// angle pos[axis of j] * freq[j].
//
// The angle is taken in double: a 31-bit position times a 24-bit frequency is 55 bits, and the turns that are thrown away are
// most of them for far tokens.  What is left of a turn goes to sine and cosine in fp32 (an error of 2^-25 turns).  They depend on
// the token and not on the head, so a thread makes those of its pairs once and takes them through the heads of its slice;
// queries and keys of one call are one list of heads.  Bytes bound it, sine and cosine where a token has few heads.
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

// W elements at a time.  halves: a slot is W pairs, at j and at pairs + j; adjacent: W / 2 pairs in W elements (W = 1: one pair);
// the slots behind the turned elements copy W of them.
template <typename T, int W, bool ADJ>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int slots, int tb, int ttiles, int slices)
{
    constexpr int NP = ADJ ? (W > 1 ? W / 2 : 1) : W;            // pairs of a slot
    constexpr int STEP = ADJ && W == 1 ? 2 : W;                  // elements of a slot's first load
    uint32_t blk = blockIdx.x;
    const int slice = (int)(blk % (uint32_t)slices); blk /= (uint32_t)slices;
    const int tt = (int)(blk % (uint32_t)ttiles), b = (int)(blk / (uint32_t)ttiles);
    const int slot = threadIdx.x % slots, rest = threadIdx.x / slots, t = tt * tb + rest % tb, hg = rest / tb, hgs = 256 / (slots * tb);
    if (hg >= hgs || t >= a.Tq) return;

    const int turned = a.pairs / NP;                             // slots that are turned
    const bool turn = slot < turned;
    const int e0 = turn ? slot * STEP : 2 * a.pairs + (slot - turned) * W, e1 = e0 + a.pairs;
    float cs[NP], sn[NP];
    if (turn) {
        int at[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) at[x] = x < a.n_axes ? a.pos[((size_t)x * a.B + b) * a.Tq + t] : 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int j = slot * NP + i;
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
        const size_t off = ((((size_t)l * a.B + b) * H + h) * a.Tq + t) * a.d;
        const T *x = static_cast<const T *>(q ? a.Q : a.K) + off;
        T *y = static_cast<T *>(q ? a.Qo : a.Ko) + off;
        if constexpr (W == 1) {
            if (turn) {
                const int f1 = ADJ ? e0 + 1 : e1;
                const float u = Storage<T>::load(x + e0), v = Storage<T>::load(x + f1);
                Storage<T>::store(y + e0, u * cs[0] - v * sn[0]);
                Storage<T>::store(y + f1, u * sn[0] + v * cs[0]);
            } else {
                y[e0] = x[e0];
            }
        } else {
            constexpr int N4 = W * (int)sizeof(T) / 16;          // 16-byte pieces (one)
            static_assert(N4 == 1, "a slot's load is 16 bytes");
            const u32x4_t raw = *reinterpret_cast<const u32x4_t *>(x + e0);
            if (!turn) {
                *reinterpret_cast<u32x4_t *>(y + e0) = raw;
                hold_store_data(raw);
                continue;
            }
            auto get = [](const u32x4_t &w, float (&o)[W]) {
#pragma unroll
                for (int i = 0; i < W; ++i)
                    o[i] = sizeof(T) == 4 ? __uint_as_float(w[i % 4]) : __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
            };
            auto put = [](T *p, const float (&o)[W]) {
                u32x4_t w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(o[i]) : pack_bf16x2(o[(2 * i) % W], o[(2 * i + 1) % W]);
                *reinterpret_cast<u32x4_t *>(p) = w;
                hold_store_data(w);
            };
            float u[W], v[W];
            get(raw, u);
            if constexpr (ADJ) {
#pragma unroll
                for (int i = 0; i < W / 2; ++i) {
                    v[2 * i] = u[2 * i] * cs[i] - u[2 * i + 1] * sn[i];
                    v[2 * i + 1] = u[2 * i] * sn[i] + u[2 * i + 1] * cs[i];
                }
                put(y + e0, v);
            } else {
                get(*reinterpret_cast<const u32x4_t *>(x + e1), v);
                float p[W], m[W];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    p[i] = u[i] * cs[i] - v[i] * sn[i];
                    m[i] = u[i] * sn[i] + v[i] * cs[i];
                }
                put(y + e0, p);
                put(y + e1, m);
            }
        }
    }
}

template <typename T>
static hipError_t launch_rotary_as(const RotaryArgs &a, hipStream_t st)
{
    constexpr int W = 16 / (int)sizeof(T);
    const bool vec = a.adjacent ? 2 * a.pairs % W == 0 : a.pairs % W == 0;
    const int w = vec ? W : 1, np = a.adjacent ? (vec ? W / 2 : 1) : w;
    const int slots = a.pairs / np + (a.d - 2 * a.pairs) / w;    // (at most d = 128)
    // a workgroup takes up to 32 tokens; what is left of its threads takes heads side by side
    int tb = 1;
    while (tb < 32 && tb < a.Tq && tb * 2 * slots <= 256) tb *= 2;
    const int ttiles = (a.Tq + tb - 1) / tb, hgs = 256 / (slots * tb);
    const int64_t heads = (a.Q ? (int64_t)a.L * a.H : 0) + (a.K ? (int64_t)a.L * a.Hkv : 0);
    // slices of the heads: enough workgroups for the chip, and no more than one pass each
    int64_t slices = (heads + hgs - 1) / hgs;
    const int64_t want = (2048 + (int64_t)a.B * ttiles - 1) / ((int64_t)a.B * ttiles);
    slices = slices < want ? slices : want;
    if (slices < 1) slices = 1;
    const int64_t blocks = (int64_t)a.B * ttiles * slices;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(256);
#define KVEV_ROT(WW, ADJ) hipLaunchKernelGGL((rotary_kernel<T, WW, ADJ>), grid, block, 0, st, a, slots, tb, ttiles, (int)slices)
    if (vec) { if (a.adjacent) KVEV_ROT(W, true); else KVEV_ROT(W, false); }
    else { if (a.adjacent) KVEV_ROT(1, true); else KVEV_ROT(1, false); }
#undef KVEV_ROT
    return hipGetLastError();
}

hipError_t launch_rotary(const RotaryArgs &a, int dtype, hipStream_t st)
{
    return dtype == KVEV_F32 ? launch_rotary_as<float>(a, st) : launch_rotary_as<bf16_t>(a, st);
}

}  // namespace kvev
