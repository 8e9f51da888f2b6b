// The paged 4-bit cache: its format on the device, and the launch interface of the kernels that work on it.
//
// A pool is [L][n_pages][H_kv] blocks of page * 17 d / 16 bytes.  A block holds the keys and values of `page` consecutive
// tokens of one key-value head in groups of 16 tokens, 17 d bytes each:
//   8 d bytes   codes of the keys, token after token (d / 2 bytes each, the element of lower index in the low half)
//   8 d bytes   codes of the values
//     d bytes   scale bytes [16 tokens][d / 32 blocks][key, value]
// so that what a wave reads of 16 tokens is one contiguous piece, whatever the page's length.  A block of 32 elements along d
// shares the scale 2^(s - 127); s = 255 marks a block that held a value that is not finite, and reads as NaN.  Codes are E2M1
// (sign, two bits of exponent, one of mantissa: 0, .5, 1, 1.5, 2, 3, 4, 6), which gfx950 converts with a scale in hardware.
// Scale bytes are 2 to 252 otherwise: every value is then zero or a normal number in bf16, and exact in it.
#pragma once
#include "common.hpp"

namespace kvev {

struct PageGeom {
    int L, B, Hkv, d;
    int page_shift;               // log2 of the tokens of a page
    int n_pages, max_pages;
};

struct RotaryArgs {
    const void *Q, *K;
    void *Qo, *Ko;
    const float *freq;
    const int32_t *pos;           // [n_axes][B][Tq]
    int L, B, H, Hkv, d, Tq;
    int n_axes, end[4];           // end[a]: first pair behind axis a's
    int pairs;                    // pairs of elements that are turned
    int adjacent;                 // 1: pair j is elements 2 j, 2 j + 1; 0: j and j + pairs
    float sign;                   // -1 turns back
};

struct PageRowsArgs {
    PageGeom g;
    const void *K, *V;            // append: new rows [L][B][Hkv][Tn][d]
    void *Ko, *Vo;                // read: the same layout
    unsigned char *pool;
    const int32_t *table, *start, *n_new;
    int Tn;
};

struct PageAttnArgs {
    PageGeom g;
    const void *Q;
    void *O;
    const unsigned char *pool;
    const int32_t *table, *length, *first, *q_start;    // first, q_start: may be null
    const void *Kc, *Vc;
    const int32_t *count;         // null: no store
    int k_cap;
    int G, Tq;
    int nsplit;                   // most workgroups that share a unit's rows
    int qtiles;                   // units per key-value head: its queries in tiles
    int run;                      // chunks of 64 rows for a workgroup (more where rows are longer than planned for)
    float *part;                  // [unit's queries][nsplit][d + 2]
    int32_t *tickets;             // one per unit, zero between calls
    int stream;                   // 1: more than the memory-side cache holds is read: loads carry the non-temporal hint
    float scale_log2e;
};

struct PagesArgs {
    PageGeom g;
    int32_t *table, *length, *refs, *status;
    const int32_t *n_new;         // reserve
    int32_t *start;
    unsigned char *pool;
    int32_t *ws;
    const int32_t *src, *dst;     // fork, copy; trim: src = rows
    const int32_t *first, *keep;  // trim
    int n;
    unsigned char *to_pool;       // compact
    int32_t *to_table, *to_refs;
    int to_pages;
    int stream;                   // compact: as in PageAttnArgs
};

hipError_t launch_rotary(const RotaryArgs &a, int dtype, hipStream_t st);
hipError_t launch_page_append(const PageRowsArgs &a, int dtype, hipStream_t st);
hipError_t launch_page_read(const PageRowsArgs &a, int dtype, hipStream_t st);
hipError_t launch_page_attention(const PageAttnArgs &a, int dtype, int queries, int waves, hipStream_t st);       // waves of a workgroup: 1, 4 or 8
hipError_t launch_page_frame(const PageAttnArgs &a, int queries, hipStream_t st);      // bf16; queries per unit: 128 or 256
hipError_t launch_pages_reserve(const PagesArgs &a, hipStream_t st);
hipError_t launch_pages_fork(const PagesArgs &a, hipStream_t st);
hipError_t launch_pages_trim(const PagesArgs &a, hipStream_t st);
hipError_t launch_pages_copy(const PagesArgs &a, hipStream_t st);
hipError_t launch_pages_compact(const PagesArgs &a, hipStream_t st);

constexpr int kGroup = 16;                                                // tokens of a group
__host__ __device__ constexpr int group_bytes(int d) { return 17 * d; }
__host__ __device__ inline size_t block_bytes(const PageGeom &g) { return (size_t)(1 << g.page_shift) / kGroup * group_bytes(g.d); }
// bytes of one page of one layer, all key-value heads
__host__ __device__ inline size_t page_bytes(const PageGeom &g) { return (size_t)g.Hkv * block_bytes(g); }
// int32 words of scratch: what a row needs and where it begins in the list of pages found, rows to copy (from, to, groups), their
// number; the list
__host__ __device__ inline size_t reserve_words(const PageGeom &g) { return 64 + (size_t)5 * g.B + g.n_pages; }
// a head; places of all pages; the pages in use
__host__ __device__ inline size_t compact_words(const PageGeom &g) { return 64 + 2 * (size_t)g.n_pages; }

#ifdef __HIP_DEVICE_COMPILE__
// A softmax's running maximum is a reference that weights are taken against, and stays while no score is more than kSlack above it
// (in powers of two): what was summed is scaled seldom, weights reach 256, and no rounding depends on it but the fp32 exponent's.
constexpr float kSlack = 8.0f;
constexpr uint32_t kNanScale = 255;
constexpr uint32_t kInfBits = 0x7F800000u;

// the power of two of a scale byte as a float (the conversion takes its exponent alone, and 255 as not-a-number)
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

// Scale byte of a block from the bit pattern of its largest magnitude: the smallest power of two with which that rounds to 6 at
// most, i.e. top <= 7 * 2^(s - 127).  Every element is then off by half a step of its code at most.  (6 * 2^126 is past the largest
// number, so 2^125 is the largest scale; codes end at 6.)
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits)
{
    const int s = (int)((top_bits + 0x1FFFFFu) >> 23) - 2;     // 4 * 1.75 = 7: one more when the mantissa is above .75
    return top_bits >= kInfBits ? kNanScale : (uint32_t)min(max(s, 2), 252);
}

// 8 codes (one word) -> 8 bf16
__device__ __forceinline__ bf16x8_t unpack8(uint32_t codes, float scale)
{
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return __builtin_bit_cast(bf16x8_t, r);
}
#endif

}  // namespace kvev
