// Rows into and out of the paged 4-bit cache (format: pages.hpp).
//
// Append: a lane takes 8 elements of a key and the 8 of the value at the same place, four lanes share a block of 32.  The
// block's largest magnitude (as a bit pattern: an infinity or NaN is then simply the largest) is found by two exchanges within
// the four lanes; the codes are rounded by the hardware conversion (to nearest, ties to even; division by a power of two is
// exact), so a row read back is the same bits on every path.  Read: a word of codes and a scale byte per lane.
// Both move bytes and little else: 2 d elements in, d + d / 16 bytes out per token and head, or back.
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

// token (l, b, h, t) of a launch's rows, its place in the pool, and whether it has one
struct Place { unsigned char *group; int row; bool ok; };

__device__ __forceinline__ Place place_of(const PageRowsArgs &a, size_t r)
{
    const PageGeom &g = a.g;
    const uint32_t lbh = (uint32_t)(r / (uint32_t)a.Tn);
    const int t = (int)(r - (size_t)lbh * (uint32_t)a.Tn);
    const uint32_t lb = lbh / (uint32_t)g.Hkv;
    const int h = (int)(lbh - lb * (uint32_t)g.Hkv), l = (int)(lb / (uint32_t)g.B), b = (int)(lb - (uint32_t)l * (uint32_t)g.B);
    const int start = a.start[b], n = a.n_new ? a.n_new[b] : a.Tn;
    const int cap = g.max_pages << g.page_shift;
    Place p{nullptr, 0, false};
    if (t >= n || start < 0 || t >= cap - start) return p;
    const int at = start + t, page = a.table[(size_t)b * g.max_pages + (at >> g.page_shift)];
    p.ok = true;
    if ((uint32_t)page >= (uint32_t)g.n_pages) return p;                  // (no page: group stays null)
    const int in = at & ((1 << g.page_shift) - 1);
    p.group = a.pool + (((size_t)l * g.n_pages + page) * g.Hkv + h) * block_bytes(g) + (size_t)(in / kGroup) * group_bytes(g.d);
    p.row = in % kGroup;
    return p;
}

#ifdef __HIP_DEVICE_COMPILE__
// the largest of four lanes' values
__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kQuadXor1, 0xf, 0xf, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kQuadXor2, 0xf, 0xf, true));
}

__device__ __forceinline__ uint32_t encode(const bf16_t *p, uint32_t &s)
{
    const u32x4_t v = *reinterpret_cast<const u32x4_t *>(p);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(max(top, (v[i] << 16) & 0x7FFFFFFFu), v[i] & 0x7FFF0000u);
    s = scale_byte(quad_max(top));
    if (s == kNanScale) return 0;
    const float f = scale_of(s);
    const uint32_t w[4] = {v[0], v[1], v[2], v[3]};              // (a bit cast of a vector's element takes the first one)
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[0]), f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[1]), f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[2]), f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[3]), f, 3);
}
__device__ __forceinline__ uint32_t encode(const float *p, uint32_t &s)
{
    float v[8];
    VecLoad<float, 8>::run(p, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    s = scale_byte(quad_max(top));
    if (s == kNanScale) return 0;
    const float f = scale_of(s);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], f, 3);
}

__device__ __forceinline__ void decode(bf16_t *p, uint32_t codes, uint32_t s)
{
    const u32x4_t v = __builtin_bit_cast(u32x4_t, unpack8(codes, scale_of(s)));
    *reinterpret_cast<u32x4_t *>(p) = v;
    hold_store_data(v);
}
__device__ __forceinline__ void decode(float *p, uint32_t codes, uint32_t s)
{
    const u32x4_t v = __builtin_bit_cast(u32x4_t, unpack8(codes, scale_of(s)));
    const u32x4_t x = {v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u}, y = {v[2] << 16, v[2] & 0xFFFF0000u, v[3] << 16, v[3] & 0xFFFF0000u};
    reinterpret_cast<u32x4_t *>(p)[0] = x;
    reinterpret_cast<u32x4_t *>(p)[1] = y;
    hold_store_data(x);
    hold_store_data(y);
}
#endif

template <typename T, int D>
__global__ __launch_bounds__(256) void page_append_kernel(PageRowsArgs a, size_t rows)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = D / 8, RPB = 256 / LPR;                  // lanes of a row, rows of a workgroup
    const int e = threadIdx.x % LPR;
    const size_t r = (size_t)blockIdx.x * RPB + threadIdx.x / LPR;
    if (r >= rows) return;
    const Place p = place_of(a, r);
    if (!p.group) return;
    uint32_t sk, sv;
    const uint32_t ck = encode(static_cast<const T *>(a.K) + r * D + e * 8, sk), cv = encode(static_cast<const T *>(a.V) + r * D + e * 8, sv);
    uint32_t *codes = reinterpret_cast<uint32_t *>(p.group) + p.row * LPR + e;
    codes[0] = ck;
    codes[2 * D] = cv;
    if (e % 4 == 0) reinterpret_cast<uint16_t *>(p.group + 16 * D)[p.row * (D / 32) + e / 4] = (uint16_t)(sk | sv << 8);
#endif
}

template <typename T, int D>
__global__ __launch_bounds__(256) void page_read_kernel(PageRowsArgs a, size_t rows)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = D / 8, RPB = 256 / LPR;
    const int e = threadIdx.x % LPR;
    const size_t r = (size_t)blockIdx.x * RPB + threadIdx.x / LPR;
    if (r >= rows) return;
    const Place p = place_of(a, r);
    if (!p.ok) return;
    uint32_t ck = 0, cv = 0, s = 0x7F7F;
    if (p.group) {
        const uint32_t *codes = reinterpret_cast<const uint32_t *>(p.group) + p.row * LPR + e;
        ck = codes[0];
        cv = codes[2 * D];
        s = reinterpret_cast<const uint16_t *>(p.group + 16 * D)[p.row * (D / 32) + e / 4];
    }
    decode(static_cast<T *>(a.Ko) + r * D + e * 8, ck, s & 255u);
    decode(static_cast<T *>(a.Vo) + r * D + e * 8, cv, s >> 8);
#endif
}

#define KVEV_ROWS_LAUNCH(kernel)                                                                                              \
    const size_t rows = (size_t)a.g.L * a.g.B * a.g.Hkv * a.Tn;                                                               \
    const size_t per = 256 / (a.g.d / 8);                                                                                     \
    const dim3 grid((unsigned)((rows + per - 1) / per)), block(256);                                                          \
    if (dtype == KVEV_F32) {                                                                                                  \
        if (a.g.d == 128) hipLaunchKernelGGL((kernel<float, 128>), grid, block, 0, st, a, rows);                              \
        else hipLaunchKernelGGL((kernel<float, 64>), grid, block, 0, st, a, rows);                                            \
    } else {                                                                                                                  \
        if (a.g.d == 128) hipLaunchKernelGGL((kernel<bf16_t, 128>), grid, block, 0, st, a, rows);                             \
        else hipLaunchKernelGGL((kernel<bf16_t, 64>), grid, block, 0, st, a, rows);                                           \
    }                                                                                                                         \
    return hipGetLastError();

hipError_t launch_page_append(const PageRowsArgs &a, int dtype, hipStream_t st) { KVEV_ROWS_LAUNCH(page_append_kernel) }
hipError_t launch_page_read(const PageRowsArgs &a, int dtype, hipStream_t st) { KVEV_ROWS_LAUNCH(page_read_kernel) }

}  // namespace kvev
