// Rows into and out of the paged 4-bit cache (format: pages.hpp).
//
// Append: a lane takes 8 elements of a key and the 8 of the value at the same place, four lanes share a block of 32.  The
// block's largest magnitude (as a bit pattern: an infinity or NaN is then simply the largest) is found by two exchanges within
// the four lanes; the codes are rounded by the hardware conversion (to nearest, ties to even; division by a power of two is
// exact), so a row read back is the same bits on every path.  Read: a word of codes and a scale byte per lane.
// Both move bytes and little else: 2 d elements in, d + d / 16 bytes out per token and head, or back.  4 rows of 5000 - 8000 tokens x 8 heads, bf16,
// d = 128: 23.3 us in, 22.4 out, 5.8 and 6.0 TB/s (a large copy: 4.9; half of it lies in the memory-side cache).  One token of 64 rows x 8 heads: 2.9
// and 2.6 us, the launch.
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

// A workgroup takes tb tokens of hb heads of one (layer, batch row), tb * hb rows: for a single token, several heads.
struct RowTiles { int log_tb, ttiles, htiles; };

// this thread's row of K and V (as many rows from their beginning), its place in the pool, and whether it is to be moved
struct Place { size_t src; unsigned char *group; int row; bool ok; };

// (u: which of U tiles of tb tokens the workgroup is at)
template <int D, int U> __device__ __forceinline__ Place place_of(const PageRowsArgs &a, const RowTiles &w, int u)
{
    const PageGeom &g = a.g;
    uint32_t x = blockIdx.x;
    const int tt = (int)(x % (uint32_t)w.ttiles) * U + u; x /= (uint32_t)w.ttiles;
    const int ht = (int)(x % (uint32_t)w.htiles), lb = (int)(x / (uint32_t)w.htiles), l = lb / g.B, b = lb - l * g.B;
    const int start = a.start[b], n = min(a.n_new ? a.n_new[b] : a.Tn, a.Tn);
    constexpr int LPR = D / 8, RPB = 256 / LPR;
    const int lr = (int)threadIdx.x / LPR, t = (tt << w.log_tb) + (lr & ((1 << w.log_tb) - 1)), h = ht * (RPB >> w.log_tb) + (lr >> w.log_tb);
    const int cap = g.max_pages << g.page_shift;
    Place p{0, nullptr, 0, false};
    if ((tt << w.log_tb) >= n || start < 0) return p;            // (the whole workgroup)
    if (t >= n || h >= g.Hkv || t >= cap - start) return p;
    const int at = start + t, page = a.table[(size_t)b * g.max_pages + (at >> g.page_shift)];
    p.ok = true;
    p.src = ((size_t)lb * g.Hkv + h) * a.Tn + t;
    if ((uint32_t)page >= (uint32_t)g.n_pages) return p;         // (no page: group stays null)
    const int in = at & ((1 << g.page_shift) - 1);
    p.group = a.pool + (((size_t)l * g.n_pages + page) * g.Hkv + h) * block_bytes(g) + (size_t)(in / kGroup) * group_bytes(D);
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

// 8 elements as loaded, and their codes and the scale byte of their block
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> {
    u32x4_t v;
    __device__ __forceinline__ void load(const bf16_t *p) { v = *reinterpret_cast<const u32x4_t *>(p); }
    __device__ __forceinline__ uint32_t encode(uint32_t &s) const
    {
        const uint32_t w[4] = {v[0], v[1], v[2], v[3]};          // (a bit cast of a vector's element takes the first one)
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(max(top, (w[i] << 16) & 0x7FFFFFFFu), w[i] & 0x7FFF0000u);
        s = scale_byte(quad_max(top));
        if (s == kNanScale) return 0;
        const float f = scale_of(s);
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[0]), f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[1]), f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[2]), f, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_hw_t, w[3]), f, 3);
    }
};
template <> struct Raw8<float> {
    float v[8];
    __device__ __forceinline__ void load(const float *p) { VecLoad<float, 8>::run(p, v); }
    __device__ __forceinline__ uint32_t encode(uint32_t &s) const
    {
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
};

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
__global__ __launch_bounds__(256) void page_append_kernel(PageRowsArgs a, RowTiles w)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = D / 8;                                   // lanes of a row
    const int e = threadIdx.x % LPR;
    const Place p = place_of<D, 1>(a, w, 0);
    if (!p.group) return;
    Raw8<T> k, v;
    k.load(static_cast<const T *>(a.K) + p.src * D + e * 8);
    v.load(static_cast<const T *>(a.V) + p.src * D + e * 8);
    uint32_t sk, sv;
    const uint32_t ck = k.encode(sk), cv = v.encode(sv);
    uint32_t *codes = reinterpret_cast<uint32_t *>(p.group) + p.row * LPR + e;
    codes[0] = ck;
    codes[2 * D] = cv;
    if (e % 4 == 0) reinterpret_cast<uint16_t *>(p.group + 16 * D)[p.row * (D / 32) + e / 4] = (uint16_t)(sk | sv << 8);
#endif
}

template <typename T, int D, int U>
__global__ __launch_bounds__(256) void page_read_kernel(PageRowsArgs a, RowTiles w)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = D / 8;
    const int e = threadIdx.x % LPR;
    Place p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) p[u] = place_of<D, U>(a, w, u);
    uint32_t ck[U], cv[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        ck[u] = cv[u] = 0;
        s[u] = 0x7F7F;
        if (p[u].group) {
            const uint32_t *codes = reinterpret_cast<const uint32_t *>(p[u].group) + p[u].row * LPR + e;
            ck[u] = codes[0];
            cv[u] = codes[2 * D];
            s[u] = reinterpret_cast<const uint16_t *>(p[u].group + 16 * D)[p[u].row * (D / 32) + e / 4];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!p[u].ok) continue;
        decode(static_cast<T *>(a.Ko) + p[u].src * D + e * 8, ck[u], s[u] & 255u);
        decode(static_cast<T *>(a.Vo) + p[u].src * D + e * 8, cv[u], s[u] >> 8);
    }
#endif
}

// Tiles of 16 rows (d = 128; 32 at 64).  A workgroup that reads takes four of them, in flight together, where there are enough for
// the chip even so: 16 rows x 32 layers x 8 heads x 13 of 64 tokens 18.8 and 10.0 us.  (Writing, there is no difference: 32 heads x
// 8000 tokens 22 us.)
static dim3 row_tiles(const PageRowsArgs &a, bool may_four, RowTiles &w, bool &four)
{
    const int rpb = 256 / (a.g.d / 8);
    w = RowTiles{0, 1, 1};
    while (1 << w.log_tb < rpb && 1 << w.log_tb < a.Tn) ++w.log_tb;
    const int64_t tiles = ((int64_t)a.Tn + (1 << w.log_tb) - 1) >> w.log_tb;
    const int hb = rpb >> w.log_tb;
    w.htiles = (a.g.Hkv + hb - 1) / hb;
    const int64_t lbh = (int64_t)a.g.L * a.g.B * w.htiles;
    four = may_four && tiles > 1 && lbh * ((tiles + 3) / 4) >= 1024;
    w.ttiles = (int)(four ? (tiles + 3) / 4 : tiles);
    return dim3((unsigned)(lbh * w.ttiles));
}

template <typename T, int D> static void launch_read_as(const PageRowsArgs &a, hipStream_t st)
{
    RowTiles w;
    bool four;
    const dim3 grid = row_tiles(a, true, w, four);
    if (four) hipLaunchKernelGGL((page_read_kernel<T, D, 4>), grid, dim3(256), 0, st, a, w);
    else hipLaunchKernelGGL((page_read_kernel<T, D, 1>), grid, dim3(256), 0, st, a, w);
}

hipError_t launch_page_append(const PageRowsArgs &a, int dtype, hipStream_t st)
{
    RowTiles w;
    bool four;
    const dim3 grid = row_tiles(a, false, w, four), block(256);
    if (dtype == KVEV_F32) {
        if (a.g.d == 128) hipLaunchKernelGGL((page_append_kernel<float, 128>), grid, block, 0, st, a, w);
        else hipLaunchKernelGGL((page_append_kernel<float, 64>), grid, block, 0, st, a, w);
    } else {
        if (a.g.d == 128) hipLaunchKernelGGL((page_append_kernel<bf16_t, 128>), grid, block, 0, st, a, w);
        else hipLaunchKernelGGL((page_append_kernel<bf16_t, 64>), grid, block, 0, st, a, w);
    }
    return hipGetLastError();
}

hipError_t launch_page_read(const PageRowsArgs &a, int dtype, hipStream_t st)
{
    if (dtype == KVEV_F32) {
        if (a.g.d == 128) launch_read_as<float, 128>(a, st);
        else launch_read_as<float, 64>(a, st);
    } else {
        if (a.g.d == 128) launch_read_as<bf16_t, 128>(a, st);
        else launch_read_as<bf16_t, 64>(a, st);
    }
    return hipGetLastError();
}

}  // namespace kvev
