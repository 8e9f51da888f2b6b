// Handing out, sharing, freeing and packing the pages of a 4-bit cache.
//
// A page is in use while refs[page] > 0, the number of table entries that name it; there is no list of free pages to keep in
// order.  Whoever needs pages takes the free ones of lowest index, in the order of the rows, so a call's outcome depends on
// nothing but what the arrays held before it.  Atomics are integer additions and exchanges whose order does not show.
// Tables and counts are small (a few bytes per page): those kernels are chains of memory round trips, one workgroup each where
// they have to see all rows (16 rows, 560 pages: reserve 6.1 us, its copies 6.5, fork 3.9, trim 3.9; compaction's ranks of 5 200 pages 8.7).  Copies
// move whole 16-byte pieces at the rate of the memory (compaction of 1.7 GB in and out: 322 us, 5.3 TB/s; copies of 512 pages of 32 layers, 2.3
// GB in and out, 455 us, 5.0, of 8192 pages of one layer 242 us, 4.7; a large copy: 4.9).
#include "kernels.hpp"
#include "pages.hpp"

namespace kvev {

constexpr int kStatusNoPages = 1, kStatusRow = 2, kStatusPair = 4;     // bits of the status word (kvev.h)
// words of the reserve scratch, after a head of 64 (word 0: rows to copy)
enum { kNeed = 0, kAt = 1, kFrom = 2, kTo = 3, kGroups = 4 };
constexpr int kHead = 64;

// exclusive sum over the threads of a workgroup of NT; `total` receives the sum of all
template <int NT> __device__ __forceinline__ int block_scan(int v, int &total)
{
    __shared__ int s_w[NT / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                       // (s_w of a scan before is read)
    if (lane == 63) s_w[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const int y = s_w[w];
        before += w < wave ? y : 0;
        total += y;
    }
    return before + x - v;
}

__device__ __forceinline__ int pages_of(int tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }

// Room for n_new[b] more tokens in every row.
__global__ __launch_bounds__(1024) void reserve_kernel(PagesArgs a)
{
    const PageGeom &g = a.g;
    const int tid = threadIdx.x, shift = g.page_shift, cap = g.max_pages << shift, in_page = (1 << shift) - 1;
    int32_t *rows = a.ws + kHead, *list = rows + (size_t)5 * g.B;
    __shared__ int s_status;
    if (tid == 0) s_status = 0;
    __syncthreads();

    // what every row needs, and where its pages begin in the list of those found
    int total = 0;
    for (int b0 = 0; b0 < g.B; b0 += 1024) {
        const int b = b0 + tid;
        int need = 0;
        if (b < g.B) {
            const int len = a.length[b], n = max(a.n_new[b], 0);
            int from = -1, bad = len < 0 || len > cap || n > cap - len;
            if (!bad && n > 0) {
                need = pages_of(len + n, shift) - pages_of(len, shift);
                if (len & in_page) {       // goes on in a page: in a copy of it if others share it
                    const int page = a.table[(size_t)b * g.max_pages + (len >> shift)];
                    if ((uint32_t)page >= (uint32_t)g.n_pages) bad = 1;
                    else if (a.refs[page] > 1) { from = page; ++need; }
                }
            }
            if (bad) { need = 0; atomicOr(&s_status, kStatusRow); }
            rows[kNeed * g.B + b] = bad ? -1 : need;
            rows[kFrom * g.B + b] = from;
        }
        int sum;
        const int at = block_scan<1024>(need, sum);
        if (b < g.B) rows[kAt * g.B + b] = total + at;
        total += sum;
    }

    // the free pages of lowest index
    int found = 0;
    constexpr int PER = 8;
    for (int64_t p0 = 0; found < total && p0 < g.n_pages; p0 += 1024 * PER) {
        const int64_t p = p0 + tid * PER;
        int free_bits = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (p + i < g.n_pages && a.refs[p + i] == 0) free_bits |= 1 << i;
        int sum, at = block_scan<1024>(__popc(free_bits), sum);
        at += found;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (free_bits >> i & 1) {
                if (at < total) list[at] = (int)p + i;
                ++at;
            }
        found += sum;
    }
    __syncthreads();
    const bool enough = found >= total;

    // tables, counts, lengths; the copies to make
    __shared__ int s_moves;
    if (tid == 0) s_moves = 0;
    __syncthreads();
    const int lane = tid & 63;
    for (int b = tid >> 6; b < g.B; b += 16) {
        const int need = rows[kNeed * g.B + b], len = a.length[b];
        if (need < 0 || !enough) {
            if (lane == 0) a.start[b] = -1;
            continue;
        }
        const int n = max(a.n_new[b], 0), at = rows[kAt * g.B + b], from = rows[kFrom * g.B + b];
        int32_t *row = a.table + (size_t)b * g.max_pages;
        const int cow = from >= 0 ? 1 : 0, have = pages_of(len, shift);
        for (int i = lane; i < need - cow; i += 64) {
            const int page = list[at + cow + i];
            row[have + i] = page;
            a.refs[page] = 1;
        }
        if (lane == 0) {
            if (cow) {
                const int page = list[at], m = atomicAdd(&s_moves, 1);
                row[len >> shift] = page;
                a.refs[page] = 1;
                atomicSub(&a.refs[from], 1);
                // (the copies are made in any order: no page is both read and written)
                rows[kFrom * g.B + b] = -1;
                rows[kTo * g.B + m] = b;
                rows[kGroups * g.B + b] = ((len & in_page) + kGroup - 1) / kGroup;
                rows[kNeed * g.B + b] = from;
                rows[kAt * g.B + b] = page;
            }
            a.length[b] = len + n;
            a.start[b] = len;
        }
    }
    __syncthreads();
    if (tid == 0) {
        a.ws[0] = s_moves;
        const int status = s_status | (enough ? 0 : kStatusNoPages);
        if (status) atomicOr(a.status, status);
    }
}

// 16-byte pieces from one place to another by NT threads, of which this is number i.  STREAM: with the non-temporal hint, for more
// than the caches hold.
template <int NT, bool STREAM> __device__ __forceinline__ void copy_pieces(unsigned char *to, const unsigned char *from, size_t bytes, int i0)
{
    u32x4_t *y = reinterpret_cast<u32x4_t *>(to);
    const u32x4_t *x = reinterpret_cast<const u32x4_t *>(from);
    const int64_t n = (int64_t)(bytes / 16);
    constexpr int U = 4;
    for (int64_t i = i0; i < n; i += NT * U) {
        u32x4_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + NT * u < n) v[u] = STREAM ? __builtin_nontemporal_load(x + i + NT * u) : x[i + NT * u];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + NT * u < n) {
                if (STREAM) __builtin_nontemporal_store(v[u], y + i + NT * u);
                else y[i + NT * u] = v[u];
                hold_store_data(v[u]);
            }
    }
}

// The groups in use of every page that a row shared and goes on in: a wave to a (row, layer, head), since most have a few groups of
// 2 KiB (15 rows x 32 layers x 8 heads, one group each: 9.2 us by a workgroup each).
__global__ __launch_bounds__(256) void reserve_copy_kernel(PagesArgs a)
{
    const PageGeom &g = a.g;
    const int32_t *rows = a.ws + kHead;
    const int64_t units = (int64_t)a.ws[0] * g.L * g.Hkv;
    const size_t block = block_bytes(g);
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
        const int64_t ml = u / g.Hkv;
        const int h = (int)(u - ml * g.Hkv), i = (int)(ml / g.L), l = (int)(ml - (int64_t)i * g.L), b = rows[kTo * g.B + i];
        const size_t from = rows[kNeed * g.B + b], to = rows[kAt * g.B + b], base = (size_t)l * g.n_pages;
        copy_pieces<64, false>(a.pool + ((base + to) * g.Hkv + h) * block, a.pool + ((base + from) * g.Hkv + h) * block,
                               (size_t)rows[kGroups * g.B + b] * group_bytes(g.d), threadIdx.x & 63);
    }
}

// whether value v stands in x[0 .. n), asked by a whole workgroup
__device__ __forceinline__ bool among(const int32_t *x, int n, int v)
{
    int hit = 0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) hit |= x[i] == v;
    return __syncthreads_or(hit);
}

// Row dst[i] becomes a second holder of row src[i]'s pages.
__global__ __launch_bounds__(256) void fork_kernel(PagesArgs a)
{
    const PageGeom &g = a.g;
    const int i = blockIdx.x, src = a.src[i], dst = a.dst[i];
    // what is refused does not depend on the order of the pairs' workgroups: a row is written by the first pair that names it, and
    // read by none that another pair writes
    bool ok = (uint32_t)src < (uint32_t)g.B && (uint32_t)dst < (uint32_t)g.B;
    ok = !among(a.dst, i, dst) && ok;
    ok = !among(a.dst, a.n, src) && ok;
    if (ok && a.length[dst] != 0) ok = false;
    if (!ok) {
        if (threadIdx.x == 0) atomicOr(a.status, kStatusPair);
        return;
    }
    const int32_t *x = a.table + (size_t)src * g.max_pages;
    int32_t *y = a.table + (size_t)dst * g.max_pages;
    for (int j = threadIdx.x; j < g.max_pages; j += 256) {
        const int page = x[j];
        y[j] = page;
        if ((uint32_t)page < (uint32_t)g.n_pages) atomicAdd(&a.refs[page], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) a.length[dst] = a.length[src];
}

// Row rows[i] keeps tokens [first, keep) of what it holds: pages that lie wholly outside are given back.
__global__ __launch_bounds__(256) void trim_kernel(PagesArgs a)
{
    const PageGeom &g = a.g;
    const int i = blockIdx.x, b = a.src ? a.src[i] : i, shift = g.page_shift;
    if ((uint32_t)b >= (uint32_t)g.B) return;
    __shared__ int s_len;
    if (threadIdx.x == 0) {
        const int len = max(a.length[b], 0), keep = a.keep ? min(max(a.keep[i], 0), len) : len;
        s_len = min(min(atomicMin(&a.length[b], keep), keep), g.max_pages << shift);
    }
    __syncthreads();
    const int len = max(s_len, 0), first = a.first ? min(max(a.first[i], 0), len) : 0;
    const int begin = first >> shift, end = pages_of(len, shift);
    int32_t *row = a.table + (size_t)b * g.max_pages;
    for (int j = threadIdx.x; j < g.max_pages; j += 256) {
        if (j >= begin && j < end) continue;
        if (row[j] < 0) continue;
        const int page = atomicExch(&row[j], -1);              // (the row may be given twice: one of them takes the entry)
        if ((uint32_t)page < (uint32_t)g.n_pages) atomicSub(&a.refs[page], 1);
    }
}

// Page dst[i] becomes a copy of page src[i], all layers and heads.
__global__ __launch_bounds__(256) void copy_kernel(PagesArgs a)
{
    const PageGeom &g = a.g;
    const size_t block = block_bytes(g);
    for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
        const int src = a.src[i], dst = a.dst[i];
        bool ok = (uint32_t)src < (uint32_t)g.n_pages && (uint32_t)dst < (uint32_t)g.n_pages;        // (as in fork_kernel)
        ok = !among(a.dst, i, dst) && ok;
        ok = !among(a.dst, a.n, src) && ok;
        if (!ok) {
            if (threadIdx.x == 0) atomicOr(a.status, kStatusPair);
            continue;
        }
        for (int l = blockIdx.y; l < g.L; l += gridDim.y)
            copy_pieces<256, false>(a.pool + ((size_t)l * g.n_pages + dst) * g.Hkv * block, a.pool + ((size_t)l * g.n_pages + src) * g.Hkv * block,
                                    g.Hkv * block, threadIdx.x);
    }
}

// The place of every page in use among those in use (or -1), the pages in use, and the counts in their new order; words 0 and 1 of
// the scratch: whether they fit, and their number.
__global__ __launch_bounds__(1024) void compact_rank_kernel(PagesArgs a)
{
    const PageGeom &g = a.g;
    int32_t *rank = a.ws + kHead, *list = rank + g.n_pages;
    int used = 0;
    constexpr int PER = 8;
    for (int64_t p0 = 0; p0 < g.n_pages; p0 += 1024 * PER) {
        const int64_t p = p0 + (int)threadIdx.x * PER;
        int bits = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (p + i < g.n_pages && a.refs[p + i] > 0) bits |= 1 << i;
        int sum, at = block_scan<1024>(__popc(bits), sum);
        at += used;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (p + i < g.n_pages) {
                const bool in = bits >> i & 1;
                rank[p + i] = in ? at : -1;
                if (in) list[at++] = (int)p + i;
            }
        used += sum;
    }
    __syncthreads();
    const bool fits = used <= a.to_pages;
    if (threadIdx.x == 0) {
        a.ws[0] = fits;
        a.ws[1] = used;
        if (!fits) atomicOr(a.status, kStatusNoPages);
    }
    if (!fits) return;
    for (int p = threadIdx.x; p < g.n_pages; p += 1024)
        if (rank[p] >= 0) a.to_refs[rank[p]] = a.refs[p];
    for (int p = used + threadIdx.x; p < a.to_pages; p += 1024) a.to_refs[p] = 0;
}

// The pages in use in parts of 32 KiB, dealt out evenly: few large pages are enough for the chip, and pages that are free cost nothing
// (1.7 GB in and out 360 -> 318 us, 129 pages of 557 KB 33 -> 27.5; parts of 16 KiB 316 and 27.5, but 11.9 for 9.3 where pages are small).
constexpr size_t kPart = 32768;
template <bool STREAM> __global__ __launch_bounds__(256) void compact_copy_kernel(PagesArgs a)
{
    if (!a.ws[0]) return;
    const PageGeom &g = a.g;
    const int32_t *rank = a.ws + kHead;
    const size_t block = block_bytes(g);
    const int64_t cells = (int64_t)g.B * g.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < cells; i += (int64_t)gridDim.x * 256) {
        const int page = a.table[i];
        a.to_table[i] = (uint32_t)page < (uint32_t)g.n_pages ? rank[page] : -1;
    }
    const int32_t *list = rank + g.n_pages;
    const int used = a.ws[1];
    const size_t bytes = g.Hkv * block, parts = (bytes + kPart - 1) / kPart, units = (size_t)used * g.L * parts;
    for (size_t u = blockIdx.x; u < units; u += gridDim.x) {
        const size_t q = u / parts, at = (u - q * parts) * kPart;
        const int l = (int)(q / (uint32_t)used), to = (int)(q - (size_t)l * used), p = list[to];
        copy_pieces<256, STREAM>(a.to_pool + ((size_t)l * a.to_pages + to) * bytes + at, a.pool + ((size_t)l * g.n_pages + p) * bytes + at,
                                 bytes - at < kPart ? bytes - at : kPart, threadIdx.x);
    }
}

static unsigned grid_of(int64_t units, int64_t most) { return (unsigned)(units < 1 ? 1 : units < most ? units : most); }

hipError_t launch_pages_reserve(const PagesArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(1024), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(reserve_copy_kernel, dim3(grid_of(((int64_t)a.g.B * a.g.L * a.g.Hkv + 3) / 4, 2048)), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_pages_fork(const PagesArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)a.n), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_pages_trim(const PagesArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(trim_kernel, dim3((unsigned)a.n), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_pages_copy(const PagesArgs &a, hipStream_t st)
{
    const unsigned pages = grid_of(a.n, 2048), layers = grid_of(a.g.L, (2048 + pages - 1) / pages);
    hipLaunchKernelGGL(copy_kernel, dim3(pages, layers), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_pages_compact(const PagesArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(compact_rank_kernel, dim3(1), dim3(1024), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t parts = (int64_t)((a.g.Hkv * block_bytes(a.g) + kPart - 1) / kPart);
    const dim3 grid(grid_of((a.g.n_pages < 2048 ? (int64_t)a.g.n_pages * a.g.L : 2048) * parts, 2048));
    if (a.stream) hipLaunchKernelGGL((compact_copy_kernel<true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((compact_copy_kernel<false>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace kvev
