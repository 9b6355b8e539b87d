// Paged key/value cache: writing new tokens (as given, int8 or e4m3) and reading whole sequences back.
//
// Both are pure data movement (a quantised row is one absolute maximum and one multiplication per element), bound by HBM:
// the floor is the bytes given + the bytes held.  A row is the head_dim elements of one (token, kv head); a lane holds 16 bytes of the
// narrower side (8 elements as given, 16 quantised), so 4 to 16 neighbouring lanes share a row, its maximum is a shuffle over them, and
// both sides move in 16-byte accesses.  A warp takes whole tokens, two neighbouring ones at a time, keys and values of all heads: where a token lies
// (its sequence, searched in shared memory, its page) is found once, by a lane of its own.  A row per group of lanes with a search each spent
// more instructions on finding than on moving (24 prompts written and read back, 674 MB: 155 us, this way 137 us, 4.9 TB/s).
#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kMaxSeqs = 2048;

// Largest i with start[i] <= x (start[0] = 0, so the skipped empty sequences share their successor's start).
__device__ __forceinline__ uint32_t find_seq(const int32_t* start, uint32_t n, int x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) { const uint32_t mid = (lo + hi) >> 1; if (start[mid] <= x) lo = mid; else hi = mid; }
    return lo;
}

// The cell of place `pos` of sequence i for kv head 0 (heads follow a page's tokens apart); -1 (and reported) where its page is not in the pool.
__device__ __forceinline__ int64_t cell_of(const SeqBatch& b, const Pages& p, uint32_t i, int pos, uint32_t* err)
{
    const uint32_t page = uint32_t(__ldg(b.page_table + uint64_t(i) * b.table_stride + (uint32_t(pos) >> p.page_shift)));
    if (page >= p.n_pages) { report(err, bePage); return -1; }
    return (int64_t(page) * p.n_kv_heads << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
}

constexpr int kRun = 2;                  // neighbouring tokens that a warp takes at a time
constexpr int kAhead = 4;                // pieces of a token that a lane has in flight

template <bool BF, int CACHE, int D>
__global__ void __launch_bounds__(kThreads) k_cache_append(SeqBatch b, Pages p, const uint8_t* k, uint64_t k_stride, const uint8_t* v, uint64_t v_stride, uint32_t* err)
{
    using A = Act<BF>;
    constexpr int E = CACHE == WWWS_CACHE_16 ? 8 : 16;   // elements per lane
    constexpr int L = D / E, R = 32 / L;                 // lanes per row, rows per warp
    __shared__ int32_t start[kMaxSeqs + 1];
    for (uint32_t i = threadIdx.x; i <= b.n_seqs; i += kThreads) start[i] = b.q_start[i];
    __syncthreads();
    const uint32_t lane = threadIdx.x % 32, part = lane % L;
    const uint32_t rows = 2 * p.n_kv_heads;              // keys' heads, then values'
    const uint32_t warps = gridDim.x * (kThreads / 32);
    for (uint32_t run = (blockIdx.x * kThreads + threadIdx.x) / 32; run * kRun < b.n_tokens; run += warps) {
        // lane t finds the cell of the run's token t (kv head 0): the searches and lookups of a run wait for memory together
        int64_t mine = -1;
        if (const uint32_t tok = run * kRun + lane; lane < kRun && tok < b.n_tokens) {
            const uint32_t i = find_seq(start, b.n_seqs, int(tok));
            const int q_len = start[i + 1] - start[i], kv = b.kv_len[i], pos = kv - q_len + int(tok) - start[i];
            if (uint32_t(q_len) > b.max_q_len || uint32_t(kv) > b.max_kv_len || start[i] < 0 || start[i] > int(tok) || start[i + 1] <= int(tok)) report(err, beOffset);
            else if (pos >= 0) mine = cell_of(b, p, i, pos, err);
        }
        for (int t = 0; t < kRun; ++t) {
            const int64_t first = __shfl_sync(0xffffffffu, mine, t);
            const uint32_t tok = run * kRun + t;
            if (first < 0) continue;
            for (uint32_t r0 = 0; r0 < rows; r0 += R * kAhead) {
                uint4 x[kAhead][E / 8];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const uint32_t r = r0 + u * R + lane / L;
                    if (r >= rows) continue;
                    const bool val = r >= p.n_kv_heads;
                    const uint32_t h = val ? r - p.n_kv_heads : r;
                    const uint4* g = reinterpret_cast<const uint4*>((val ? v : k) + (uint64_t(tok) * (val ? v_stride : k_stride) + h * D + part * E) * 2);
#pragma unroll
                    for (int e = 0; e < E / 8; ++e) x[u][e] = __ldg(g + e);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const uint32_t r = r0 + u * R + lane / L;
                    const bool on = r < rows, val = r >= p.n_kv_heads;
                    const int64_t cell = first + (int64_t(val ? r - p.n_kv_heads : r) << p.page_shift);
                    uint4* dst = reinterpret_cast<uint4*>(val ? p.v : p.k) + cell * L + part;
                    if constexpr (CACHE == WWWS_CACHE_16) {
                        if (on) *dst = x[u][0];
                    } else {
                        constexpr float kTop = CACHE == WWWS_CACHE_INT8 ? 127.0f : 448.0f;
                        uint32_t w[E / 2];
                        memcpy(w, x[u], sizeof w);
                        // the largest magnitude as bits, two at a time: NaN > infinity > every finite value
                        uint32_t two = 0;
#pragma unroll
                        for (int e = 0; e < E / 2; ++e) asm("max.u16x2 %0, %0, %1;" : "+r"(two) : "r"(w[e] & 0x7fff7fffu));
#pragma unroll
                        for (int m = 1; m < L; m <<= 1) { const uint32_t o = __shfl_xor_sync(0xffffffffu, two, m); asm("max.u16x2 %0, %0, %1;" : "+r"(two) : "r"(o)); }
                        const float top = __uint_as_float(max(__float_as_uint(A::lo(two)), __float_as_uint(A::hi(two))));
                        const bool finite = __float_as_uint(top) < 0x7f800000u;
                        const float scale = !finite ? __uint_as_float(0x7fffffffu) : top < 0x1p-100f ? 0.0f : top * (1.0f / kTop);
                        const float inv = finite && scale > 0.0f ? __fdiv_rn(1.0f, scale) : 0.0f;
                        // No clamp is needed: |x| inv exceeds the top code by a few parts in 2^23 at most, which rounds to it (int8) or saturates (e4m3).
                        uint32_t c[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float y0 = A::lo(w[2 * q]) * inv, y1 = A::hi(w[2 * q]) * inv, y2 = A::lo(w[2 * q + 1]) * inv, y3 = A::hi(w[2 * q + 1]) * inv;
                            if constexpr (CACHE == WWWS_CACHE_INT8) {
                                // 1.5 * 2^23 + y has round-to-even(y) in its low byte
                                constexpr float kShift = 12582912.0f;
                                const uint32_t lo = __byte_perm(__float_as_uint(y0 + kShift), __float_as_uint(y1 + kShift), 0x0040), hi = __byte_perm(__float_as_uint(y2 + kShift), __float_as_uint(y3 + kShift), 0x0040);
                                c[q] = __byte_perm(lo, hi, 0x5410);
                            } else {
                                uint16_t lo, hi;
                                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y1), "f"(y0));
                                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y3), "f"(y2));
                                c[q] = uint32_t(lo) | uint32_t(hi) << 16;
                            }
                            if (!finite) c[q] = 0;
                        }
                        if (on) {
                            *dst = make_uint4(c[0], c[1], c[2], c[3]);
                            if (part == 0) (val ? p.v_scale : p.k_scale)[cell] = scale;
                        }
                    }
                }
            }
        }
    }
}

template <bool BF, int CACHE, int D>
__global__ void __launch_bounds__(kThreads) k_cache_read(SeqBatch b, Pages p, const int32_t* row_start, uint32_t n_rows, uint8_t* k_out, uint8_t* v_out, uint32_t* err)
{
    using A = Act<BF>;
    constexpr int E = CACHE == WWWS_CACHE_16 ? 8 : 16;
    constexpr int L = D / E, R = 32 / L;
    __shared__ int32_t start[kMaxSeqs + 1];
    for (uint32_t i = threadIdx.x; i <= b.n_seqs; i += kThreads) start[i] = row_start[i];
    __syncthreads();
    const uint32_t lane = threadIdx.x % 32, part = lane % L;
    const uint32_t rows = 2 * p.n_kv_heads;
    const uint32_t warps = gridDim.x * (kThreads / 32);
    for (uint32_t run = (blockIdx.x * kThreads + threadIdx.x) / 32; run * kRun < n_rows; run += warps) {
        int64_t mine = -1;
        if (const uint32_t tok = run * kRun + lane; lane < kRun && tok < n_rows) {
            const uint32_t i = find_seq(start, b.n_seqs, int(tok));
            const int pos = int(tok) - start[i], kv = b.kv_len[i];
            if (start[i] < 0 || start[i] > int(tok) || start[i + 1] <= int(tok) || uint32_t(kv) > b.max_kv_len || pos >= kv) report(err, beOffset);
            else mine = cell_of(b, p, i, pos, err);
        }
        for (int t = 0; t < kRun; ++t) {
            const int64_t first = __shfl_sync(0xffffffffu, mine, t);
            const uint32_t tok = run * kRun + t;
            if (first < 0) continue;
            for (uint32_t r0 = 0; r0 < rows; r0 += R * kAhead) {
                uint4 x[kAhead];
                float sc[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const uint32_t r = r0 + u * R + lane / L;
                    if (r >= rows) continue;
                    const bool val = r >= p.n_kv_heads;
                    const int64_t cell = first + (int64_t(val ? r - p.n_kv_heads : r) << p.page_shift);
                    x[u] = __ldg(reinterpret_cast<const uint4*>(val ? p.v : p.k) + cell * L + part);
                    if constexpr (CACHE != WWWS_CACHE_16) sc[u] = __ldg((val ? p.v_scale : p.k_scale) + cell);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const uint32_t r = r0 + u * R + lane / L;
                    if (r >= rows) continue;
                    const bool val = r >= p.n_kv_heads;
                    uint4* o = reinterpret_cast<uint4*>((val ? v_out : k_out) + ((uint64_t(tok) * p.n_kv_heads + (val ? r - p.n_kv_heads : r)) * D + part * E) * 2);
                    if constexpr (CACHE == WWWS_CACHE_16) {
                        o[0] = x[u];
                    } else {
                        uint32_t w[8];
                        const uint32_t c[4] = { x[u].x, x[u].y, x[u].z, x[u].w };
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t t = widen<false, CACHE>((c[e / 2] >> (16 * (e % 2))) & 0xffffu);
                            w[e] = A::pack(Act<false>::lo(t) * sc[u], Act<false>::hi(t) * sc[u]);
                        }
                        o[0] = make_uint4(w[0], w[1], w[2], w[3]);
                        o[1] = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            }
        }
    }
}

template <class F> cudaError_t by_type(uint32_t head_dim, int dtype, int cache, F&& f)
{
    auto dim = [&](auto bf, auto c) { return head_dim == 64 ? f(bf, c, std::integral_constant<int, 64>()) : f(bf, c, std::integral_constant<int, 128>()); };
    auto kind = [&](auto bf) {
        return cache == WWWS_CACHE_16 ? dim(bf, std::integral_constant<int, 0>()) : cache == WWWS_CACHE_INT8 ? dim(bf, std::integral_constant<int, 1>())
                                                                                                             : dim(bf, std::integral_constant<int, 2>());
    };
    return dtype == WWWS_BF16 ? kind(std::true_type()) : kind(std::false_type());
}

uint32_t grid_for(uint64_t tokens)
{
    constexpr uint64_t per_block = kThreads / 32 * kRun;
    const uint64_t blocks = (tokens + per_block - 1) / per_block;
    return uint32_t(blocks < 148 * 16 ? blocks : 148 * 16);
}

}  // namespace

cudaError_t launch_cache_append(const SeqBatch& b, const Pages& p, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride,
                                uint32_t head_dim, int dtype, int cache, uint32_t* err, cudaStream_t s)
{
    return by_type(head_dim, dtype, cache, [&](auto bf, auto c, auto d) {
        k_cache_append<decltype(bf)::value, decltype(c)::value, decltype(d)::value><<<grid_for(b.n_tokens), kThreads, 0, s>>>(
            b, p, static_cast<const uint8_t*>(k), k_stride, static_cast<const uint8_t*>(v), v_stride, err);
        return cudaGetLastError();
    });
}

cudaError_t launch_cache_read(const SeqBatch& b, const Pages& p, const int32_t* row_start, uint64_t n_rows, void* k_out, void* v_out,
                              uint32_t head_dim, int dtype, int cache, uint32_t* err, cudaStream_t s)
{
    return by_type(head_dim, dtype, cache, [&](auto bf, auto c, auto d) {
        k_cache_read<decltype(bf)::value, decltype(c)::value, decltype(d)::value><<<grid_for(n_rows), kThreads, 0, s>>>(
            b, p, row_start, uint32_t(n_rows), static_cast<uint8_t*>(k_out), static_cast<uint8_t*>(v_out), err);
        return cudaGetLastError();
    });
}

}  // namespace wwws
