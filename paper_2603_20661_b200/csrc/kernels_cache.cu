// Paged key/value cache: writing new tokens (as given, int8 or e4m3) and reading whole sequences back.
//
// Both are pure data movement (a quantised row is one absolute maximum and one multiplication per element), bound by HBM:
// the floor is the bytes given + the bytes held.  A row is the head_dim elements of one (token, kv head); a thread holds 16
// bytes of the narrower side (8 elements as given, 16 quantised), so 4 to 16 neighbouring lanes share a row, its maximum
// is a shuffle over them, and both sides move in 16-byte accesses.  Blocks walk the rows with a grid stride, two rows per
// thread in flight, after one pass over the batch's offsets in shared memory (where a row's sequence is then searched).
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

struct Row { int64_t cell; int64_t io; bool on; };      // row of the page pool (units of head_dim), row of the array

template <bool BF, int CACHE, int D>
__global__ void __launch_bounds__(kThreads) k_cache_append(SeqBatch b, Pages p, const uint8_t* k, uint64_t k_stride, const uint8_t* v, uint64_t v_stride, uint32_t* err)
{
    using A = Act<BF>;
    constexpr int E = CACHE == WWWS_CACHE_16 ? 8 : 16;   // elements per thread
    constexpr int L = D / E;                             // lanes per row
    __shared__ int32_t start[kMaxSeqs + 1];
    for (uint32_t i = threadIdx.x; i <= b.n_seqs; i += kThreads) start[i] = b.q_start[i];
    __syncthreads();
    const uint8_t* src = blockIdx.y ? v : k;
    const uint64_t stride = blockIdx.y ? v_stride : k_stride;
    uint8_t* dst = blockIdx.y ? p.v : p.k;
    float* dst_scale = blockIdx.y ? p.v_scale : p.k_scale;
    const uint32_t lane = threadIdx.x % L;
    const uint32_t rows = b.n_tokens * p.n_kv_heads;
    const uint32_t step = gridDim.x * (kThreads / L);
    constexpr int U = 2;
    // every lane of a warp takes the same number of turns: the maximum below is a shuffle
    for (uint32_t first = blockIdx.x * (kThreads / L); first < rows; first += U * step) {
        uint4 x[U][E / 8];
        Row at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t r = first + u * step + threadIdx.x / L;
            at[u].on = r < rows;
            if (!at[u].on) continue;
            const uint32_t tok = r / p.n_kv_heads, h = r % p.n_kv_heads;
            const uint4* g = reinterpret_cast<const uint4*>(src + (uint64_t(tok) * stride + h * D + lane * E) * 2);
#pragma unroll
            for (int e = 0; e < E / 8; ++e) x[u][e] = __ldg(g + e);
            const uint32_t i = find_seq(start, b.n_seqs, int(tok));
            const int q_len = start[i + 1] - start[i], kv = b.kv_len[i], pos = kv - q_len + int(tok) - start[i];
            if (uint32_t(q_len) > b.max_q_len || uint32_t(kv) > b.max_kv_len || start[i] < 0 || start[i] > int(tok) || start[i + 1] <= int(tok)) { report(err, beOffset); at[u].on = false; continue; }
            if (pos < 0) { at[u].on = false; continue; }
            const uint32_t page = uint32_t(b.page_table[uint64_t(i) * b.table_stride + (uint32_t(pos) >> p.page_shift)]);
            if (page >= p.n_pages) { report(err, bePage); at[u].on = false; continue; }
            at[u].cell = ((int64_t(page) * p.n_kv_heads + h) << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (CACHE == WWWS_CACHE_16) {
                if (at[u].on) reinterpret_cast<uint4*>(dst)[at[u].cell * L + lane] = x[u][0];
            } else {
                constexpr float kTop = CACHE == WWWS_CACHE_INT8 ? 127.0f : 448.0f;
                float f[E];
                uint32_t amax = 0;      // of the absolute values' bits: NaN > infinity > every finite value
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint4 w4 = x[u][e / 8];
                    const uint32_t w = (e / 2) % 4 == 0 ? w4.x : (e / 2) % 4 == 1 ? w4.y : (e / 2) % 4 == 2 ? w4.z : w4.w;
                    f[e] = e % 2 ? A::hi(w) : A::lo(w);
                    amax = max(amax, __float_as_uint(f[e]) & 0x7fffffffu);
                }
#pragma unroll
                for (int m = 1; m < L; m <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, m));
                const bool finite = amax < 0x7f800000u;
                const float top = __uint_as_float(amax);
                const float scale = !finite ? __uint_as_float(0x7fffffffu) : top < 0x1p-100f ? 0.0f : top * (1.0f / kTop);
                const float inv = finite && scale > 0.0f ? __fdiv_rn(1.0f, scale) : 0.0f;
                uint32_t c[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = finite ? fminf(fmaxf(f[w * 4 + e] * inv, -kTop), kTop) : 0.0f;
                    if constexpr (CACHE == WWWS_CACHE_INT8) {
                        const uint32_t b0 = uint32_t(__float2int_rn(y[0])) & 255u, b1 = uint32_t(__float2int_rn(y[1])) & 255u;
                        const uint32_t b2 = uint32_t(__float2int_rn(y[2])) & 255u, b3 = uint32_t(__float2int_rn(y[3])) & 255u;
                        c[w] = b0 | b1 << 8 | b2 << 16 | b3 << 24;
                    } else {
                        uint16_t lo, hi;
                        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y[1]), "f"(y[0]));
                        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y[3]), "f"(y[2]));
                        c[w] = uint32_t(lo) | uint32_t(hi) << 16;
                    }
                }
                if (at[u].on) {
                    reinterpret_cast<uint4*>(dst)[at[u].cell * L + lane] = make_uint4(c[0], c[1], c[2], c[3]);
                    if (lane == 0) dst_scale[at[u].cell] = scale;
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
    constexpr int L = D / E;
    __shared__ int32_t start[kMaxSeqs + 1];
    for (uint32_t i = threadIdx.x; i <= b.n_seqs; i += kThreads) start[i] = row_start[i];
    __syncthreads();
    const uint8_t* src = blockIdx.y ? p.v : p.k;
    const float* src_scale = blockIdx.y ? p.v_scale : p.k_scale;
    uint8_t* dst = blockIdx.y ? v_out : k_out;
    const uint32_t lane = threadIdx.x % L;
    const uint64_t rows = uint64_t(n_rows) * p.n_kv_heads;
    const uint64_t step = uint64_t(gridDim.x) * (kThreads / L);
    constexpr int U = 2;
    for (uint64_t first = blockIdx.x * (kThreads / L); first < rows; first += U * step) {
        uint4 x[U];
        float sc[U];
        uint64_t to[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t r = first + u * step + threadIdx.x / L;
            on[u] = r < rows;
            if (!on[u]) continue;
            // rows in page order: the heads of one token lie a page apart in the pool, the tokens of one head side by side
            const uint32_t tok = uint32_t(r / p.n_kv_heads), h = uint32_t(r % p.n_kv_heads);
            const uint32_t i = find_seq(start, b.n_seqs, int(tok));
            const int pos = int(tok) - start[i];
            if (start[i] < 0 || start[i] > int(tok) || start[i + 1] <= int(tok) || uint32_t(b.kv_len[i]) > b.max_kv_len || pos >= b.kv_len[i]) { report(err, beOffset); on[u] = false; continue; }
            const uint32_t page = uint32_t(b.page_table[uint64_t(i) * b.table_stride + (uint32_t(pos) >> p.page_shift)]);
            if (page >= p.n_pages) { report(err, bePage); on[u] = false; continue; }
            const int64_t cell = ((int64_t(page) * p.n_kv_heads + h) << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
            x[u] = __ldg(reinterpret_cast<const uint4*>(src) + cell * L + lane);
            if constexpr (CACHE != WWWS_CACHE_16) sc[u] = __ldg(src_scale + cell);
            to[u] = r;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!on[u]) continue;
            uint4* o = reinterpret_cast<uint4*>(dst + (to[u] * D + lane * E) * 2);
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

template <class F> cudaError_t by_type(uint32_t head_dim, int dtype, int cache, F&& f)
{
    auto dim = [&](auto bf, auto c) { return head_dim == 64 ? f(bf, c, std::integral_constant<int, 64>()) : f(bf, c, std::integral_constant<int, 128>()); };
    auto kind = [&](auto bf) {
        return cache == WWWS_CACHE_16 ? dim(bf, std::integral_constant<int, 0>()) : cache == WWWS_CACHE_INT8 ? dim(bf, std::integral_constant<int, 1>())
                                                                                                             : dim(bf, std::integral_constant<int, 2>());
    };
    return dtype == WWWS_BF16 ? kind(std::true_type()) : kind(std::false_type());
}

dim3 grid_for(uint64_t rows, uint32_t head_dim, int cache)
{
    const uint64_t per_block = kThreads / (head_dim / (cache == WWWS_CACHE_16 ? 8 : 16));
    const uint64_t blocks = (rows + per_block - 1) / per_block;
    return dim3(uint32_t(blocks < 148 * 8 ? blocks : 148 * 8), 2);
}

}  // namespace

cudaError_t launch_cache_append(const SeqBatch& b, const Pages& p, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride,
                                uint32_t head_dim, int dtype, int cache, uint32_t* err, cudaStream_t s)
{
    return by_type(head_dim, dtype, cache, [&](auto bf, auto c, auto d) {
        k_cache_append<decltype(bf)::value, decltype(c)::value, decltype(d)::value><<<grid_for(uint64_t(b.n_tokens) * p.n_kv_heads, head_dim, cache), kThreads, 0, s>>>(
            b, p, static_cast<const uint8_t*>(k), k_stride, static_cast<const uint8_t*>(v), v_stride, err);
        return cudaGetLastError();
    });
}

cudaError_t launch_cache_read(const SeqBatch& b, const Pages& p, const int32_t* row_start, uint64_t n_rows, void* k_out, void* v_out,
                              uint32_t head_dim, int dtype, int cache, uint32_t* err, cudaStream_t s)
{
    return by_type(head_dim, dtype, cache, [&](auto bf, auto c, auto d) {
        k_cache_read<decltype(bf)::value, decltype(c)::value, decltype(d)::value><<<grid_for(n_rows * p.n_kv_heads, head_dim, cache), kThreads, 0, s>>>(
            b, p, row_start, uint32_t(n_rows), static_cast<uint8_t*>(k_out), static_cast<uint8_t*>(v_out), err);
        return cudaGetLastError();
    });
}

}  // namespace wwws
