// Logits shaping: penalties for repeated tokens, biases, a grammar mask, and the row's largest logit, in one pass.
//
// Bound by HBM: every logit is read once and written once.  What makes it more than a copy is the history: a row's tokens
// come in no order, and the penalty of a token depends on how often it occurs.  A block owns a slice of one row's vocabulary
// and counts the history's tokens that fall into the slice in shared memory (one word per token: bit 31 = seen in the
// prompt, the rest = count in the output; integer atomics, so the result does not depend on their order), notes which bias
// entry applies to a token (the last one: an integer maximum), and then streams its slice through.  The history is read once
// per slice, from L2 after the first.  The largest logit is a 64-bit integer maximum of (rounded value as an ordered integer, ~index):
// the lowest index wins a tie, and again the order of the atomics does not matter.  The row's last block to arrive writes the
// token and leaves the row's words at zero for the next call.
#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 256;

template <int DT> struct Elem;
template <> struct Elem<WWWS_F32> {
    static constexpr int kPer16 = 4;
    using Raw = uint32_t;
    static __device__ float get(Raw r) { return __uint_as_float(r); }
    static __device__ Raw put(float f) { return __float_as_uint(f); }
};
template <> struct Elem<WWWS_BF16> {
    static constexpr int kPer16 = 8;
    using Raw = uint16_t;
    static __device__ float get(Raw r) { return __uint_as_float(uint32_t(r) << 16); }
    static __device__ Raw put(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
};
template <> struct Elem<WWWS_F16> {
    static constexpr int kPer16 = 8;
    using Raw = uint16_t;
    static __device__ float get(Raw r) { return __half2float(__ushort_as_half(r)); }
    static __device__ Raw put(float f) { return __half_as_ushort(__float2half_rn(f)); }
};

// Floats as unsigned integers in the same order; NaN and -infinity become 0, which every other value exceeds.
__device__ __forceinline__ uint32_t ordered(float f)
{
    const uint32_t b = __float_as_uint(f);
    if (!(f > -INFINITY)) return 0;
    if (f == 0.0f) return 0x80000000u;          // -0 and +0 are equal
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int DT>
__global__ void __launch_bounds__(kThreads) k_shape_logits(ShapeArgs a)
{
    using E = Elem<DT>;
    using Raw = typename E::Raw;
    extern __shared__ uint32_t words[];          // [slice] counts, then [slice] bias entries where the call has biases
    __shared__ unsigned long long best_of_warp[kThreads / 32];
    const uint32_t row = blockIdx.y, first = blockIdx.x * a.slice;
    const uint32_t n = min(a.slice, a.vocab - first);
    uint32_t* counts = words;
    uint32_t* bias = words + a.slice;

    int h0 = 0, h1 = 0, prompt_end = 0, b0 = 0, b1 = 0;
    if (a.s.history) {
        h0 = a.s.history_start[row]; h1 = a.s.history_start[row + 1];
        if (h0 < 0 || h1 < h0 || uint64_t(h1) > a.s.n_history) { report(a.err, beOffset); h0 = h1 = 0; }
        prompt_end = h0 + (a.s.prompt_len ? a.s.prompt_len[row] : 0);
    }
    if (a.s.bias_id) {
        b0 = a.s.bias_start[row]; b1 = a.s.bias_start[row + 1];
        if (b0 < 0 || b1 < b0 || uint64_t(b1) > a.s.n_bias) { report(a.err, beOffset); b0 = b1 = 0; }
    }
    const uint32_t* mask = nullptr;
    if (a.s.mask) {
        const int m = a.s.mask_index ? a.s.mask_index[row] : int(row);
        if (m >= 0 && uint32_t(m) < a.s.n_masks) mask = a.s.mask + uint64_t(m) * a.s.mask_stride;
        else if (m >= 0) report(a.err, beMask);
    }
    const bool has_history = h1 > h0, has_bias = b1 > b0;
    if (has_history) for (uint32_t i = threadIdx.x; i < n; i += kThreads) counts[i] = 0;
    if (has_bias) for (uint32_t i = threadIdx.x; i < n; i += kThreads) bias[i] = 0;
    __syncthreads();
    for (int i = h0 + int(threadIdx.x); i < h1; i += kThreads) {
        const uint32_t id = uint32_t(a.s.history[i]), at = id - first;
        if (id >= a.vocab) { report(a.err, beToken); continue; }
        if (at >= n) continue;
        if (i < prompt_end) atomicOr(&counts[at], 0x80000000u); else atomicAdd(&counts[at], 1u);
    }
    for (int i = b0 + int(threadIdx.x); i < b1; i += kThreads) {
        const uint32_t id = uint32_t(a.s.bias_id[i]), at = id - first;
        if (id >= a.vocab) { report(a.err, beToken); continue; }
        if (at < n) atomicMax(&bias[at], uint32_t(i - b0) + 1u);
    }
    __syncthreads();

    const float rep = a.s.repetition ? a.s.repetition[row] : 1.0f;
    const float freq = a.s.frequency ? a.s.frequency[row] : 0.0f;
    const float pres = a.s.presence ? a.s.presence[row] : 0.0f;
    unsigned long long best = 0;
    // the operations and their order are the header's; nothing is contracted (the library is built without fused multiply-adds)
    auto shape = [&](Raw raw, uint32_t i, bool allowed) -> Raw {
        float x = E::get(raw);
        if (has_history) {
            const uint32_t c = counts[i];
            if (c) {
                x = x > 0.0f ? __fdiv_rn(x, rep) : x * rep;
                const uint32_t times = c & 0x7fffffffu;
                if (times) { x = x - freq * float(times); x = x - pres; }
            }
        }
        if (has_bias) { const uint32_t e = bias[i]; if (e) x = x + a.s.bias_value[b0 + int(e) - 1]; }
        const Raw r = E::put(allowed ? x : -INFINITY);
        if (a.token) {
            const unsigned long long key = (unsigned long long)(ordered(E::get(r))) << 32 | uint32_t(~(first + i));
            if (key > best) best = key;
        }
        return r;
    };

    const Raw* in = reinterpret_cast<const Raw*>(a.in) + uint64_t(row) * a.in_stride + first;
    Raw* out = reinterpret_cast<Raw*>(a.out) + uint64_t(row) * a.out_stride + first;
    auto scalar = [&](uint32_t i) {
        const uint32_t v = first + i;
        out[i] = shape(in[i], i, !mask || ((mask[v >> 5] >> (v & 31)) & 1u));
    };
    // 16-byte accesses between the first and the last 16-byte boundary of the slice, single elements outside, or throughout
    // where input and output are not aligned alike
    constexpr uint32_t P = E::kPer16;
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(in) & 15), off_out = uint32_t(reinterpret_cast<uintptr_t>(out) & 15);
    const uint32_t head = off == off_out ? min(n, uint32_t(((16 - off) & 15) / sizeof(Raw))) : n;
    const uint32_t vecs = (n - head) / P;
    for (uint32_t i = threadIdx.x; i < head; i += kThreads) scalar(i);
    for (uint32_t j = threadIdx.x; j < vecs; j += kThreads) {
        const uint32_t i = head + j * P, v = first + i;
        const uint4 x = __ldcs(reinterpret_cast<const uint4*>(in + i));
        uint32_t bits = 0xffffffffu;
        if (mask) {
            const uint32_t s = v & 31;
            bits = mask[v >> 5] >> s;
            if (s + P > 32) bits |= mask[(v >> 5) + 1] << (32 - s);
        }
        Raw e[P];
        memcpy(e, &x, 16);
#pragma unroll
        for (uint32_t t = 0; t < P; ++t) e[t] = shape(e[t], i + t, (bits >> t) & 1u);
        uint4 y;
        memcpy(&y, e, 16);
        __stcs(reinterpret_cast<uint4*>(out + i), y);
    }
    for (uint32_t i = head + vecs * P + threadIdx.x; i < n; i += kThreads) scalar(i);
    if (!a.token) return;

#pragma unroll
    for (int m = 16; m; m >>= 1) { const unsigned long long o = __shfl_xor_sync(0xffffffffu, best, m); if (o > best) best = o; }
    if (threadIdx.x % 32 == 0) best_of_warp[threadIdx.x / 32] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) if (best_of_warp[w] > best) best = best_of_warp[w];
        atomicMax(&a.best[row], best);
        __threadfence();
        if (atomicAdd(&a.ticket[row], 1u) == a.n_slices - 1) {
            __threadfence();
            const unsigned long long all = atomicExch(&a.best[row], 0ull);
            a.token[row] = (all >> 32) ? int32_t(~uint32_t(all)) : -1;
            a.ticket[row] = 0;
        }
    }
}

}  // namespace

// Tokens per block: 8,192 (64 KB of counts and bias entries at most) where that gives the GPU enough blocks, fewer down to
// 1,024 for few rows.
uint32_t shape_slice(uint32_t n_rows, uint32_t vocab)
{
    uint32_t slice = 8192;
    while (slice > 1024 && uint64_t(n_rows) * ((vocab + slice - 1) / slice) < 148 * 2) slice /= 2;
    return slice;
}

cudaError_t launch_shape_logits(const ShapeArgs& a, int dtype, cudaStream_t s)
{
    auto go = [&](auto kernel) {
        const uint32_t smem = a.slice * 4 * (a.s.bias_id ? 2 : 1);
        if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536); e != cudaSuccess) return e;
        kernel<<<dim3(a.n_slices, a.n_rows), kThreads, smem, s>>>(a);
        return cudaGetLastError();
    };
    return dtype == WWWS_F32 ? go(k_shape_logits<WWWS_F32>) : dtype == WWWS_BF16 ? go(k_shape_logits<WWWS_BF16>) : go(k_shape_logits<WWWS_F16>);
}

}  // namespace wwws
