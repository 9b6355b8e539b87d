// Logits shaping: penalties for repeated tokens, biases, a grammar mask, and the row's largest logit, in one pass.
//
// Bound by HBM: every logit is read once and written once.  What makes it more than a copy is the history: a row's tokens
// come in no order, and the penalty of a token depends on how often it occurs.  A block owns a slice of one row's vocabulary:
//   1. its logits are requested, into registers;
//   2. while they are on their way, the row's history is counted in shared memory (16 bits per token: bit 15 = seen in the prompt, the
//      rest = count in the output; integer atomics, so the result does not depend on their order), and the bias entry that applies to
//      a token is noted (the last one: an integer maximum).  The history is read once per slice, from L2 after the first;
//   3. eight tokens at a time: untouched ones, nearly all, are only masked and compared, as bits; the others take the arithmetic.
// Rows with more than 32,767 tokens of history are counted in 32 bits, half a slice at a time.  The largest logit is a 64-bit integer
// maximum of (rounded value as an ordered integer, ~index): the lowest index wins a tie, and again the order of the atomics does not
// matter.  The row's last block to arrive writes the token and leaves the row's words at zero for the next call.
#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 512;
constexpr int kMaxCount = 32767;                 // of a 16-bit count

template <int DT> struct Elem;
template <> struct Elem<WWWS_F32> {
    using Raw = uint32_t;
    static __device__ float get(Raw r) { return __uint_as_float(r); }
    static __device__ Raw put(float f) { return __float_as_uint(f); }
};
template <> struct Elem<WWWS_BF16> {
    using Raw = uint16_t;
    static __device__ float get(Raw r) { return __uint_as_float(uint32_t(r) << 16); }
    static __device__ Raw put(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
};
template <> struct Elem<WWWS_F16> {
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

// kVecs 16-byte pieces per thread: a slice is kThreads * kVecs * 16 bytes of logits.
template <int DT, int kVecs>
__global__ void __launch_bounds__(kThreads) k_shape_logits(ShapeArgs a)
{
    using E = Elem<DT>;
    using Raw = typename E::Raw;
    constexpr uint32_t P = 16 / sizeof(Raw), kSlice = kThreads * kVecs * P, kHalf = kSlice / 2;
    extern __shared__ __align__(16) uint8_t smem[];
    uint16_t* count16 = reinterpret_cast<uint16_t*>(smem);                           // [kSlice], or
    uint32_t* count32 = reinterpret_cast<uint32_t*>(smem);                           // [kHalf]
    uint16_t* bias16 = reinterpret_cast<uint16_t*>(smem) + kSlice;                   // [kSlice], where the call has biases: entry + 1
    __shared__ unsigned long long best_of_warp[kThreads / 32];
    const uint32_t row = blockIdx.y, first = blockIdx.x * (kSlice - P);              // (P tokens short: room for an unaligned start)
    const uint32_t n = min(kSlice - P, a.vocab - first);

    const Raw* in = reinterpret_cast<const Raw*>(a.in) + uint64_t(row) * a.in_stride + first;
    Raw* out = reinterpret_cast<Raw*>(a.out) + uint64_t(row) * a.out_stride + first;
    // 16-byte accesses between the first and the last 16-byte boundary of the slice, single elements outside, or throughout
    // where input and output are not aligned alike
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(in) & 15), off_out = uint32_t(reinterpret_cast<uintptr_t>(out) & 15);
    const uint32_t head = off == off_out ? min(n, uint32_t(((16 - off) & 15) / sizeof(Raw))) : n;
    const uint32_t vecs = (n - head) / P, shift = (P - head % P) % P;                // token i's words are at i + shift: pieces start at multiples of P
    uint4 x[kVecs];
#pragma unroll
    for (int t = 0; t < kVecs; ++t) {
        const uint32_t j = threadIdx.x + t * kThreads;
        if (j < vecs) x[t] = __ldcs(reinterpret_cast<const uint4*>(in + head) + j);
    }

    int h0 = 0, h1 = 0, prompt_end = 0, b0 = 0, b1 = 0;
    if (a.s.history) {
        h0 = a.s.history_start[row]; h1 = a.s.history_start[row + 1];
        if (h0 < 0 || h1 < h0 || uint64_t(h1) > a.s.n_history) { report(a.err, beOffset); h0 = h1 = 0; }
        prompt_end = h0 + (a.s.prompt_len ? a.s.prompt_len[row] : 0);
    }
    if (a.s.bias_id) {
        b0 = a.s.bias_start[row]; b1 = a.s.bias_start[row + 1];
        if (b0 < 0 || b1 < b0 || b1 - b0 > 65535 || uint64_t(b1) > a.s.n_bias) { report(a.err, beOffset); b0 = b1 = 0; }
    }
    const uint32_t* mask = nullptr;
    if (a.s.mask) {
        const int m = a.s.mask_index ? a.s.mask_index[row] : int(row);
        if (m >= 0 && uint32_t(m) < a.s.n_masks) mask = a.s.mask + uint64_t(m) * a.s.mask_stride;
        else if (m >= 0) report(a.err, beMask);
    }
    const float rep = a.s.repetition ? a.s.repetition[row] : 1.0f;
    const float freq = a.s.frequency ? a.s.frequency[row] : 0.0f;
    const float pres = a.s.presence ? a.s.presence[row] : 0.0f;
    const bool has_history = h1 > h0, has_bias = b1 > b0, wide = h1 - h0 > kMaxCount;

    float best = -INFINITY;
    uint32_t best_at = 0;
    auto consider = [&](float v, uint32_t i) { if (v > best) { best = v; best_at = i; } };       // a thread meets its tokens in ascending order, except as noted
    if (has_bias) {
        for (uint32_t i = threadIdx.x; i < kSlice / 8; i += kThreads) reinterpret_cast<uint4*>(bias16)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        for (int i = b0 + int(threadIdx.x); i < b1; i += kThreads) {
            const uint32_t id = uint32_t(a.s.bias_id[i]), at = id - first;
            if (id >= a.vocab) { report(a.err, beToken); continue; }
            if (at >= n) continue;
            // the largest entry of a token, in its half of a word
            uint32_t* word = reinterpret_cast<uint32_t*>(bias16) + ((at + shift) >> 1);
            const uint32_t up = ((at + shift) & 1) * 16, e = uint32_t(i - b0) + 1u;
            uint32_t was = *word;
            while (((was >> up) & 0xffffu) < e) {
                const uint32_t seen = atomicCAS(word, was, (was & ~(0xffffu << up)) | e << up);
                if (seen == was) break;
                was = seen;
            }
        }
    }
    for (uint32_t part = 0; part < (wide ? 2u : 1u); ++part) {
        const uint32_t from = part * kHalf, size = wide ? kHalf : kSlice;            // the words [from, from + size) of this part
        if (has_history) {
            if (part) __syncthreads();
            for (uint32_t i = threadIdx.x; i < kSlice / 8; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            for (int i = h0 + int(threadIdx.x); i < h1; i += kThreads) {
                const uint32_t id = uint32_t(__ldg(a.s.history + i)), at = id - first;
                if (id >= a.vocab) { report(a.err, beToken); continue; }
                const uint32_t w = at + shift - from;
                if (at >= n || w >= size) continue;
                if (wide) {
                    if (i < prompt_end) atomicOr(count32 + w, 0x80000000u); else atomicAdd(count32 + w, 1u);
                } else {
                    uint32_t* word = count32 + (w >> 1);
                    const uint32_t up = (w & 1) * 16;
                    if (i < prompt_end) atomicOr(word, 0x8000u << up); else atomicAdd(word, 1u << up);
                }
            }
        }
        if (has_history || has_bias) __syncthreads();

        // the operations and their order are the header's; nothing is contracted (the library is built without fused multiply-adds)
        auto shape = [&](Raw raw, uint32_t i, bool allowed) -> Raw {
            float v = E::get(raw);
            if (has_history) {
                const uint32_t w = i + shift - from;
                uint32_t seen, times;
                if (wide) { const uint32_t c = count32[w]; seen = c; times = c & 0x7fffffffu; }
                else { const uint32_t c = count16[w]; seen = c; times = c & 0x7fffu; }
                if (seen) {
                    v = v > 0.0f ? __fdiv_rn(v, rep) : v * rep;
                    if (times) { v = v - freq * float(times); v = v - pres; }
                }
            }
            if (has_bias) { const uint32_t e = bias16[i + shift]; if (e) v = v + a.s.bias_value[b0 + int(e) - 1]; }
            return E::put(allowed ? v : -INFINITY);
        };
        auto scalar = [&](uint32_t i) {
            const uint32_t v = first + i;
            if (i + shift - from >= size) return;
            const Raw r = shape(in[i], i, !mask || ((mask[v >> 5] >> (v & 31)) & 1u));
            out[i] = r;
            const float f = E::get(r);
            if (f > best || (f == best && i < best_at && f > -INFINITY)) { best = f; best_at = i; }
        };
        for (uint32_t i = threadIdx.x; i < head; i += kThreads) scalar(i);
#pragma unroll
        for (int t = 0; t < kVecs; ++t) {
            const uint32_t j = threadIdx.x + t * kThreads, i = head + j * P, w = i + shift - from;
            if (j >= vecs || w >= size) continue;
            const uint32_t v = first + i;
            uint32_t bits = (1u << P) - 1;
            if (mask) {
                const uint32_t s = v & 31;
                uint32_t m = mask[v >> 5] >> s;
                if (s + P > 32) m |= mask[(v >> 5) + 1] << (32 - s);
                bits &= m;
            }
            uint32_t touched = 0;                                                    // any word of these tokens
            if (has_history) {
                if (wide) {
#pragma unroll
                    for (uint32_t e = 0; e < P; ++e) touched |= count32[w + e];
                } else if constexpr (P == 8) { const uint4 c = *reinterpret_cast<const uint4*>(count16 + w); touched = c.x | c.y | c.z | c.w; }
                else { const uint2 c = *reinterpret_cast<const uint2*>(count16 + w); touched = c.x | c.y; }
            }
            if (has_bias) {
                if constexpr (P == 8) { const uint4 c = *reinterpret_cast<const uint4*>(bias16 + i + shift); touched |= c.x | c.y | c.z | c.w; }
                else { const uint2 c = *reinterpret_cast<const uint2*>(bias16 + i + shift); touched |= c.x | c.y; }
            }
            uint32_t q[4] = { x[t].x, x[t].y, x[t].z, x[t].w };
            if (touched) {
                Raw e[P];
                memcpy(e, q, 16);
#pragma unroll
                for (uint32_t k = 0; k < P; ++k) e[k] = shape(e[k], i + k, (bits >> k) & 1u);
                memcpy(q, e, 16);
            } else if (bits != (1u << P) - 1) {
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    if constexpr (P == 8) {
                        constexpr uint32_t kNone = DT == WWWS_BF16 ? 0xff80u : 0xfc00u;
                        const uint32_t keep = ((bits >> (2 * k)) & 1u) * 0xffffu | ((bits >> (2 * k + 1)) & 1u) * 0xffff0000u;
                        q[k] = (q[k] & keep) | (~keep & (kNone | kNone << 16));
                    } else q[k] = (bits >> k) & 1u ? q[k] : 0xff800000u;
                }
            }
            if (a.token) {
                float f[P];
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    if constexpr (P == 8) { f[2 * k] = E::get(Raw(q[k])); f[2 * k + 1] = E::get(Raw(q[k] >> 16)); }
                    else f[k] = E::get(Raw(q[k]));
                }
                float top = f[0];
#pragma unroll
                for (uint32_t k = 1; k < P; ++k) top = fmaxf(top, f[k]);
                // (the head's single tokens lie below, so a tie keeps what is there)
                if (top > best) {
#pragma unroll
                    for (uint32_t k = 0; k < P; ++k) consider(f[k], i + k);
                }
            }
            __stcs(reinterpret_cast<uint4*>(out + i), make_uint4(q[0], q[1], q[2], q[3]));
        }
        for (uint32_t i = head + vecs * P + threadIdx.x; i < n; i += kThreads) scalar(i);
    }
    if (!a.token) return;

    unsigned long long key = best > -INFINITY ? (unsigned long long)(ordered(best)) << 32 | uint32_t(~(first + best_at)) : 0ull;
#pragma unroll
    for (int m = 16; m; m >>= 1) { const unsigned long long o = __shfl_xor_sync(0xffffffffu, key, m); if (o > key) key = o; }
    if (threadIdx.x % 32 == 0) best_of_warp[threadIdx.x / 32] = key;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) if (best_of_warp[w] > key) key = best_of_warp[w];
        unsigned long long all = key;
        if (a.n_slices > 1) {
            if (key) atomicMax(&a.best[row], key);
            __threadfence();
            if (atomicAdd(&a.ticket[row], 1u) != gridDim.x - 1) return;
            __threadfence();
            all = atomicExch(&a.best[row], 0ull);
            a.ticket[row] = 0;
        }
        a.token[row] = (all >> 32) ? int32_t(~uint32_t(all)) : -1;
    }
}

}  // namespace

// Slices of 32 KB of logits (16,384 16-bit tokens: counts and bias entries take 64 KB of shared memory) where that gives every SM two blocks, down
// to 8 KB for few rows, whose time is that of one block.
cudaError_t launch_shape_logits(const ShapeArgs& given, int dtype, cudaStream_t s)
{
    auto go = [&](auto type, auto vecs) -> cudaError_t {
        constexpr int DT = decltype(type)::value, kVecs = decltype(vecs)::value;
        constexpr uint32_t P = DT == WWWS_F32 ? 4 : 8, slice = kThreads * kVecs * P;
        constexpr auto kernel = k_shape_logits<DT, kVecs>;
        ShapeArgs a = given;
        a.n_slices = (a.vocab + slice - P - 1) / (slice - P);
        if (cudaError_t e = allow_smem<kernel>(slice * 4); e != cudaSuccess) return e;
        kernel<<<dim3(a.n_slices, a.n_rows), kThreads, slice * (a.s.bias_id ? 4 : 2), s>>>(a);
        return cudaGetLastError();
    };
    using std::integral_constant;
    auto size = [&](auto type) {
        const uint64_t bytes = uint64_t(given.n_rows) * given.vocab * (decltype(type)::value == WWWS_F32 ? 4 : 2);
        return bytes >= 148 * 2 * 32768ull ? go(type, integral_constant<int, 4>()) : bytes >= 148 * 2 * 16384ull ? go(type, integral_constant<int, 2>()) : go(type, integral_constant<int, 1>());
    };
    return dtype == WWWS_F32 ? size(integral_constant<int, WWWS_F32>()) : dtype == WWWS_BF16 ? size(integral_constant<int, WWWS_BF16>()) : size(integral_constant<int, WWWS_F16>());
}

}  // namespace wwws
