// Logits shaping: penalties for repeated tokens, biases, a grammar mask, and the row's largest logit, in one pass.
//
// Bound by HBM: every logit is read once and written once.  What makes it more than a copy is the history: a row's tokens
// come in no order, and the penalty of a token depends on how often it occurs.  Few rows are bound by latency and go to k_shape_few at the end of this file.
// In a large batch a block takes a part of one row (all of it where there are enough rows) and first sorts the part's history by slices of 1,024 tokens
// (2 KB of 16-bit logits) into shared memory, a counting sort, while
// the first logits are on their way.  From there on its warps work alone, without a barrier, a slice at a time:
//   1. the slice's history is counted and its biases are noted in a word per token: 20 bits of count in the output, a bit for the prompt, 11 bits
//      for the last bias entry that names the token (integer atomics: their order does not matter);
//   2. eight tokens at a time, all are masked and written as bits, and their maximum is taken two at a time;
//   3. the next slice's logits are requested, and the touched tokens are done over, a lane each, and their
//      words cleared; where they are many (low ids, mostly) step 2 takes their arithmetic on the way.
// Doing the touched tokens over, not in step 2, spares nearly every warp the arithmetic of all its tokens for the sake of one or two.
// Measured at 256 x 131,072 bf16 logits with 2,000 tokens of history a row: arithmetic in step 2 166 us; a block per slice of 16,384 tokens, its
// phases between barriers, 97 us; this way 66 us, 29 of them without a history.
// The maximum of step 2 counts touched tokens by their old logits; should it be in a piece with one of those, the warp takes it again without them.
// The largest logit is a 64-bit integer maximum of (rounded value as an ordered integer, ~index): the lowest index wins a tie, and again the
// order of the atomics does not matter.  The block that brings a row's last part writes the token and leaves the row's words at zero for the
// next call.
#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kBlocks = 4;     // blocks per SM
constexpr uint32_t kTokens = 1024;               // of a slice
constexpr uint32_t kSlices = 256;                // of a part, at most
constexpr uint32_t kIds = 8192;                  // history entries of a part that are sorted; with more, every slice goes through the history
constexpr uint32_t kBiases = 512;                // bias entries that are kept in shared memory
constexpr uint32_t kHeavy = 128;                 // touched tokens of a slice above which they are done with the others
constexpr uint32_t kMaxBias = 2047, kMaxHistory = (1u << 20) - 1;
constexpr uint32_t kPrompt = 1u << 20, kCount = kPrompt - 1;           // fields of a token's word; the bias entry + 1 is above them

// max2: the larger of two packed pairs (f32: of two numbers); a NaN loses.
template <int DT> struct Elem;
template <> struct Elem<WWWS_F32> {
    using Raw = uint32_t;
    static __device__ uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ float last(uint32_t w) { return __uint_as_float(w); }
    static __device__ float get(Raw r) { return __uint_as_float(r); }
    static __device__ Raw put(float f) { return __float_as_uint(f); }
};
template <> struct Elem<WWWS_BF16> {
    using Raw = uint16_t;
    static __device__ uint32_t max2(uint32_t a, uint32_t b) { uint32_t r; asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
    static __device__ float last(uint32_t w) { return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ float get(Raw r) { return __uint_as_float(uint32_t(r) << 16); }
    static __device__ Raw put(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
};
template <> struct Elem<WWWS_F16> {
    using Raw = uint16_t;
    static __device__ uint32_t max2(uint32_t a, uint32_t b) { uint32_t r; asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
    static __device__ float last(uint32_t w) { return fmaxf(__half2float(__ushort_as_half(uint16_t(w))), __half2float(__ushort_as_half(uint16_t(w >> 16)))); }
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

// What a row asks for; offsets and indices out of range are reported and left out.
struct Row {
    int h0 = 0, h1 = 0, prompt_end = 0, b0 = 0, nb = 0;       // its history and where its prompt ends, its biases
    const uint32_t* mask = nullptr;
    float rep, freq, pres;
    __device__ __forceinline__ Row(const ShapeArgs& a, uint32_t row)
    {
        if (a.s.history) {
            h0 = a.s.history_start[row]; h1 = a.s.history_start[row + 1];
            if (h0 < 0 || h1 < h0 || uint64_t(h1) > a.s.n_history || h1 - h0 > int(kMaxHistory)) { report(a.err, beOffset); h0 = h1 = 0; }
            prompt_end = h0 + (a.s.prompt_len ? min(max(a.s.prompt_len[row], 0), h1 - h0) : 0);
        }
        if (a.s.bias_id) {
            b0 = a.s.bias_start[row]; nb = a.s.bias_start[row + 1] - b0;
            if (b0 < 0 || nb < 0 || nb > int(kMaxBias) || uint64_t(b0) + uint64_t(nb) > a.s.n_bias) { report(a.err, beOffset); b0 = nb = 0; }
        }
        if (a.s.mask) {
            const int m = a.s.mask_index ? a.s.mask_index[row] : int(row);
            if (m >= 0 && uint32_t(m) < a.s.n_masks) mask = a.s.mask + uint64_t(m) * a.s.mask_stride;
            else if (m >= 0) report(a.err, beMask);
        }
        rep = a.s.repetition ? a.s.repetition[row] : 1.0f;
        freq = a.s.frequency ? a.s.frequency[row] : 0.0f;
        pres = a.s.presence ? a.s.presence[row] : 0.0f;
    }
    // The logit of a token with word c.  The operations and their order are the header's; nothing is contracted (the library is built without fused multiply-adds).
    __device__ __forceinline__ float shaped(const ShapeArgs& a, float f, uint32_t c) const
    {
        // (selected, not branched to: several tokens' divisions overlap)
        const float g = f > 0.0f ? __fdiv_rn(f, rep) : f * rep;
        f = c & (kPrompt | kCount) ? g : f;
        const float h = f - freq * float(c & kCount);
        f = c & kCount ? h - pres : f;
        if (c >> 21) f = f + a.s.bias_value[b0 + int(c >> 21) - 1];
        return f;
    }
};

// The tokens [i, i + P) of a row whose first is token v: hidden ones become -infinity.
template <int DT> __device__ __forceinline__ void hide(uint4& x, const uint32_t* mask, uint32_t v)
{
    constexpr uint32_t P = 16 / sizeof(typename Elem<DT>::Raw);
    const uint32_t s = v & 31;
    uint32_t bits = __ldg(mask + (v >> 5)) >> s;
    if (s + P > 32) bits |= __ldg(mask + (v >> 5) + 1) << (32 - s);
    auto put = [&](uint32_t& q, uint32_t k) {
        if constexpr (P == 8) {
            constexpr uint32_t kNone = DT == WWWS_BF16 ? 0xff80u : 0xfc00u;
            const uint32_t keep = ((bits >> (2 * k)) & 1u) * 0xffffu | ((bits >> (2 * k + 1)) & 1u) * 0xffff0000u;
            q = (q & keep) | (~keep & (kNone | kNone << 16));
        } else q = (bits >> k) & 1u ? q : 0xff800000u;
    };
    put(x.x, 0); put(x.y, 1); put(x.z, 2); put(x.w, 3);
}

// The row's largest over its blocks: a warp's lanes, the block's warps, then the blocks; the last block writes the token.
template <int kWarpsOf> __device__ __forceinline__ void settle(const ShapeArgs& a, uint32_t row, unsigned long long key, unsigned long long* best_of_warp)
{
#pragma unroll
    for (int m = 16; m; m >>= 1) { const unsigned long long o = __shfl_xor_sync(0xffffffffu, key, m); if (o > key) key = o; }
    if (threadIdx.x % 32 == 0) best_of_warp[threadIdx.x / 32] = key;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < kWarpsOf; ++w) if (best_of_warp[w] > key) key = best_of_warp[w];
        if (gridDim.x > 1) {
            if (key) atomicMax(&a.best[row], key);
            __threadfence();
            if (atomicAdd(&a.ticket[row], 1u) != gridDim.x - 1) return;
            __threadfence();
            key = atomicExch(&a.best[row], 0ull);
            a.ticket[row] = 0;
        }
        a.token[row] = (key >> 32) ? int32_t(~uint32_t(key)) : -1;
    }
}

// A warp's words have room for 8 tokens more than a slice, so that 16-byte pieces start at multiples of theirs whatever the row's alignment.
constexpr uint32_t kWords = kTokens + 8;
constexpr uint32_t kSmem = kWarps * kWords * 4 + kIds * 2 + kSlices * 4 + kBiases * 4 + kWarps * kHeavy * 2;

template <int DT>
__global__ void __launch_bounds__(kThreads, kBlocks) k_shape_logits(ShapeArgs a)
{
    using E = Elem<DT>;
    using Raw = typename E::Raw;
    constexpr uint32_t P = 16 / sizeof(Raw);     // tokens of 16 bytes
    constexpr int kVecs = kTokens / P / 32;      // 16-byte pieces of a lane
    extern __shared__ __align__(16) uint32_t smem[];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t* words = smem + warp * kWords;
    uint32_t* slice_end = smem + kWarps * kWords;                                    // [kSlices] where a slice's entries end in ids
    uint32_t* bias_ids = slice_end + kSlices;
    uint16_t* ids = reinterpret_cast<uint16_t*>(bias_ids + kBiases);                 // [kIds] token within its slice, bit 15 = in the prompt
    uint16_t* listed = ids + kIds + warp * kHeavy;                                   // [kHeavy] touched tokens of the slice
    __shared__ unsigned long long best_of_warp[kWarps];
    __shared__ uint32_t sum_of_warp[kWarps];

    const uint32_t row = blockIdx.y, n_slices = (a.vocab + kTokens - 1) / kTokens;
    const uint32_t s0 = uint32_t(uint64_t(n_slices) * blockIdx.x / gridDim.x), s1 = uint32_t(uint64_t(n_slices) * (blockIdx.x + 1) / gridDim.x);

    // A slice's place: 16-byte accesses between its first and last 16-byte boundary, single elements outside, or throughout where input and
    // output are not aligned alike.  Token i's word is at i + shift: pieces start at multiples of P.
    struct Place { const Raw* in; Raw* out; uint32_t first, n, head, vecs, shift; };
    auto place = [&](uint32_t slice) {
        Place p;
        p.first = slice * kTokens;
        p.n = min(kTokens, a.vocab - p.first);
        p.in = reinterpret_cast<const Raw*>(a.in) + uint64_t(row) * a.in_stride + p.first;
        p.out = reinterpret_cast<Raw*>(a.out) + uint64_t(row) * a.out_stride + p.first;
        const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p.in) & 15), off_out = uint32_t(reinterpret_cast<uintptr_t>(p.out) & 15);
        p.head = off == off_out ? min(p.n, uint32_t(((16 - off) & 15) / sizeof(Raw))) : p.n;
        p.vecs = (p.n - p.head) / P;
        p.shift = (P - p.head % P) % P;
        return p;
    };
    uint4 x[kVecs];
    auto request = [&](uint32_t slice) {
        if (slice >= s1) return;
        const Place p = place(slice);
#pragma unroll
        for (int t = 0; t < kVecs; ++t) if (lane + t * 32 < p.vecs) x[t] = *(reinterpret_cast<const uint4*>(p.in + p.head) + lane + t * 32);     // (kept in L2: touched tokens are read again)
    };
    request(s0 + warp);

    const Row what(a, row);
    const int h0 = what.h0, h1 = what.h1, prompt_end = what.prompt_end, b0 = what.b0, nb = what.nb;
    const uint32_t* mask = what.mask;

    bool sorted = true;
    if (h1 > h0 || nb) {
        for (uint32_t i = threadIdx.x; i < kWarps * kWords / 4; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
        for (int i = threadIdx.x; i < min(nb, int(kBiases)); i += kThreads) {
            const uint32_t id = uint32_t(__ldg(a.s.bias_id + b0 + i));
            if (id >= a.vocab) report(a.err, beToken);
            bias_ids[i] = id;
        }
        if (h1 > h0) {           // the counting sort; the order within a slice does not matter
            slice_end[threadIdx.x] = 0;
            static_assert(kSlices == kThreads, "a thread per slice");
            __syncthreads();
            auto places = [&](int pass) {
                constexpr int kAhead = 4;                    // entries per thread that are requested together
                for (int first = h0 + int(threadIdx.x); first < h1; first += kAhead * kThreads) {
                    uint32_t id[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) id[k] = first + k * kThreads < h1 ? uint32_t(__ldg(a.s.history + first + k * kThreads)) : 0xffffffffu;
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) {
                        const int i = first + k * kThreads;
                        const uint32_t slice = id[k] / kTokens;
                        if (id[k] >= a.vocab) { if (i < h1 && pass == 0) report(a.err, beToken); }
                        else if (slice >= s0 && slice < s1) {
                            const uint32_t at = atomicAdd(&slice_end[slice - s0], 1u);
                            if (pass) ids[at] = uint16_t(id[k] % kTokens | (i < prompt_end ? 0x8000u : 0u));
                        }
                    }
                }
            };
            places(0);
            __syncthreads();
            const uint32_t mine = slice_end[threadIdx.x];
            uint32_t sum = mine;
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) { const uint32_t o = __shfl_up_sync(0xffffffffu, sum, m); if (lane >= uint32_t(m)) sum += o; }
            if (lane == 31) sum_of_warp[warp] = sum;
            __syncthreads();
            uint32_t before = 0, all = 0;
#pragma unroll
            for (uint32_t w = 0; w < kWarps; ++w) { if (w < warp) before += sum_of_warp[w]; all += sum_of_warp[w]; }
            sorted = all <= kIds;
            if (sorted) {
                slice_end[threadIdx.x] = before + sum - mine;            // where the slice starts; the second pass moves it to the end
                __syncthreads();
                places(1);
            }
        }
        __syncthreads();
    }
    const bool has_history = h1 > h0, plain = !has_history && !nb;

    float best = -INFINITY;                                  // of this lane's touched and single tokens
    uint32_t best_at = 0, warp_best = 0, warp_best_at = 0;   // of untouched tokens, ordered(); the warp's lanes agree
    for (uint32_t slice = s0 + warp; slice < s1; slice += kWarps) {
        const Place p = place(slice);
        const uint32_t e0 = sorted && has_history && slice > s0 ? slice_end[slice - s0 - 1] : 0, e1 = sorted && has_history ? slice_end[slice - s0] : 0;
        // bias entries and history into the words; the tokens whose word was empty are listed
        uint32_t n_listed = 0;
        auto list = [&](bool first, uint32_t at) {
            const uint32_t who = __ballot_sync(0xffffffffu, first), k = n_listed + __popc(who & ((1u << lane) - 1));
            if (first && k < kHeavy) listed[k] = uint16_t(at);
            n_listed += __popc(who);
        };
        for (int i0 = 0; i0 < nb; i0 += 32) {
            const int i = i0 + int(lane);
            uint32_t at = 0xffffffffu;
            if (i < nb) {
                const uint32_t id = i < int(kBiases) ? bias_ids[i] : uint32_t(__ldg(a.s.bias_id + b0 + i));
                if (id < a.vocab) at = id - p.first; else if (i >= int(kBiases)) report(a.err, beToken);
            }
            list(at < p.n && atomicMax(words + at + p.shift, uint32_t(i + 1) << 21) == 0, at);
        }
        if (nb) __syncwarp();
        // entries [i0, end) of the history, four per lane at a time (the atomics' latency is most of it); get: an entry's place in the slice and
        // whether it is in the prompt
        auto count = [&](int i0, int end, auto&& get) {
            for (; i0 < end; i0 += 128) {
                uint32_t at[4], was[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + 32 * k + int(lane);
                    bool prompt = false;
                    at[k] = 0xffffffffu;
                    if (i < end) get(i, at[k], prompt);
                    was[k] = 1;
                    if (at[k] < p.n) was[k] = prompt ? atomicOr(words + at[k] + p.shift, kPrompt) : atomicAdd(words + at[k] + p.shift, 1u);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) list(was[k] == 0, at[k]);
            }
        };
        if (sorted) count(int(e0), int(e1), [&](int i, uint32_t& at, bool& prompt) { const uint32_t v = ids[i]; at = v & 0x3ffu; prompt = v >> 15; });
        else count(h0, h1, [&](int i, uint32_t& at, bool& prompt) { const uint32_t id = uint32_t(__ldg(a.s.history + i)); at = id < a.vocab ? id - p.first : 0xffffffffu; prompt = i < prompt_end; });
        __syncwarp();

        // Slices with many touched tokens (low ids, mostly) take the arithmetic on the way, where the logits are in registers.
        const bool heavy = n_listed > kHeavy;
        auto shaped = [&](float f, uint32_t c) { return what.shaped(a, f, c); };
        auto allows = [&](uint32_t i) { const uint32_t v = p.first + i; return !mask || ((__ldg(mask + (v >> 5)) >> (v & 31)) & 1u); };
        auto touched = [&](uint32_t i) { return !plain && words[i + p.shift] != 0; };
        auto better = [&](float v, uint32_t i) { if (v > best || (v == best && p.first + i < best_at && v > -INFINITY)) { best = v; best_at = p.first + i; } };
        auto single = [&](uint32_t i) {
            Raw r = p.in[i];
            const uint32_t c = heavy ? words[i + p.shift] : 0;
            if (c) { words[i + p.shift] = 0; r = E::put(shaped(E::get(r), c)); }
            if (!allows(i)) r = E::put(-INFINITY);
            p.out[i] = r;
            if (!touched(i)) better(E::get(r), i);
        };
        for (uint32_t i = lane; i < p.head; i += 32) single(i);
        for (uint32_t i = p.head + p.vecs * P + lane; i < p.n; i += 32) single(i);
        if (heavy) {
            // in a loop that is not unrolled (its code would be most of the kernel's), by way of the output, which the lane itself reads back
#pragma unroll 1
            for (uint32_t j = lane; j < p.vecs; j += 32) {
                const uint32_t i = p.head + j * P;
                uint4 q = *(reinterpret_cast<const uint4*>(p.in + p.head) + j);
                Raw e[P];
                memcpy(e, &q, 16);
#pragma unroll
                for (uint32_t k = 0; k < P; ++k) {
                    const uint32_t c = words[i + k + p.shift];
                    const Raw r = E::put(shaped(E::get(e[k]), c));
                    e[k] = c ? r : e[k];
                }
#pragma unroll
                for (uint32_t k = 0; k < P; k += 4) *reinterpret_cast<uint4*>(words + i + k + p.shift) = make_uint4(0, 0, 0, 0);
                memcpy(&q, e, 16);
                *(reinterpret_cast<uint4*>(p.out + p.head) + j) = q;
            }
#pragma unroll
            for (int t = 0; t < kVecs; ++t) if (lane + t * 32 < p.vecs) x[t] = *(reinterpret_cast<const uint4*>(p.out + p.head) + lane + t * 32);
        }
        float top = -INFINITY;                               // the largest of this lane's pieces, and the first piece that has it
        int top_t = 0;
#pragma unroll
        for (int t = 0; t < kVecs; ++t) {
            if (lane + t * 32 >= p.vecs) continue;
            const uint32_t i = p.head + (lane + t * 32) * P;
            if (mask) hide<DT>(x[t], mask, p.first + i);
            __stcs(reinterpret_cast<uint4*>(p.out + i), x[t]);
            const float f = E::last(E::max2(E::max2(x[t].x, x[t].y), E::max2(x[t].z, x[t].w)));
            if (f > top) { top = f; top_t = t; }
        }
        if (a.token) {
            // The warp's largest, where it exceeds what the warp has (later tokens lose ties).  The lanes that hold it find the token; if
            // their pieces have touched tokens, the warp looks again without those.
            uint32_t mine = ordered(top), all = __reduce_max_sync(0xffffffffu, mine);
            if (all > warp_best) {
                uint32_t at = 0xffffffffu;
                bool clash = false;
                if (mine == all) {
#pragma unroll
                    for (int t = 0; t < kVecs; ++t) {
                        if (t != top_t) continue;
                        const uint32_t i = p.head + (lane + t * 32) * P;
                        Raw e[P];
                        memcpy(e, &x[t], 16);
#pragma unroll
                        for (int k = int(P) - 1; k >= 0; --k) { clash = clash || touched(i + k); if (E::get(e[k]) == top) at = i + k; }
                    }
                }
                if (__any_sync(0xffffffffu, clash)) {
                    top = -INFINITY; at = 0xffffffffu;
#pragma unroll
                    for (int t = 0; t < kVecs; ++t) {
                        if (lane + t * 32 >= p.vecs) continue;
                        const uint32_t i = p.head + (lane + t * 32) * P;
                        Raw e[P];
                        memcpy(e, &x[t], 16);
#pragma unroll
                        for (uint32_t k = 0; k < P; ++k) { const float f = E::get(e[k]); if (f > top && !touched(i + k)) { top = f; at = i + k; } }
                    }
                    mine = ordered(top); all = __reduce_max_sync(0xffffffffu, mine);
                }
                at = __reduce_min_sync(0xffffffffu, mine == all ? at : 0xffffffffu);
                if (all > warp_best) { warp_best = all; warp_best_at = p.first + at; }
            }
        }
        request(slice + kWarps);
        if (plain) continue;
        __syncwarp();                                        // what is done over below has been written
        if (!heavy) {
            // two at a time: their logits are on their way together
            for (uint32_t i = lane; i < n_listed; i += 64) {
                const bool two = i + 32 < n_listed;
                const uint32_t at0 = listed[i], at1 = two ? listed[i + 32] : 0;
                const Raw in0 = p.in[at0], in1 = two ? p.in[at1] : Raw(0);
                const bool on0 = allows(at0), on1 = two && allows(at1);              // the others are masked above
                if (on0) { const Raw r = E::put(shaped(E::get(in0), words[at0 + p.shift])); p.out[at0] = r; better(E::get(r), at0); }
                if (on1) { const Raw r = E::put(shaped(E::get(in1), words[at1 + p.shift])); p.out[at1] = r; better(E::get(r), at1); }
                words[at0 + p.shift] = 0;
                if (two) words[at1 + p.shift] = 0;
            }
        }
        __syncwarp();
    }
    if (!a.token) return;

    unsigned long long key = best > -INFINITY ? (unsigned long long)(ordered(best)) << 32 | uint32_t(~best_at) : 0ull;
    const unsigned long long of_warp = warp_best ? (unsigned long long)(warp_best) << 32 | uint32_t(~warp_best_at) : 0ull;
    if (of_warp > key) key = of_warp;
    settle<kWarps>(a, row, key, best_of_warp);
}

// Few rows: a block for each kFewTokens tokens, which counts the row's whole history into its words as it comes, while its logits are on their way,
// and does the arithmetic of touched tokens where they are.  One launch, two barriers: a judge's verdict (one row of 32,003 f32 logits, 300 tokens of
// history) takes 9.8 us a call, most of it the call's own; sorted it took 17.5.
constexpr int kFewThreads = 256;
constexpr uint32_t kFewTokens = 2048;

template <int DT>
__global__ void __launch_bounds__(kFewThreads) k_shape_few(ShapeArgs a)
{
    using E = Elem<DT>;
    using Raw = typename E::Raw;
    constexpr uint32_t P = 16 / sizeof(Raw);
    constexpr int kVecs = kFewTokens / P / kFewThreads;
    __shared__ __align__(16) uint32_t words[kFewTokens + 8];
    __shared__ unsigned long long best_of_warp[kFewThreads / 32];
    const uint32_t row = blockIdx.y, first = blockIdx.x * kFewTokens, n = min(kFewTokens, a.vocab - first);
    const Raw* in = reinterpret_cast<const Raw*>(a.in) + uint64_t(row) * a.in_stride + first;
    Raw* out = reinterpret_cast<Raw*>(a.out) + uint64_t(row) * a.out_stride + first;
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(in) & 15), off_out = uint32_t(reinterpret_cast<uintptr_t>(out) & 15);
    const uint32_t head = off == off_out ? min(n, uint32_t(((16 - off) & 15) / sizeof(Raw))) : n, vecs = (n - head) / P, shift = (P - head % P) % P;
    uint4 x[kVecs];
#pragma unroll
    for (int t = 0; t < kVecs; ++t) if (threadIdx.x + t * kFewThreads < vecs) x[t] = *(reinterpret_cast<const uint4*>(in + head) + threadIdx.x + t * kFewThreads);

    const Row what(a, row);
    const bool plain = what.h1 == what.h0 && what.nb == 0;
    if (!plain) {
        for (uint32_t i = threadIdx.x; i < (kFewTokens + 8) / 4; i += kFewThreads) reinterpret_cast<uint4*>(words)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        for (int i = threadIdx.x; i < what.nb; i += kFewThreads) {
            const uint32_t id = uint32_t(__ldg(a.s.bias_id + what.b0 + i));
            if (id >= a.vocab) report(a.err, beToken);
            else if (id - first < n) atomicMax(words + (id - first) + shift, uint32_t(i + 1) << 21);
        }
        if (what.nb) __syncthreads();                        // (the maximum is taken of whole words: counts follow)
        constexpr int kAhead = 4;
        for (int i0 = what.h0 + int(threadIdx.x); i0 < what.h1; i0 += kAhead * kFewThreads) {
            uint32_t id[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) id[k] = i0 + k * kFewThreads < what.h1 ? uint32_t(__ldg(a.s.history + i0 + k * kFewThreads)) : 0u;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = i0 + k * kFewThreads;
                if (i >= what.h1) continue;
                if (id[k] >= a.vocab) report(a.err, beToken);
                else if (id[k] - first < n) { uint32_t* w = words + (id[k] - first) + shift; if (i < what.prompt_end) atomicOr(w, kPrompt); else atomicAdd(w, 1u); }
            }
        }
        __syncthreads();
    }

    float best = -INFINITY;                                  // a thread meets its tokens in ascending order
    uint32_t best_at = 0;
    auto single = [&](uint32_t i) {
        Raw r = in[i];
        const uint32_t c = plain ? 0 : words[i + shift], v = first + i;
        if (c) r = E::put(what.shaped(a, E::get(r), c));
        if (what.mask && !((__ldg(what.mask + (v >> 5)) >> (v & 31)) & 1u)) r = E::put(-INFINITY);
        out[i] = r;
        if (E::get(r) > best) { best = E::get(r); best_at = v; }
    };
    for (uint32_t i = threadIdx.x; i < head; i += kFewThreads) single(i);
#pragma unroll
    for (int t = 0; t < kVecs; ++t) {
        const uint32_t j = threadIdx.x + t * kFewThreads, i = head + j * P;
        if (j >= vecs) continue;
        Raw e[P];
        if (!plain) {
            uint32_t c[P];
#pragma unroll
            for (uint32_t k = 0; k < P; k += 4) *reinterpret_cast<uint4*>(c + k) = *reinterpret_cast<const uint4*>(words + i + k + shift);
            uint32_t any = 0;
#pragma unroll
            for (uint32_t k = 0; k < P; ++k) any |= c[k];
            if (any) {
                memcpy(e, &x[t], 16);
#pragma unroll
                for (uint32_t k = 0; k < P; ++k) { const Raw r = E::put(what.shaped(a, E::get(e[k]), c[k])); e[k] = c[k] ? r : e[k]; }
                memcpy(&x[t], e, 16);
            }
        }
        if (what.mask) hide<DT>(x[t], what.mask, first + i);
        *reinterpret_cast<uint4*>(out + i) = x[t];
        const float top = E::last(E::max2(E::max2(x[t].x, x[t].y), E::max2(x[t].z, x[t].w)));
        if (top > best) {
            memcpy(e, &x[t], 16);
            best = top;
#pragma unroll
            for (int k = int(P) - 1; k >= 0; --k) if (E::get(e[k]) == top) best_at = first + i + k;
        }
    }
    for (uint32_t i = head + vecs * P + threadIdx.x; i < n; i += kFewThreads) single(i);
    if (a.token) settle<kFewThreads / 32>(a, row, best > -INFINITY ? (unsigned long long)(ordered(best)) << 32 | uint32_t(~best_at) : 0ull, best_of_warp);
}

}  // namespace

cudaError_t launch_shape_logits(const ShapeArgs& a, int dtype, cudaStream_t s)
{
    auto go = [&](auto type) -> cudaError_t {
        // Up to 2,048 blocks of 2,048 tokens a history counted as it comes is cheaper than one sorted (us a call, as it comes / sorted, 131,072 tokens and
        // 2,000 of history a row: 1 row of bf16 11.6 / 21.0, 16 rows 13.2 / 25.3, 32 rows (2,048 blocks) 21.8 / 27.3, without a history 13.2 / 12.4; 64 rows 34.7 / 35.5
        // and 21.1 / 15.0; f32 21.0 / 35.5, 13.3 / 14.5 and 33.5 / 45.9, 21.2 / 18.9): beyond, every block reads its row's history for too few tokens.
        const uint32_t few = (a.vocab + kFewTokens - 1) / kFewTokens;
        if (uint64_t(few) * a.n_rows <= 2048) {
            k_shape_few<decltype(type)::value><<<dim3(few, a.n_rows), kFewThreads, 0, s>>>(a);
            return cudaGetLastError();
        }
        constexpr auto kernel = k_shape_logits<decltype(type)::value>;
        if (cudaError_t e = allow_smem<kernel>(kSmem); e != cudaSuccess) return e;
        // Parts of a row: as many as give the GPU its blocks, of a slice per warp at least and kSlices at most.
        const uint32_t slices = (a.vocab + kTokens - 1) / kTokens, least = (slices + kSlices - 1) / kSlices, most = (slices + kWarps - 1) / kWarps;
        uint32_t parts = 148 * kBlocks / a.n_rows;
        parts = parts < least ? least : parts > most ? most : parts;
        kernel<<<dim3(parts, a.n_rows), kThreads, kSmem, s>>>(a);
        return cudaGetLastError();
    };
    using std::integral_constant;
    return dtype == WWWS_F32 ? go(integral_constant<int, WWWS_F32>()) : dtype == WWWS_BF16 ? go(integral_constant<int, WWWS_BF16>()) : go(integral_constant<int, WWWS_F16>());
}

}  // namespace wwws
