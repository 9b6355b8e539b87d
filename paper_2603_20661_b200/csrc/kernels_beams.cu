// Beam search's selection: of every request, the best continuations over its beams and the vocabulary.
//
// score(beam, v) = total_beam + x_v - log sum_w exp(x_w), compared in 64 bits, ties to the lowest (beam, token).
// Bound by HBM: the logits are read once and nothing else is long.
//   - Stream: a warp takes chunks of a row, 64 bytes a lane, the next chunk's loads in flight meanwhile, and keeps nothing but each chunk's maximum and, per lane, a
//     running maximum m and sum_w 2^((x_w - m) L), L = log2 e in fp32, two elements at a time; the logarithm is m + log2(sum) / L in 64 bits.  No barriers: blocks
//     that kept the best of their slices as they went spent two thirds of their time at them (256 rows of 131,072 bf16 logits: 42 us).
//   - Selection, by the last block of a request to arrive: the best `keep` elements lie in the `keep` chunks of largest maxima (in the order of score, beam,
//     token: each of these holds one at least as good as any element elsewhere).  Those are found among the threads' maxima, read again, mostly from L2, and what
//     reaches the last one's maximum is ranked by counting.
//   - Where more than kMost elements or chunks reach a bound (constant rows) the best element is taken out `keep` times, the best of every chunk being kept in the scratch.
//   - 256 rows of 131,072 bf16 logits: 25 us on the GPU, 2,700 GB/s; 256 rows of 50,021 in f16, 64 of 32 beams kept: 35 us, of which the joining is about 20; 4 rows of
//     32,003 in f32: 8 us.
//   - Element to lane goes by the token, not by the address: equal rows have equal sums to the bit, wherever they begin.  Rows off 16-byte boundaries are
//     read at these all the same and shifted, the rest of a piece coming from the next lane.
#include "backend.cuh"
#include "tcgen.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMost = 1024;              // chunks or elements that are ranked at once
constexpr int kVecs = 4;                 // 16-byte pieces of a lane and chunk
constexpr uint32_t kHeld = 2048;         // chunks of a request whose maxima are kept at hand
constexpr float kLog2e = 1.44269504f;

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// A sum relative to m as one relative to mn >= m; a NaN goes on into it.
__device__ __forceinline__ float part_of(float s, float m, float mn) { return s == 0.0f ? 0.0f : s * ex2((m - mn) * kLog2e); }

// Floats in the order of whole numbers (no NaN); 0 stands below all of them.
__device__ __forceinline__ uint32_t ordered(float x) { const uint32_t b = __float_as_uint(x); return b & 0x80000000u ? ~b : b | 0x80000000u; }
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t token) { return (unsigned long long)ordered(x + 0.0f) << 32 | ~token; }   // (-0 is 0)

template <int DT> struct Elem {
    static constexpr int kPer = DT == WWWS_F32 ? 4 : 8, kSize = DT == WWWS_F32 ? 4 : 2;      // elements of 16 bytes
    static constexpr uint32_t kChunk = kVecs * 32 * kPer;                                    // tokens
    static constexpr uint32_t kNone = DT == WWWS_F32 ? 0xff800000u : DT == WWWS_BF16 ? 0xff80ff80u : 0xfc00fc00u;      // -infinity
    static __device__ __forceinline__ float at(const uint4& v, int e)
    {
        const uint32_t w[4] = { v.x, v.y, v.z, v.w };
        if constexpr (DT == WWWS_F32) return __uint_as_float(w[e]);
        else return e % 2 ? Act<DT == WWWS_BF16>::hi(w[e / 2]) : Act<DT == WWWS_BF16>::lo(w[e / 2]);
    }
    // the larger of two words, element by element; a NaN only if both are
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        uint32_t r;
        if constexpr (DT == WWWS_F32) r = __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        else if constexpr (DT == WWWS_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float element(const uint8_t* row, uint32_t token)
    {
        if constexpr (DT == WWWS_F32) return __ldg(reinterpret_cast<const float*>(row) + token);
        else return Act<DT == WWWS_BF16>::lo(__ldg(reinterpret_cast<const uint16_t*>(row) + token));
    }
    static __device__ __forceinline__ float largest(uint32_t w)
    {
        if constexpr (DT == WWWS_F32) return __uint_as_float(w);
        else return fmaxf(Act<DT == WWWS_BF16>::lo(w), Act<DT == WWWS_BF16>::hi(w));
    }
    static __device__ __forceinline__ float largest(const uint4& v) { return largest(larger(larger(v.x, v.y), larger(v.z, v.w))); }
};

// The pieces of a chunk that this lane holds, as they lie in memory: 16 bytes at a 16-byte boundary, -infinity in the place of what is not the row's.
// In a skewed row piece u begins `skew` bytes before the lane's tokens, which end in the next lane's piece (lane 31: in the first lane's next one).
template <int DT, bool kSkewed> struct Pieces {
    using E = Elem<DT>;
    uint4 raw[kVecs], behind;                    // behind: of lane 0, what follows the chunk

    static __device__ __forceinline__ uint4 piece(const uint8_t* row, int64_t at, uint32_t vocab)      // `at`: token at which the 16 bytes begin
    {
        if (at >= 0 && at + E::kPer <= int64_t(vocab)) return __ldg(reinterpret_cast<const uint4*>(row + at * E::kSize));
        uint32_t w[4] = { E::kNone, E::kNone, E::kNone, E::kNone };
#pragma unroll
        for (int e = 0; e < E::kPer; ++e)
            if (at + e >= 0 && at + e < int64_t(vocab)) {
                if constexpr (DT == WWWS_F32) w[e] = __ldg(reinterpret_cast<const uint32_t*>(row) + at + e);
                else {
                    const uint32_t h = __ldg(reinterpret_cast<const uint16_t*>(row) + at + e);
                    w[e / 2] = e % 2 ? (w[e / 2] & 0xffffu) | h << 16 : (w[e / 2] & 0xffff0000u) | h;
                }
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void load(const uint8_t* row, uint32_t skew, uint32_t c, uint32_t lane, uint32_t vocab)
    {
        const int64_t first = int64_t(c) * E::kChunk - (kSkewed ? int(skew / E::kSize) : 0), at = first + lane * E::kPer;
        if (first >= 0 && first + E::kChunk + (kSkewed ? E::kPer : 0) <= int64_t(vocab)) {           // (the same for the whole warp)
            const uint4* from = reinterpret_cast<const uint4*>(row + at * E::kSize);
#pragma unroll
            for (int u = 0; u < kVecs; ++u) raw[u] = __ldg(from + u * 32);
            if constexpr (kSkewed) if (lane == 0) behind = __ldg(from + kVecs * 32);
        } else {
#pragma unroll 1
            for (int u = 0; u < kVecs + (kSkewed && lane == 0); ++u) {
                const uint4 v = piece(row, at + u * 32 * E::kPer, vocab);
#pragma unroll
                for (int k = 0; k < kVecs; ++k) if (u == k) raw[k] = v;
                if (u == kVecs) behind = v;
            }
        }
    }
    __device__ __forceinline__ void take(uint4 (&x)[kVecs], uint32_t skew, uint32_t lane) const
    {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) x[u] = raw[u];
        if constexpr (kSkewed) {
            if (skew == 0) return;
#pragma unroll
            for (int u = 0; u < kVecs; ++u) x[u] = shifted(raw[u], lane == 0 ? (u + 1 < kVecs ? raw[u + 1 < kVecs ? u + 1 : 0] : behind) : raw[u], skew, lane);
        }
    }
    // the lane's tokens from its 16 bytes and the next lane's, who gives `give`
    static __device__ __forceinline__ uint4 shifted(const uint4& raw, const uint4& give, uint32_t skew, uint32_t lane)
    {
        uint32_t w0 = raw.x, w1 = raw.y, w2 = raw.z, w3 = raw.w;
        uint32_t w4 = __shfl_sync(0xffffffffu, give.x, (lane + 1) & 31), w5 = __shfl_sync(0xffffffffu, give.y, (lane + 1) & 31), w6 = __shfl_sync(0xffffffffu, give.z, (lane + 1) & 31);
        const uint32_t w7 = __shfl_sync(0xffffffffu, give.w, (lane + 1) & 31), by = (skew & 2) * 8;
        if (skew == 0) return raw;
        if (skew & 8) { w0 = w2; w1 = w3; w2 = w4; w3 = w5; w4 = w6; w5 = w7; }
        if (skew & 4) { w0 = w1; w1 = w2; w2 = w3; w3 = w4; w4 = w5; }
        return make_uint4(__funnelshift_r(w0, w1, by), __funnelshift_r(w1, w2, by), __funnelshift_r(w2, w3, by), __funnelshift_r(w3, w4, by));
    }
};

template <int DT, bool kSkewed> struct Row {
    const uint8_t* base; uint32_t skew;
    __device__ __forceinline__ Row(const BeamArgs& a, uint32_t row)
    {
        base = a.in + uint64_t(row) * a.stride * Elem<DT>::kSize;
        skew = kSkewed ? uint32_t(reinterpret_cast<uintptr_t>(base) & 15) : 0;
    }
    __device__ __forceinline__ void chunk(uint4 (&x)[kVecs], uint32_t c, uint32_t lane, uint32_t vocab) const
    {
        Pieces<DT, kSkewed> p;
        p.load(base, skew, c, lane, vocab);
        p.take(x, skew, lane);
    }
};

// 64-bit floats in the order of whole numbers; 0 stands below all of them.  (Scores are worked out in 64-bit floats and compared as whole numbers: the joining of a
// request of 4 beams took 20 us with comparisons on the 64-bit unit.)
__device__ __forceinline__ unsigned long long ordered(double y) { const long long b = __double_as_longlong(y); return b < 0 ? ~b : b | (1ll << 63); }
__device__ __forceinline__ double unordered(unsigned long long k) { return __longlong_as_double(k >> 63 ? k & ~(1ull << 63) : ~k); }
__device__ __forceinline__ float to_float(unsigned long long k) { return k ? float(unordered(k)) : -INFINITY; }           // (rounding keeps the order)

// (ordered score, id) in the order of the result: the larger score, then the lower id (beam, then token or chunk).
struct Best { unsigned long long y, id; };
__device__ __forceinline__ bool before(unsigned long long y, unsigned long long id, unsigned long long z, unsigned long long jd) { return y > z || (y == z && id < jd); }

struct Joint {                                                                                   // shared memory of a block that joins a request
    Best found[kMost];
    Best chunk[kMaxKeep];                                                                        // the best chunks
    double lse[kMaxBeams];
    float off[kMaxBeams];                                                                        // total - lse, about
    float tops[kThreads];
    float held[kHeld];
    uint32_t piece[kMaxKeep * kVecs];                                                            // (best chunk, piece of it)
    float x_least[kMaxKeep];
    float bound;
    uint32_t n, n_pieces;
};

// What is largest of the block's (y, id), for all threads.
__device__ Best block_best(Joint& s, unsigned long long y, unsigned long long id)
{
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const unsigned long long z = __shfl_xor_sync(0xffffffffu, y, k), jd = __shfl_xor_sync(0xffffffffu, id, k);
        if (before(z, jd, y, id)) { y = z; id = jd; }
    }
    __syncthreads();
    if (threadIdx.x % 32 == 0) s.found[threadIdx.x / 32] = Best{ y, id };
    __syncthreads();
    Best b = s.found[0];
    for (int w = 1; w < kWarps; ++w) if (const Best o = s.found[w]; before(o.y, o.id, b.y, b.id)) b = o;
    return b;
}

// The score of a logit of beam b, ordered; 0: none.
__device__ __forceinline__ unsigned long long score_of(const BeamArgs& a, const Joint& s, uint32_t seq, uint32_t b, float x)
{
    const double y = double(__ldg(a.total + uint64_t(seq) * a.beams + b)) + (double(x) - s.lse[b]);
    return x > -INFINITY && y > double(-INFINITY) ? ordered(y) : 0;
}
__device__ __forceinline__ void put(const BeamArgs& a, uint32_t seq, uint32_t r, unsigned long long y, unsigned long long id)
{
    const uint64_t to = uint64_t(seq) * a.keep + r;
    a.score[to] = to_float(y);
    a.parent[to] = y ? int32_t(seq * a.beams + uint32_t(id >> 32)) : -1; a.token[to] = y ? int32_t(uint32_t(id)) : -1;
}

template <int DT, bool kSkewed> __device__ __noinline__ void join_slowly(const BeamArgs& a, uint32_t seq, Joint& s)
{
    using E = Elem<DT>;
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, n = a.beams * a.chunks;
    auto score = [&](uint32_t b, float x) { return score_of(a, s, seq, b, x); };
    // Too many at a bound: the best element of every chunk, then the best of these `keep` times over, its chunk looked through again for what comes behind it.
    unsigned long long* heads = a.heads + uint64_t(seq) * n;
    // The best element of chunk i behind the one of logit `last` at `last_token`, by a warp; the first of all where last is infinite.  By score, not by logit: beside a large
    // total unequal logits may have equal scores.  Scores do not fall as logits rise, and logits further apart than `near` have different ones (two roundings of
    // 2^-53 of numbers no larger than the terms together, on either side), so 64-bit scores are worked out for unequal logits nearer than that alone.
    auto head = [&](uint32_t i, float last, uint32_t last_token) {
        const uint32_t b = i / a.chunks, c = i - b * a.chunks;
        uint4 x[kVecs];
        Row<DT, kSkewed>(a, seq * a.beams + b).chunk(x, c, lane, a.vocab);
        const float terms = fabsf(__ldg(a.total + uint64_t(seq) * a.beams + b)) + fabsf(float(s.lse[b]));
        auto near = [&](float v) { return (fabsf(v) + terms) * 0x1p-50f; };
        const float under = last < INFINITY ? __fsub_rd(last, near(last)) : last, over = last < INFINITY ? __fadd_ru(last, near(last)) : last;
        const unsigned long long last_y = score(b, last);
        auto token_of = [&](int u, int e) { return c * E::kChunk + (u * 32 + lane) * E::kPer + e; };
        uint32_t left = 0;                                       // elements behind the last one, a bit each
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < kVecs; ++u)
#pragma unroll
            for (int e = 0; e < E::kPer; ++e) {
                const float v = E::at(x[u], e);
                bool mine = v < under;
                if (v == last) mine = token_of(u, e) > last_token;
                else if (!mine && !(v > over)) { const unsigned long long y = score(b, v); mine = y && before(last_y, last_token, y, token_of(u, e)); }
                left |= uint32_t(mine) << (u * E::kPer + e);
                if (mine) most = fmaxf(most, v);
            }
        most = unordered(__reduce_max_sync(0xffffffffu, ordered(most + 0.0f)));
        const unsigned long long y = score(b, most);
        const float least = __fsub_rd(most, near(most));
        uint32_t token = ~0u;
        float w = 0.0f;
#pragma unroll
        for (int u = kVecs - 1; u >= 0; --u)
#pragma unroll
            for (int e = E::kPer - 1; e >= 0; --e) {
                const float v = E::at(x[u], e);
                if (left >> (u * E::kPer + e) & 1u && !(v < least) && (v == most || score(b, v) == y)) { token = token_of(u, e); w = v; }
            }
        const uint32_t first = __reduce_min_sync(0xffffffffu, token);
        if (first == ~0u || y == 0) { if (lane == 0) heads[i] = 0; }
        else if (token == first) heads[i] = key_of(w, token);
    };
    for (uint32_t i = warp; i < n; i += kWarps) head(i, INFINITY, 0);
    for (uint32_t r = 0; r < a.keep; ++r) {
        __syncthreads();                                                                         // (orders the block's writes to the heads too)
        unsigned long long best = 0, id = ~0ull;
        for (uint32_t i = tid; i < n; i += kThreads) {
            const unsigned long long k = __ldcg(heads + i);
            const uint32_t b = i / a.chunks;
            const unsigned long long z = k ? score(b, unordered(uint32_t(k >> 32))) : 0, jd = (unsigned long long)b << 32 | uint32_t(~k);
            if (z && before(z, jd, best, id)) { best = z; id = jd; }
        }
        const Best w = block_best(s, best, id);
        if (tid == 0) put(a, seq, r, w.y, w.id);
        if (w.y && warp == 0) {
            const uint32_t b = uint32_t(w.id >> 32), token = uint32_t(w.id), i = b * a.chunks + token / E::kChunk;
            const unsigned long long k = __ldcg(heads + i);
            __syncwarp();
            head(i, unordered(uint32_t(k >> 32)), token);
        }
    }
}

template <int DT, bool kSkewed> __device__ void join(const BeamArgs& a, uint32_t seq, Joint& s)
{
    using E = Elem<DT>;
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, n = a.beams * a.chunks;
    const float2* stat = a.stat + uint64_t(seq) * a.beams * a.slices;
    const float4* top = a.top + uint64_t(seq) * n;
    const float* total = a.total + uint64_t(seq) * a.beams;
    if (tid == 0) s.n = 0;
    // the chunks' maxima, kHeld of them in shared memory
    auto look = [&](uint32_t i) { const float4 v = __ldcg(top + i); return fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)); };
#pragma unroll 4
    for (uint32_t i = tid; i < min(n, kHeld); i += kThreads) s.held[i] = look(i);
#pragma unroll 1
    for (uint32_t b = tid / 8; b < (a.beams + 31) / 32 * 32; b += kThreads / 8) {                // 8 lanes per row
        float m = -INFINITY, sum = 0.0f;
        if (b < a.beams)
            for (uint32_t k = tid % 8; k < a.slices; k += 8) {
                const float2 p = __ldcg(&stat[b * a.slices + k]);
                const float mn = fmaxf(m, p.x);
                sum = part_of(sum, m, mn) + part_of(p.y, p.x, mn);
                m = mn;
            }
#pragma unroll
        for (int k = 1; k < 8; k <<= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, m, k), os = __shfl_xor_sync(0xffffffffu, sum, k), mn = fmaxf(m, om);
            sum = part_of(sum, m, mn) + part_of(os, om, mn);
            m = mn;
        }
        // log2 of the sum as its exponent and the logarithm of 0.75 .. 1.5, whose fp32 error is 2^-24
        const int e = int((__float_as_uint(sum) - 0x3f400000u)) >> 23;
        const float rest = __uint_as_float(__float_as_uint(sum) - (uint32_t(e) << 23));
        if (tid % 8 == 0 && b < a.beams) {
            const double lse = sum > 0.0f && sum < INFINITY ? double(m) + (double(e) + double(log2f(rest))) * (1.0 / double(kLog2e)) : double(NAN);      // NaN: the row counts for nothing
            s.lse[b] = lse;
            s.off[b] = float(double(__ldg(total + b)) - lse);
        }
    }
    __syncthreads();
    auto score = [&](uint32_t b, float x) { return score_of(a, s, seq, b, x); };
    // f(rank, entry) of what was found: an entry is compared by 4, 2 or 1 threads
    auto ranked = [&](uint32_t found, auto&& f) {
        const uint32_t by = found <= kThreads / 4 ? 4 : found <= kThreads / 2 ? 2 : 1;
#pragma unroll 1
        for (uint32_t base = 0; base < found; base += kThreads / by) {
            const uint32_t i = base + tid / by;
            const Best o = s.found[min(i, found - 1)];
            uint32_t r = 0;
#pragma unroll 4
            for (uint32_t j = tid % by; j < found; j += by) r += before(s.found[j].y, s.found[j].id, o.y, o.id);
            if (by >= 2) r += __shfl_xor_sync(0xffffffffu, r, 1);
            if (by >= 4) r += __shfl_xor_sync(0xffffffffu, r, 2);
            if (i < found && tid % by == 0) f(r, o);
        }
    };
    // Scores in fp32, as bounds on either side: three roundings of numbers no larger than the two terms, so 2^-22 of them is more than they are off.
    auto about = [&](uint32_t i, float x, float side) {
        const float off = s.off[i / a.chunks], y = x + off + side * (fabsf(x) + fabsf(off)) * 0x1p-22f;
        return !(x > -INFINITY && off == off) ? -INFINITY : y == y ? y : side * INFINITY;            // (beyond fp32's range no bound is one on either side)
    };
    auto largest = [&](uint32_t i) { return i < kHeld ? s.held[i] : look(i); };
    // Lower bounds, their maxima in groups of threads (about four times as many as are kept): the keep-th largest bounds the best chunks from below.
    float least_here = -INFINITY, most_here = -INFINITY;
#pragma unroll 1
    for (uint32_t i = tid; i < n; i += kThreads) {
        const float x = largest(i);
        least_here = fmaxf(least_here, about(i, x, -1.0f)); most_here = fmaxf(most_here, about(i, x, 1.0f));
    }
    const uint32_t size = a.keep <= 32 ? 4 : a.keep <= 64 ? 2 : 1, each = kThreads / size / size;      // threads of a group; values that each of them compares
    float t = least_here;
    if (size >= 2) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
    if (size >= 4) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
    const uint32_t me = tid / size, from = tid % size * each;
    if (tid % size == 0) s.tops[me] = t;
    __syncthreads();
    uint32_t rank = 0;
#pragma unroll 1
    for (uint32_t j = from; j < from + each; j += 4) {
        const float4 o = *reinterpret_cast<const float4*>(s.tops + j);
        rank += (o.x > t || (o.x == t && j < me)) + (o.y > t || (o.y == t && j + 1 < me)) + (o.z > t || (o.z == t && j + 2 < me)) + (o.w > t || (o.w == t && j + 3 < me));
    }
    if (size >= 2) rank += __shfl_xor_sync(0xffffffffu, rank, 1);
    if (size >= 4) rank += __shfl_xor_sync(0xffffffffu, rank, 2);
    if (rank == a.keep - 1) s.bound = t;
    __syncthreads();
    const float bound = s.bound;
    if (most_here >= bound)
#pragma unroll 1
        for (uint32_t i = tid; i < n; i += kThreads) {
            const float x = largest(i);
            if (about(i, x, 1.0f) >= bound)
                if (const unsigned long long z = score(i / a.chunks, x)) {
                    const uint32_t at = atomicAdd(&s.n, 1u);
                    if (at < kMost) s.found[at] = Best{ z, i };
                }
        }
    __syncthreads();
    uint32_t found = s.n;
    if (found <= kMost) {
        ranked(found, [&](uint32_t r, const Best& o) { if (r < a.keep) s.chunk[r] = o; });
        __syncthreads();
        if (tid == 0) s.n = s.n_pieces = 0;
        const uint32_t n_chunks = min(found, a.keep);
        const unsigned long long least = n_chunks == a.keep ? s.chunk[a.keep - 1].y : 1;         // as many elements reach it
        __syncthreads();
        // the pieces of these chunks that have such elements, and the least logit that may be one (in fp32, with the same allowance)
        for (uint32_t k = tid; k < n_chunks * kVecs; k += kThreads) {
            const uint32_t i = uint32_t(s.chunk[k / kVecs].id), b = i / a.chunks;
            const float off = s.off[b], y = to_float(least) - off, x_least = n_chunks < a.keep ? -INFINITY : y - (fabsf(y) + 2.0f * fabsf(off)) * 0x1p-22f;
            if (k % kVecs == 0) s.x_least[k / kVecs] = x_least;
            if (const float x = reinterpret_cast<const float*>(top + i)[k % kVecs]; x > -INFINITY && !(x < x_least)) s.piece[atomicAdd(&s.n_pieces, 1u)] = k;
        }
        __syncthreads();
        // Pieces are read element by element, a lane's at intervals of 32, two pieces of a warp at a time.
        const uint32_t pieces = s.n_pieces;
#pragma unroll 1
        for (uint32_t p0 = 2 * warp; p0 < pieces; p0 += 2 * kWarps) {
            float v[2][E::kPer];
            uint32_t token[2], beam[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t k = s.piece[min(p0 + j, pieces - 1)], i = uint32_t(s.chunk[k / kVecs].id);
                beam[j] = i / a.chunks;
                token[j] = (i - beam[j] * a.chunks) * E::kChunk + k % kVecs * 32 * E::kPer + lane;
                const uint8_t* row = a.in + uint64_t(seq * a.beams + beam[j]) * a.stride * E::kSize;
#pragma unroll
                for (int e = 0; e < E::kPer; ++e) v[j][e] = token[j] + e * 32 < a.vocab ? E::element(row, token[j] + e * 32) : -INFINITY;
            }
            uint32_t hit = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float x_least = p0 + j < pieces ? s.x_least[s.piece[p0 + j] / kVecs] : INFINITY;
#pragma unroll
                for (int e = 0; e < E::kPer; ++e) hit |= uint32_t(!(v[j][e] < x_least)) << (j * E::kPer + e);
            }
            if (p0 + 1 >= pieces) hit &= (1u << E::kPer) - 1;
#pragma unroll 1
            while (hit) {
                const int at = __ffs(hit) - 1, j = at / E::kPer, e = at % E::kPer;
                hit &= hit - 1;
                float w = v[0][0];
#pragma unroll
                for (int q = 1; q < 2 * E::kPer; ++q) if (at == q) w = v[q / E::kPer][q % E::kPer];
                const uint32_t b = j ? beam[1] : beam[0];
                if (const unsigned long long z = score(b, w); z >= least) {
                    const uint32_t to = atomicAdd(&s.n, 1u);
                    if (to < kMost) s.found[to] = Best{ z, (unsigned long long)b << 32 | ((j ? token[1] : token[0]) + uint32_t(e) * 32) };
                }
            }
        }
        __syncthreads();
        found = s.n;
        if (found <= kMost) {
            ranked(found, [&](uint32_t r, const Best& o) { if (r < a.keep) put(a, seq, r, o.y, o.id); });
            for (uint32_t r = found + tid; r < a.keep; r += kThreads) put(a, seq, r, 0, 0);
            return;
        }
    }
    join_slowly<DT, kSkewed>(a, seq, s);
}

template <int DT, bool kSkewed> __global__ void __launch_bounds__(kThreads, 4) k_beams(BeamArgs a)
{
    using E = Elem<DT>;
    __shared__ __align__(16) unsigned char shared[sizeof(Joint)];
    __shared__ float2 parts[kWarps];
    __shared__ uint32_t last_flag;
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const uint32_t slice = blockIdx.x, row = blockIdx.y, seq = row / a.beams;
    const float total = __ldg(a.total + row);
    const uint32_t c0 = slice * a.per_slice + warp, c1 = min(a.chunks, (slice + 1) * a.per_slice);
    float4* top = a.top + uint64_t(row) * a.chunks;
    float m = -INFINITY, s = 0.0f;
    if (fabsf(total) < INFINITY) {
        const Row<DT, kSkewed> from(a, row);
        Pieces<DT, kSkewed> next;
        if (c0 < c1) next.load(from.base, from.skew, c0, lane, a.vocab);
        uint64_t sum = pack2(0.0f, 0.0f);
        for (uint32_t c = c0; c < c1; c += kWarps) {
            uint4 x[kVecs];
            next.take(x, from.skew, lane);
            if (c + kWarps < c1) next.load(from.base, from.skew, c + kWarps, lane, a.vocab);
            float y = -INFINITY;
            uint32_t best[kVecs];
#pragma unroll
            for (int u = 0; u < kVecs; ++u) { const float t = fmaxf(-INFINITY, E::largest(x[u])); y = fmaxf(y, t); best[u] = __reduce_max_sync(0xffffffffu, ordered(t)); }
            if (lane == 0) top[c] = make_float4(unordered(best[0]), unordered(best[1]), unordered(best[2]), unordered(best[3]));
            if (y > m) {
                const float less = ex2((m - y) * kLog2e);          // (0 the first time)
                sum = mul2(sum, pack2(less, less)); m = y;
            }
            const float mm = m == -INFINITY ? 0.0f : m;
            const uint64_t less = pack2(-mm, -mm), by = pack2(kLog2e, kLog2e);
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
                for (int e = 0; e < E::kPer; e += 2) {
                    float y0, y1;
                    unpack2(mul2(add2(pack2(E::at(x[u], e), E::at(x[u], e + 1)), less), by), y0, y1);
                    sum = add2(sum, pack2(ex2(y0), ex2(y1)));
                }
        }
        float s0, s1;
        unpack2(sum, s0, s1);
        s = s0 + s1;
    } else if (lane == 0)
        for (uint32_t c = c0; c < c1; c += kWarps) top[c] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    // the slice's maximum and sum
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, k), os = __shfl_xor_sync(0xffffffffu, s, k), mn = fmaxf(m, om);
        s = part_of(s, m, mn) + part_of(os, om, mn);
        m = mn;
    }
    if (lane == 0) parts[warp] = make_float2(m, s);
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kWarps; ++w) {
            const float2 o = parts[w];
            const float mn = fmaxf(m, o.x);
            s = part_of(s, m, mn) + part_of(o.y, o.x, mn);
            m = mn;
        }
        __stcg(a.stat + uint64_t(row) * a.slices + slice, make_float2(m, s));
        __threadfence();                                           // (the other threads' maxima too: they came before the barrier)
        last_flag = atomicAdd(&a.ticket[seq], 1u) == a.beams * a.slices - 1;
    }
    __syncthreads();
    if (last_flag) {
        __threadfence();
        join<DT, kSkewed>(a, seq, *reinterpret_cast<Joint*>(shared));
        if (tid == 0) a.ticket[seq] = 0;
    }
}

uint32_t chunks_of(uint32_t vocab, int dtype)
{
    const uint32_t chunk = dtype == WWWS_F32 ? Elem<WWWS_F32>::kChunk : Elem<WWWS_BF16>::kChunk;
    return (vocab + chunk - 1) / chunk;
}
// Chunks of a slice: whole rounds of a block's warps, as many as leave the GPU about four blocks an SM, in one wave.
uint32_t slice_of(uint32_t rows, uint32_t vocab, int dtype)
{
    const uint32_t rounds = (chunks_of(vocab, dtype) + kWarps - 1) / kWarps, slices = rows && rows < 148 * 4 ? 148 * 4 / rows : 1;
    return (rounds + slices - 1) / slices * kWarps;
}

}  // namespace

uint64_t beams_scratch(uint32_t rows, uint32_t vocab, int dtype)
{
    const uint64_t chunks = chunks_of(vocab, dtype), per = slice_of(rows, vocab, dtype);
    return rows * (8 * ((chunks + per - 1) / per) + (16 + 8) * chunks);
}

cudaError_t launch_beams(BeamArgs a, uint32_t rows, int dtype, void* scratch, cudaStream_t s)
{
    a.chunks = chunks_of(a.vocab, dtype);
    a.per_slice = slice_of(rows, a.vocab, dtype);
    a.slices = (a.chunks + a.per_slice - 1) / a.per_slice;
    a.top = static_cast<float4*>(scratch);
    a.heads = reinterpret_cast<unsigned long long*>(a.top + uint64_t(rows) * a.chunks);
    a.stat = reinterpret_cast<float2*>(a.heads + uint64_t(rows) * a.chunks);
    const bool skewed = (reinterpret_cast<uintptr_t>(a.in) | (rows > 1 ? a.stride * (dtype == WWWS_F32 ? 4 : 2) : 0)) & 15;
    const dim3 grid(a.slices, rows);
    auto go = [&](auto dt) {
        if (skewed) k_beams<decltype(dt)::value, true><<<grid, kThreads, 0, s>>>(a);
        else k_beams<decltype(dt)::value, false><<<grid, kThreads, 0, s>>>(a);
        return cudaGetLastError();
    };
    using std::integral_constant;
    return dtype == WWWS_F32 ? go(integral_constant<int, WWWS_F32>()) : dtype == WWWS_BF16 ? go(integral_constant<int, WWWS_BF16>()) : go(integral_constant<int, WWWS_F16>());
}

}  // namespace wwws
