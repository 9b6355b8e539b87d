// Beam search's selection: of every request, the best continuations over its beams and the vocabulary.
//
// score(beam, v) = total_beam + x_v - log sum_w exp(x_w).  Within a beam the order is that of the logits, so a block takes a slice of one row, keeps its
// `keep` best logits and its part of the sum, and the last block of a request to arrive joins the slices: the rows' sums, then the best scores, in 64 bits.
// Bound by HBM: the logits are read once (into registers, a slice is 256 threads * kVecs * 16 bytes) and nothing else is long.
//   - Sum: sum_w 2^((x_w - m) L), m the slice's largest, L = log2 e in fp32, two elements at a time; the logarithm is m + log2(sum) / L in 64 bits.
//   - Selection in one pass over registers: of 64 (or 256) groups of threads the keep-th largest maximum is a bound that at least `keep` elements
//     reach, and hardly more do (-64 ln(1 - keep / 64) of them on random data); these are ranked by counting.  Keys are (value, lowest index first), all different,
//     so neither the ranks nor the result depend on the order of arrival.  Slices with more than kMost elements at the bound (constant rows) take
//     the largest key `keep` times instead.
#include "backend.cuh"
#include "tcgen.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 256;
constexpr int kMost = 1024;              // elements at or above a bound that are ranked at once
constexpr float kLog2e = 1.44269504f;

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// Floats in the order of whole numbers (no NaN); 0 stands below all of them.
__device__ __forceinline__ uint32_t ordered(float x) { const uint32_t b = __float_as_uint(x); return b & 0x80000000u ? ~b : b | 0x80000000u; }
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t token) { return (unsigned long long)ordered(x + 0.0f) << 32 | ~token; }   // (-0 is 0)

template <int DT> struct Elem {
    static constexpr int kPer = DT == WWWS_F32 ? 4 : 8, kSize = DT == WWWS_F32 ? 4 : 2;      // elements of 16 bytes
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
    static __device__ __forceinline__ float largest(uint32_t w)
    {
        if constexpr (DT == WWWS_F32) return __uint_as_float(w);
        else return fmaxf(Act<DT == WWWS_BF16>::lo(w), Act<DT == WWWS_BF16>::hi(w));
    }
};

// The best of the request's parts, by a whole block.
__device__ void join(const BeamArgs& a, uint32_t seq, unsigned char* shared)
{
    double* score_of = reinterpret_cast<double*>(shared);                                        // [kMost]
    unsigned long long* id_of = reinterpret_cast<unsigned long long*>(shared + 8 * kMost);       // [kMost] beam, token
    __shared__ double lse[kMaxBeams], tops[kThreads];
    __shared__ uint32_t n_found;
    __shared__ double bound_s;
    const uint32_t tid = threadIdx.x, lists = a.beams * a.slices, n = lists * a.keep;
    const float2* stat = a.stat + uint64_t(seq) * lists;
    const unsigned long long* keys = a.keys + uint64_t(seq) * n;
    for (uint32_t b = tid; b < a.beams; b += kThreads) {
        float c = -INFINITY;
        for (uint32_t s = 0; s < a.slices; ++s) c = fmaxf(c, __ldcg(&stat[b * a.slices + s].x));
        double sum = 0.0;
        for (uint32_t s = 0; s < a.slices; ++s) {
            const float2 p = __ldcg(&stat[b * a.slices + s]);
            if (!(p.y == 0.0f)) sum += double(p.y) * exp2((double(p.x) - double(c)) * double(kLog2e));              // (a NaN goes on into the sum)
        }
        lse[b] = double(c) + log2(sum) / double(kLog2e);                                         // a row without a sum: NaN, and none of its scores counts
    }
    if (tid == 0) n_found = 0;
    __syncthreads();
    auto score = [&](uint32_t i, unsigned long long& id) {
        const unsigned long long key = __ldcg(keys + i);
        const uint32_t b = i % lists / a.slices;
        id = (unsigned long long)b << 32 | uint32_t(~key);
        const double y = double(__ldg(a.total + uint64_t(seq) * a.beams + b)) + (double(unordered(uint32_t(key >> 32))) - lse[b]);
        return key == 0 || !(y > -INFINITY) ? -INFINITY : y;
    };
    double top = -INFINITY;
    unsigned long long id;
    for (uint32_t i = tid; i < n; i += kThreads) { const double y = score(i, id); top = y > top ? y : top; }
    tops[tid] = top;
    __syncthreads();
    uint32_t rank = 0;
    for (uint32_t j = 0; j < kThreads; ++j) rank += tops[j] > top || (tops[j] == top && j < tid);
    if (rank == a.keep - 1) bound_s = top;
    __syncthreads();
    const double bound = bound_s;
    if (top >= bound)
        for (uint32_t i = tid; i < n; i += kThreads) {
            const double y = score(i, id);
            if (y >= bound && y > -INFINITY) {
                const uint32_t at = atomicAdd(&n_found, 1u);
                if (at < kMost) { score_of[at] = y; id_of[at] = id; }
            }
        }
    __syncthreads();
    uint32_t found = n_found;
    auto put = [&](uint32_t r, double y, unsigned long long w) {
        const uint64_t to = uint64_t(seq) * a.keep + r;
        a.score[to] = float(y); a.parent[to] = int32_t(seq * a.beams + uint32_t(w >> 32)); a.token[to] = int32_t(uint32_t(w));
    };
    if (found > kMost) {                 // the best one, `keep` times over
        double last = INFINITY; unsigned long long last_id = 0; bool any = true, begun = false;
        for (uint32_t r = 0; r < a.keep; ++r) {
            double best = -INFINITY; unsigned long long best_id = ~0ull;
            if (any)
                for (uint32_t i = tid; i < n; i += kThreads) {
                    const double y = score(i, id);
                    if (begun && !(y < last || (y == last && id > last_id))) continue;
                    if (y > best || (y == best && id < best_id)) { best = y; best_id = id; }
                }
            __syncthreads();
            score_of[tid] = best; id_of[tid] = best_id;
            __syncthreads();
            for (uint32_t k = kThreads / 2; k; k >>= 1) {
                if (tid < k && (score_of[tid + k] > score_of[tid] || (score_of[tid + k] == score_of[tid] && id_of[tid + k] < id_of[tid]))) { score_of[tid] = score_of[tid + k]; id_of[tid] = id_of[tid + k]; }
                __syncthreads();
            }
            last = score_of[0]; last_id = id_of[0]; begun = true;
            any = last > -INFINITY;
            if (any && tid == 0) put(r, last, last_id);
        }
        return;                          // (more than kMost >= keep of them are above -infinity)
    }
    for (uint32_t i = tid; i < found; i += kThreads) {
        const double y = score_of[i]; const unsigned long long w = id_of[i];
        uint32_t r = 0;
        for (uint32_t j = 0; j < found; ++j) r += score_of[j] > y || (score_of[j] == y && id_of[j] < w);
        if (r < a.keep) put(r, y, w);
    }
    for (uint32_t r = found + tid; r < a.keep; r += kThreads) {
        const uint64_t to = uint64_t(seq) * a.keep + r;
        a.score[to] = -INFINITY; a.parent[to] = -1; a.token[to] = -1;
    }
}

template <int DT, int kVecs> __global__ void __launch_bounds__(kThreads) k_beams(BeamArgs a)
{
    using E = Elem<DT>;
    constexpr int P = E::kPer;
    __shared__ __align__(16) unsigned char shared[16 * kMost];
    __shared__ float tops[kThreads], parts[kThreads / 32];
    __shared__ uint32_t n_found, last_flag;
    __shared__ float bound_s;
    unsigned long long* found_keys = reinterpret_cast<unsigned long long*>(shared);
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const uint32_t slice = blockIdx.x, row = blockIdx.y, seq = row / a.beams, list = row % a.beams * a.slices + slice, lists = a.beams * a.slices;
    unsigned long long* keys = a.keys + uint64_t(seq) * lists * a.keep + list;                   // key r at r * lists: neighbouring lists lie side by side
    const float total = __ldg(a.total + row);
    if (tid == 0) n_found = 0;
    if (fabsf(total) < INFINITY) {
        const uint8_t* base = a.in + uint64_t(row) * a.stride * E::kSize;
        // Element e of piece u of this thread is token first + u * kThreads * P + e, wherever the row begins: equal rows have equal sums, to the bit.
        const uint32_t skew = uint32_t(reinterpret_cast<uintptr_t>(base) & 15);
        const uint32_t first = (slice * kVecs * kThreads + tid) * P;
        uint4 x[kVecs];
        auto edge = [&](uint32_t at) {                         // a piece that the row ends (or, from the middle of 16 bytes, begins) in
            uint32_t w[4] = { E::kNone, E::kNone, E::kNone, E::kNone };
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (at + e < a.vocab) {
                    if constexpr (DT == WWWS_F32) w[e] = __ldg(reinterpret_cast<const uint32_t*>(base) + at + e);
                    else {
                        const uint32_t h = __ldg(reinterpret_cast<const uint16_t*>(base) + at + e);
                        w[e / 2] = e % 2 ? (w[e / 2] & 0xffffu) | h << 16 : (w[e / 2] & 0xffff0000u) | h;
                    }
                }
            return make_uint4(w[0], w[1], w[2], w[3]);
        };
        if (skew == 0) {
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                const uint32_t at = first + u * kThreads * P;
                if (at + P <= a.vocab) x[u] = __ldcs(reinterpret_cast<const uint4*>(base + uint64_t(at) * E::kSize));
                else x[u] = edge(at);
            }
        } else {                                               // two neighbouring 16 bytes, the second from L1 as a rule, shifted
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                const uint32_t at = first + u * kThreads * P;
                if (at && at + 2 * P <= a.vocab) {
                    const uint4* from = reinterpret_cast<const uint4*>(base - skew + uint64_t(at) * E::kSize);
                    const uint4 lo = __ldg(from), hi = __ldg(from + 1);
                    uint32_t w0 = lo.x, w1 = lo.y, w2 = lo.z, w3 = lo.w, w4 = hi.x, w5 = hi.y, w6 = hi.z;
                    if (skew & 8) { w0 = w2; w1 = w3; w2 = w4; w3 = w5; w4 = w6; w5 = hi.w; }
                    if (skew & 4) { w0 = w1; w1 = w2; w2 = w3; w3 = w4; w4 = w5; }
                    const uint32_t by = (skew & 2) * 8;
                    x[u] = make_uint4(__funnelshift_r(w0, w1, by), __funnelshift_r(w1, w2, by), __funnelshift_r(w2, w3, by), __funnelshift_r(w3, w4, by));
                } else x[u] = edge(at);
            }
        }
        uint32_t most = E::kNone;
#pragma unroll
        for (int u = 0; u < kVecs; ++u) most = E::larger(E::larger(most, E::larger(x[u].x, x[u].y)), E::larger(x[u].z, x[u].w));
        const float mine = E::largest(most);
        // maxima of groups of threads, of warps, of the slice
        float m = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const uint32_t groups = a.keep <= 32 ? kThreads / 4 : kThreads;
        if (groups == kThreads) tops[tid] = mine; else if (tid % 4 == 0) tops[tid / 4] = m;
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
        if (lane == 0) parts[warp] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, parts[w]);
        if (tid < groups) {
            const float t = tops[tid];
            uint32_t rank = 0;
            for (uint32_t j = 0; j < groups; j += 4) {
                const float4 o = *reinterpret_cast<const float4*>(tops + j);
                rank += (o.x > t || (o.x == t && j < tid)) + (o.y > t || (o.y == t && j + 1 < tid)) + (o.z > t || (o.z == t && j + 2 < tid)) + (o.w > t || (o.w == t && j + 3 < tid));
            }
            if (rank == a.keep - 1) bound_s = t;
        }
        // the slice's part of the sum
        float s0 = 0.0f, s1 = 0.0f;
        if (m > -INFINITY) {
            const uint64_t less = pack2(-m, -m), by = pack2(kLog2e, kLog2e);
            uint64_t both = pack2(0.0f, 0.0f);
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
                for (int e = 0; e < P; e += 2) {
                    float y0, y1;
                    unpack2(mul2(add2(pack2(E::at(x[u], e), E::at(x[u], e + 1)), less), by), y0, y1);
                    both = add2(both, pack2(ex2(y0), ex2(y1)));
                }
            unpack2(both, s0, s1);
        } else {                                               // nothing above -infinity, but there may be NaN
#pragma unroll 1
            for (int e = 0; e < P; ++e)
#pragma unroll
                for (int u = 0; u < kVecs; ++u) if (const float v = E::at(x[u], e); v != v) s0 = v;
        }
        float sum = s0 + s1;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        __syncthreads();                                       // the maxima are read, the bound is written
        if (lane == 0) parts[warp] = sum;
        const float bound = bound_s;
        if (mine >= bound && mine > -INFINITY) {
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float v = E::at(x[u], e);
                    if (v >= bound && v > -INFINITY) {
                        const uint32_t at = atomicAdd(&n_found, 1u);
                        if (at < kMost) found_keys[at] = key_of(v, first + u * kThreads * P + e);
                    }
                }
        }
        __syncthreads();
        if (tid == 0) {
            float t = 0.0f;
            for (int w = 0; w < kThreads / 32; ++w) t += parts[w];
            a.stat[uint64_t(seq) * lists + list] = make_float2(m, t);
        }
        const uint32_t found = n_found;
        if (found <= kMost) {
            for (uint32_t i = tid; i < found; i += kThreads) {
                const unsigned long long k = found_keys[i];
                uint32_t r = 0;
                for (uint32_t j = 0; j < found; ++j) r += found_keys[j] > k;
                if (r < a.keep) keys[uint64_t(r) * lists] = k;
            }
            for (uint32_t r = found + tid; r < a.keep; r += kThreads) keys[uint64_t(r) * lists] = 0;
        } else {
            unsigned long long last = ~0ull;
            for (uint32_t r = 0; r < a.keep; ++r) {
                unsigned long long best = 0;
#pragma unroll
                for (int u = 0; u < kVecs; ++u)
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const float v = E::at(x[u], e);
                        if (v > -INFINITY) {
                            const unsigned long long k = key_of(v, first + u * kThreads * P + e);
                            if (k < last && k > best) best = k;
                        }
                    }
                for (int k = 1; k < 32; k <<= 1) { const unsigned long long o = __shfl_xor_sync(0xffffffffu, best, k); best = o > best ? o : best; }
                __syncthreads();
                if (lane == 0) found_keys[warp] = best;
                __syncthreads();
                for (int w = 0; w < kThreads / 32; ++w) best = found_keys[w] > best ? found_keys[w] : best;
                last = best;                                   // (more than kMost >= keep elements are above -infinity: there always is one)
                if (tid == 0) keys[uint64_t(r) * lists] = best;
            }
        }
    } else {
        if (tid == 0) a.stat[uint64_t(seq) * lists + list] = make_float2(-INFINITY, 0.0f);
        for (uint32_t r = tid; r < a.keep; r += kThreads) keys[uint64_t(r) * lists] = 0;
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) last_flag = atomicAdd(&a.ticket[seq], 1u) == lists - 1;
    __syncthreads();
    if (last_flag) {
        __threadfence();
        join(a, seq, shared);
        if (tid == 0) a.ticket[seq] = 0;
    }
}

// 16-byte pieces of a thread: 8 (32 KB of a row per block) where that leaves a block for every SM, else 2.
constexpr int kWide = 8, kNarrow = 2;
uint32_t slices_for(uint32_t vocab, int dtype, int vecs)
{
    const uint64_t per = dtype == WWWS_F32 ? 4 : 8, pieces = (vocab + per - 1) / per;
    return uint32_t((pieces + uint64_t(vecs) * kThreads - 1) / (uint64_t(vecs) * kThreads));
}
int vecs_for(uint32_t rows, uint32_t vocab, int dtype) { return uint64_t(rows) * slices_for(vocab, dtype, kWide) >= 148 ? kWide : kNarrow; }

}  // namespace

uint64_t beams_scratch(uint32_t rows, uint32_t vocab, int dtype, uint32_t keep)
{
    const uint64_t lists = uint64_t(rows) * slices_for(vocab, dtype, vecs_for(rows, vocab, dtype));
    return lists * 8 * (keep + 1ull);
}

cudaError_t launch_beams(BeamArgs a, uint32_t rows, int dtype, void* scratch, cudaStream_t s)
{
    const int vecs = vecs_for(rows, a.vocab, dtype);
    a.slices = slices_for(a.vocab, dtype, vecs);
    a.stat = static_cast<float2*>(scratch);
    a.keys = reinterpret_cast<unsigned long long*>(a.stat + uint64_t(rows) * a.slices);
    const dim3 grid(a.slices, rows);
    auto go = [&](auto dt) {
        if (vecs == kWide) k_beams<decltype(dt)::value, kWide><<<grid, kThreads, 0, s>>>(a);
        else k_beams<decltype(dt)::value, kNarrow><<<grid, kThreads, 0, s>>>(a);
        return cudaGetLastError();
    };
    using std::integral_constant;
    return dtype == WWWS_F32 ? go(integral_constant<int, WWWS_F32>()) : dtype == WWWS_BF16 ? go(integral_constant<int, WWWS_BF16>()) : go(integral_constant<int, WWWS_F16>());
}

}  // namespace wwws
