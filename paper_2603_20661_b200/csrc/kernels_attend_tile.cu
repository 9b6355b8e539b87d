// Attention of many rows per kv head over the paged cache (chunks of prompts, whole prompts): tcgen05 tiles fed by TMA.
//
// A block works on 256 rows of one (sequence, kv head) at a time, as two tiles of 128: a row is a (new token, query head) pair,
// the query heads of a kv head side by side, so every key tile serves all of them.  Per tile of 128 keys
//     S = Q K^T            128 x 128 x head_dim into tensor memory, fp32
//     P = 2^(x - m)        x = scale * log2(e) * S, running maximum and sum per row, a row per thread (per two threads for a quantised cache)
//     O = O + P V          P back into tensor memory over S, rounded to the activation type; O stays in tensor memory, fp32
// One warp issues all matrix instructions in the order PV0 S0 PV1 S1: while the tensor cores work on one row tile, the softmax warps of the
// other turn its S into P.  m is allowed to lag behind the true maximum by a factor 2^kLag, so that O is rescaled (a pass over
// tensor memory) in the first few tiles only; the result is the same sum, since numerator and denominator share m.
//   - Floor per key tile at head_dim 128: 4 x 128^3 multiply-adds, 2,048 clocks of the tensor cores, and 2 x 16,384 exponentials at 16 a clock,
//     as many.  Measured: two prompts of 8,192 tokens (32 heads, 8 kv heads, 1.10e12 operations) in 1.10 to 1.14 ms, 965 to 1,000 TFLOP/s, 60 % of
//     the library's rate for a large product; back to back for seconds 1.14 ms at a median of 1,680 MHz under the power cap, about 4,000 clocks
//     a tile with its share of loads and stores.  What is left is the chain of a row tile: scores, softmax, P back, PV, the next scores; the two row
//     tiles hide half of it from one another, and tensor memory (2 x 128 columns of S, 2 x head_dim of O) has no room for a third.  Tried and slower: 64-key tiles with two S each (1.26 ms: the cost per tile is mostly fixed),
//     polynomials for a quarter of the exponentials (1.22 against 1.10 ms: their constants cost more moves than the unit saves).
//   - The issuing warp stays converged and predicates each instruction on one lane: in a branch for one lane the descriptors went through
//     vector registers, 90 clocks per instruction instead of 30.
//   - Work is cut by key tiles, as in kernels_attend.cu: all (unit, tile) pairs laid end to end, an equal share for each of 148
//     blocks, cut units joined by the last of their blocks.  The position of a share is found from closed sums, so
//     causal triangles, windows and ragged lengths need no plan.
//   - K and V tiles come by TMA page by page into the 128-byte-swizzled layout that the matrix instructions read; pages that no row
//     sees are fetched from beyond the tensor's end, which fills zeros.  16-bit values are looked through by a warp of its own (see there).
//   - Quantised caches: codes land in a staging ring, two more warps widen them into the operand layout (exactly: 16-bit floats
//     hold the codes); scales multiply the scores (keys) and the weights (values) in fp32.
#include <cuda.h>

#include <type_traits>

#include "backend.cuh"
#include "tcgen.cuh"

namespace wwws {
namespace {

constexpr int kBM = 128, kBN = 128;
constexpr float kLow = -3.0e38f;

template <bool BF, int CACHE, int D> struct Cfg {
    static constexpr bool kQuant = CACHE != WWWS_CACHE_16;
    static constexpr int kSlabs = D / 64;
    static constexpr int kQ = kBM * D * 2;                  // one row tile of queries
    static constexpr int kTile = kBN * D * 2;               // one operand tile of keys or values
    static constexpr int kCodes = kBN * D;                  // the same as codes
    static constexpr int kStages = kQuant ? (D == 128 ? 3 : 6) : (D == 128 ? 4 : 8);
    static constexpr int kStaging = kQuant ? (D == 128 ? 3 : 6) : 0;
    static constexpr int kScales = kQuant ? 4 * 2 * kBN * 4 : 0;            // four tiles' key and value scales
    static constexpr int kOffRing = 2 * kQ;
    static constexpr int kOffStaging = kOffRing + kStages * kTile;
    static constexpr int kOffScales = kOffStaging + kStaging * kCodes;
    static constexpr int kOffExchange = kOffScales + kScales;               // quantised: two floats per row, row tile and half: maximum, sum
    static constexpr int kOffBars = kOffExchange + (kQuant ? 2 * 4 * kBM * 4 : 0);
    static constexpr int kSmem = kOffBars + 512 + 1024;                     // the rings start at a 1,024-byte boundary
    // Threads per row: one where the scores are used as they come; two for a quantised cache, whose scales have to be fetched for every column
    // (a thread per row, 24 int8 prompts: 0.79 ms, two 0.62; two prompts of 8,192 tokens in 16 bits: 1.03 ms with one, 1.10 with two).
    static constexpr int kHalves = kQuant ? 2 : 1;
    static constexpr int kSoftmaxWarps = 8 * kHalves, kConvert = kQuant ? 64 : 32;    // kConvert: threads that widen codes, or look through 16-bit values
    static constexpr int kWarpConvert = kSoftmaxWarps, kWarpMma = kWarpConvert + kConvert / 32, kWarpLoad = kWarpMma + 1;
    static constexpr int kThreads = (kWarpLoad + 1) * 32;
    static constexpr uint32_t kColP = kQuant ? 0 : 64;      // where P lies over S: the columns whose scores are in registers by then
    // Weights in f16 over a quantised cache are kept relative to the power of two below the largest value scale of the segment so far, or small
    // values would push them into f16's subnormals, and times kLift: 2^kLag * 2 * kLift = 2^15 < 65,504, and what is lost below 2^-24 is 2^-36
    // of the row's largest weight.  bf16 has the range for the scales as they are.
    static constexpr bool kRelative = !BF && kQuant;
    static constexpr float kLag = kRelative ? 3.0f : 8.0f;
    static constexpr float kLift = kRelative ? 2048.0f : 1.0f;
    // f16 weights over 16-bit values carry 2^kRaise from the exponential on, and so do their sums: again 2^15 at most, faint ones exact to 2^-32.
    static constexpr float kRaise = !BF && !kQuant ? 7.0f : 0.0f;
    static constexpr uint32_t kColS = 0, kColO = 256, kCols = 512;
};

// ---- the linear space of (unit, kv head, key tile) ----
// A unit counts kUnitCost tiles more than it has: what loading its queries and storing its result costs, in tiles.
constexpr int kUnitCost = 2;

// sum_{i<n} floor((a i + b) / kBN) = (sum_{i<n} (a i + b) - sum_{i<n} (a i + b) mod kBN) / kBN, a > 0, b >= 0.  kBN is a power of two, so with g = gcd(a, kBN) the
// remainders repeat after p = kBN / g of them, and p neighbouring ones are b mod g, b mod g + g, b mod g + 2 g, ... in some order: whole periods have a
// closed sum, and fewer than p (a is even: 64 at most) are left to add.
__device__ __forceinline__ long long floors(long long n, int a, long long b)
{
    if (n <= 0) return 0;
    const int g = min(a & -a, kBN), p = kBN / g;
    long long rest = n / p * (p * (int(b) & (g - 1)) + p * (p - 1) / 2 * g);
    int x = int(b) & (kBN - 1);
    for (int i = int(n) & (p - 1); i; --i) { rest += x; x = (x + a) & (kBN - 1); }
    return (n * (n - 1) / 2 * a + n * b - rest) / kBN;
}

struct Seq {
    int q0, q_len, kv, place0, units;      // units: blocks of `step` tokens
};
struct Space {
    int step;                              // tokens of a unit: two row tiles
    int window, sink_tiles;
    __device__ __forceinline__ void span(const Seq& s, int u, int& hi, int& lo, int& lo_tile, int& n_sink, int& tiles) const
    {
        hi = min(s.kv, s.place0 + min(s.q_len, (u + 1) * step));
        lo = window ? max(0, s.place0 + u * step - window + 1) : 0;
        if (hi <= 0) { hi = 0; lo = lo_tile = n_sink = 0; tiles = 1; return; }     // nothing seen: one empty tile, the rows get zeros
        lo_tile = lo / kBN;
        n_sink = min(sink_tiles, lo_tile);
        tiles = n_sink + (hi + kBN - 1) / kBN - lo_tile;
    }
    // cost of the first n units, in tiles
    __device__ long long sum(const Seq& s, int n) const
    {
        if (n <= 0) return 0;
        long long total = (long long)n * kUnitCost;
        int last = n;
        if (n == s.units) { int hi, lo, lt, ns, t; span(s, n - 1, hi, lo, lt, ns, t); total += t; last = n - 1; }
        if (last == 0) return total;
        // units [0, last) are whole: their keys end at place0 + (u + 1) step
        int first = 0;
        if (s.place0 + step <= 0) first = min(last, (-s.place0) / step);           // units that see nothing: one tile each
        total += first;
        total += floors(last - first, step, (long long)s.place0 + (long long)(first + 1) * step + kBN - 1);
        if (window) {                                                              // less floor((place0 + u step - window + 1) / 128) - sink tiles, where positive
            const long long b = (long long)s.place0 - window + 1 - (long long)sink_tiles * kBN;
            long long u0 = b >= 0 ? 0 : (-b + step - 1) / step;
            if (u0 < last) total -= floors(last - u0, step, b + u0 * step);
        }
        return total;
    }
};

// Walks a block's share, segment by segment: a segment is a run of key tiles of one (sequence, unit, kv head).  Every role holds one.
// Positions are relative to the share's begin.
struct Walk {
    int y, end, base;          // base: position of the first tile of (seq, u) and kv head 0
    uint32_t seq; int u;
    int q0, q_len, kv;
    // the segment
    int h, t0, t1, tiles;      // key tiles [t0, t1) of the unit's `tiles`
    int from;                  // position of tile t0
    int hi, lo, lo_tile, n_sink;
    bool more;

    __device__ __forceinline__ bool load(const AttendArgs& a)
    {
        return sequence(a.b, seq, q0, q_len, kv, a.err) && q_len;
    }
    __device__ __forceinline__ Seq as_seq(const Space& sp) const { return Seq{ q0, q_len, kv, kv - q_len, (q_len + sp.step - 1) / sp.step }; }
    __device__ __forceinline__ void span(const Space& sp) { sp.span(as_seq(sp), u, hi, lo, lo_tile, n_sink, tiles); }
    __device__ __forceinline__ bool next(const AttendArgs& a, const Space& sp)
    {
        if (y >= end) return false;
        while (true) {
            while (y >= base + (tiles + kUnitCost) * int(a.p.n_kv_heads)) {
                base += (tiles + kUnitCost) * int(a.p.n_kv_heads);
                if (++u * sp.step >= q_len) {
                    u = 0;
                    do { ++seq; } while (seq < a.b.n_seqs && !load(a));
                    if (seq >= a.b.n_seqs) { y = end; return false; }
                }
                span(sp);
            }
            h = (y - base) / (tiles + kUnitCost); t0 = (y - base) % (tiles + kUnitCost);
            from = y;
            y += tiles + kUnitCost - t0;
            if (t0 < tiles) break;
            if (y >= end) return false;         // the share began behind the unit's last tile
        }
        t1 = min(tiles, t0 + end - from);
        return true;
    }
    __device__ __forceinline__ int tok0(const Space& sp) const { return u * sp.step; }             // first token of the unit
    __device__ __forceinline__ bool two(const Space& sp) const { return u * sp.step + sp.step / 2 < q_len; }   // the second row tile has tokens
    __device__ __forceinline__ int tile_key(int t) const { return (t < n_sink ? t : lo_tile + t - n_sink) * kBN; }
    // whether the key tile has keys that some rows of the unit do not see
    __device__ __forceinline__ bool mixed(const AttendArgs& a, const Space& sp, int key0) const
    {
        const int first = kv - q_len + u * sp.step, last = kv - q_len + min(q_len, (u + 1) * sp.step) - 1;
        return key0 + kBN - 1 > first || (a.window && key0 < last - int(a.window) + 1 && key0 + kBN > int(a.sinks));
    }
};

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// The largest of three (NaN only if all are).
__device__ __forceinline__ float max3(float a, float b, float c) { float d; asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }

__device__ __forceinline__ void scale2(uint32_t* x, uint64_t by)
{
    float y0, y1;
    unpack2(mul2(pack2(__uint_as_float(x[0]), __uint_as_float(x[1])), by), y0, y1);
    x[0] = __float_as_uint(y0); x[1] = __float_as_uint(y1);
}

// The values of keys [key0, end) that are infinite or not numbers, added to the sums (tensor memory, at tO) of this warp's rows that see them; `place`: of this
// thread's row.  The product had zeros in their place.  (Not inlined, and its loops not unrolled: it hardly ever runs.)
template <bool BF, int D>
__device__ __noinline__ void add_unreal(const int32_t* table, const uint8_t* v, uint32_t n_pages, uint32_t page_shift, uint32_t n_kv_heads, uint32_t h, int key0, int end,
                                        int lo, int window, int sinks, int place, uint32_t tO)
{
#pragma unroll 1
    for (int key = key0; key < end; ++key) {
        if (window && key < lo && key >= sinks) continue;
        const uint32_t page = uint32_t(__ldg(table + (key >> page_shift)));
        if (page >= n_pages) continue;
        const uint4* row = reinterpret_cast<const uint4*>(v + (((uint64_t(page) * n_kv_heads + h) << page_shift) + (key & ((1 << page_shift) - 1))) * (D * 2));
        const bool sees = key <= place && (!window || key > place - window || key < sinks);
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
            const uint4 x0 = __ldg(row + 2 * c), x1 = __ldg(row + 2 * c + 1);
            uint32_t top = 0;
            largest_halves(top, x0); largest_halves(top, x1);
            if (!unreal2<BF>(top)) continue;                  // (the same for the whole warp)
            const uint32_t x[8] = { x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w };
            uint32_t o[16];
            tm_ld16(tO + 16 * c, o);
            tm_wait_ld16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t half = x[e / 2] >> (e % 2 * 16) & 0xffffu;
                if (sees && unreal<BF>(half)) o[e] = __float_as_uint(__uint_as_float(o[e]) + Act<BF>::lo(half));
            }
            tm_st16(tO + 16 * c, o);
            tm_wait_st();
        }
    }
}

template <bool BF, int CACHE, int D>
__global__ void __launch_bounds__(Cfg<BF, CACHE, D>::kThreads, 1)
k_attend_tile(AttendArgs a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using C = Cfg<BF, CACHE, D>;
    using A = Act<BF>;
    constexpr bool kQuant = C::kQuant;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024 - (smem_at(raw) & 1023)) & 1023);
    const uint32_t base = smem_at(smem);
    // barriers: full and empty per stage, the same for staging, queries full and free, S ready / P ready (its first half, all of it) / PV done per row tile, join, pairs of warps, all instructions done, widening warps, values looked through
    const uint32_t bars = base + C::kOffBars;
    auto kv_full = [&](int s) { return bars + 8 * s; };
    auto kv_empty = [&](int s) { return bars + 8 * (C::kStages + s); };
    auto st_full = [&](int s) { return bars + 8 * (2 * C::kStages + s); };
    auto st_empty = [&](int s) { return bars + 8 * (2 * C::kStages + C::kStaging + s); };
    constexpr int kRest = 2 * (C::kStages + C::kStaging);
    const uint32_t q_full = bars + 8 * kRest, q_empty = q_full + 8;
    auto s_full = [&](int w) { return q_full + 16 + 8 * w; };
    auto p_full = [&](int w) { return q_full + 32 + 8 * w; };
    auto o_done = [&](int w) { return q_full + 48 + 8 * w; };
    auto p_half = [&](int w) { return q_full + 64 + 8 * w; };
    const uint32_t join = q_full + 80;
    auto pair_bar = [&](int k) { return q_full + 88 + 8 * k; };
    const uint32_t drained = q_full + 152, widened = q_full + 160;
    auto v_ready = [&](int s) { return q_full + 168 + 8 * (s / 2); };                // 16-bit values, which lie in the odd stages: looked through
    static_assert(8 * (kRest + 21 + C::kStages / 2) <= 400 && (kQuant || C::kStages % 2 == 0), "barriers fit");
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + C::kOffBars + 400);        // [0] tensor memory, [1] dead, [2] last to arrive, [3] bit 0: a page outside the pool was met, bit 1: a value that is no number was taken out, [4..] the share's start
    volatile uint32_t* dead = words + 1;
    int* start = reinterpret_cast<int*>(words + 4);                                 // [0] base, [1] sequence, [2] unit
    float* unit_of = reinterpret_cast<float*>(words + 8);                           // [4 tiles] what their value scales are relative to
    uint32_t* largest = words + 12;                                                 // [2 tiles][2 widening warps]

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
    const uint32_t Hkv = a.p.n_kv_heads, G = a.group;
    const int tq = kBM / int(G);                                                    // tokens of a row tile
    const Space sp{ 2 * tq, int(a.window), int((a.sinks + kBN - 1) / kBN) };

    // ---- the block's share ----
    long long* prefix = reinterpret_cast<long long*>(smem);                         // [n_seqs + 1], over the rings before they are used
    __shared__ long long warp_sum[32];
    long long carry = 0;
    for (uint32_t b0 = 0; b0 < a.b.n_seqs; b0 += C::kThreads) {
        long long v = 0;
        Walk w; w.seq = b0 + tid;
        if (w.seq < a.b.n_seqs && w.load(a)) { const Seq q = w.as_seq(sp); v = sp.sum(q, q.units); }
        long long inc = v;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, inc, m); if (lane >= m) inc += y; }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        long long before = carry;
        for (int k = 0; k < C::kThreads / 32; ++k) { if (k < warp) before += warp_sum[k]; carry += warp_sum[k]; }
        if (w.seq < a.b.n_seqs) prefix[w.seq] = before + inc - v;
        __syncthreads();
    }
    const long long total = carry * Hkv;
    const long long share = max((total + gridDim.x - 1) / gridDim.x, 2ll);
    const long long begin = blockIdx.x * share, end = min(total, begin + share);
    if (begin >= end) return;
    if (tid == 0) {
        const long long per_head = begin / Hkv;
        uint32_t i = 0, hi = a.b.n_seqs;
        while (hi - i > 1) { const uint32_t mid = (i + hi) >> 1; if (prefix[mid] <= per_head) i = mid; else hi = mid; }
        Walk w; w.seq = i; w.load(a);
        const Seq q = w.as_seq(sp);
        int u = 0, uh = q.units;
        while (uh - u > 1) { const int mid = (u + uh) >> 1; if (prefix[i] + sp.sum(q, mid) <= per_head) u = mid; else uh = mid; }
        start[0] = int((prefix[i] + sp.sum(q, u)) * Hkv - begin); start[1] = int(i); start[2] = u;
        words[1] = words[3] = 0;
        for (int s = 0; s < C::kStages; ++s) { bar_init(kv_full(s), kQuant ? C::kConvert : 1); bar_init(kv_empty(s), 1); }
        for (int s = 0; s < C::kStaging; ++s) { bar_init(st_full(s), 1); bar_init(st_empty(s), C::kConvert); }
        bar_init(q_full, 1); bar_init(q_empty, 1);
        for (int w2 = 0; w2 < 2; ++w2) { bar_init(s_full(w2), 1); bar_init(p_full(w2), 128 * C::kHalves); bar_init(p_half(w2), 128); bar_init(o_done(w2), 1); }
        bar_init(join, 256 * C::kHalves);
        for (int k = 0; k < 8; ++k) bar_init(pair_bar(k), 64);
        bar_init(drained, 1);
        bar_init(widened, C::kConvert);
        for (int s = 1; s < C::kStages; s += 2) bar_init(v_ready(s), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();                                                                // the share is known, prefix is done with
    if (warp == 0) tmem_alloc(smem_at(words), C::kCols);
    // query rows that no copy fills (128 is no multiple of the group) are zero
    for (int e = tid; e < 2 * C::kQ / 16; e += C::kThreads) reinterpret_cast<uint4*>(smem)[e] = make_uint4(0, 0, 0, 0);
    fence_async_proxy();
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, words[0], 0);

    // each warp's walk lives in shared memory: its first lane steps it, and it takes no registers from the loops below
    __shared__ Walk walks[C::kThreads / 32];
    Walk& g = walks[warp];
    if (lane == 0) {
        Walk w;
        w.y = 0; w.end = int(end - begin); w.base = start[0]; w.seq = uint32_t(start[1]); w.u = start[2];
        w.load(a); w.span(sp);
        g = w;
    }
    auto next = [&] {
        __syncwarp();
        if (lane == 0) { Walk w = g; w.more = w.next(a, sp); g = w; }
        __syncwarp();
        return g.more;
    };
#define WAIT(bar, parity) __all_sync(0xffffffffu, bar_wait(bar, parity, dead))

    if (warp == C::kWarpLoad) {
        // ---- copies: queries of a segment, then its key and value tiles in turn ----
        const uint32_t page_tokens = 1u << a.p.page_shift;
        constexpr int kBoxSlabs = kQuant ? 1 : C::kSlabs;
        const int n_box = kBN / int(page_tokens) * kBoxSlabs;
        const int nowhere = int(a.p.n_pages * Hkv) << a.p.page_shift;               // beyond the last row: zeros
        uint32_t it = 0, seg = 0;
        bool ok = true;
        while (ok && next()) {
            for (int t = g.t0; ok && t < g.t1; ++t) {
                // a lane per box: the page's row in the pool, or nowhere
                int row = nowhere;
                const int b = lane / kBoxSlabs, key0 = g.tile_key(t), key = key0 + b * int(page_tokens);
                if (lane < n_box && key < g.hi && (!a.window || key + int(page_tokens) > g.lo || key < int(a.sinks))) {
                    const uint32_t page = uint32_t(__ldg(a.b.page_table + uint64_t(g.seq) * a.b.table_stride + (uint32_t(key) >> a.p.page_shift)));
                    if (page < a.p.n_pages) row = int((page * Hkv + uint32_t(g.h)) << a.p.page_shift);
                    else { report(a.err, bePage); atomicOr(words + 3, 1u); }     // (seen by the softmax warps by way of the barriers below)
                }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    constexpr int N = kQuant ? C::kStaging : C::kStages;
                    const int s = int(it % N);
                    const uint32_t full = kQuant ? st_full(s) : kv_full(s), empty = kQuant ? st_empty(s) : kv_empty(s);
                    if (it >= N && !(ok = WAIT(empty, uint32_t(it / N - 1) & 1))) break;
                    if (lane == 0) bar_expect(full, kQuant ? C::kCodes : C::kTile);
                    __syncwarp();
                    if (lane < n_box) {
                        const CUtensorMap* map = kv ? &v_map : &k_map;
                        if constexpr (kQuant) tma_2d(base + C::kOffStaging + s * C::kCodes + b * int(page_tokens) * D, map, 0, row, full);
                        else tma_2d(base + C::kOffRing + s * C::kTile + lane % kBoxSlabs * (kBN * 128) + b * int(page_tokens) * 128, map, lane % kBoxSlabs * 64, row, full);
                    }
                    ++it;
                    if (t == g.t0 && kv == 0) {         // the segment's queries go behind its first keys: they wait for the last segment's scores
                        if (seg && !(ok = WAIT(q_empty, uint32_t(seg - 1) & 1))) break;
                        if (lane == 0) {
                            const uint32_t one = uint32_t(tq) * G * 128 * C::kSlabs;            // bytes of one row tile
                            bar_expect(q_full, g.two(sp) ? 2 * one : one);
                            for (int w = 0; w < (g.two(sp) ? 2 : 1); ++w)
                                for (int d = 0; d < C::kSlabs; ++d) tma_3d(base + w * C::kQ + d * (kBM * 128), &q_map, d * 64, g.h * int(G), g.q0 + g.tok0(sp) + w * tq, q_full);
                        }
                        ++seg;
                    }
                }
            }
        }
        // leave no copy in flight behind: where all went well they have landed long ago; otherwise the waits end after 1e8 cycles
        constexpr int N = kQuant ? C::kStaging : C::kStages;
        const long long t0 = clock64();
        auto landed = [&](uint32_t bar, uint32_t parity) { while (!bar_try(bar, parity) && clock64() - t0 < 100000000ll) {} };
        for (uint32_t k = it > N ? it - N : 0; k < it; ++k) landed(kQuant ? st_full(int(k % N)) : kv_full(int(k % N)), uint32_t(k / N) & 1);
        if (seg) landed(q_full, uint32_t(seg - 1) & 1);
    } else if (warp == C::kWarpMma) {
        // ---- matrix instructions: S of the first tile, then per tile PV and the next S, the two row tiles in turn ----
        constexpr uint32_t kDescS = mma_desc(BF, false, kBN), kDescO = mma_desc(BF, true, D);
        uint32_t it = 0, seg = 0;                              // ring items and tiles so far (the parity of p_full goes by tiles of each row tile)
        uint32_t tiles_of[2] = { 0, 0 };
        bool ok = true;
        const uint32_t one = elect_one();
        auto commit = [&](uint32_t bar) { tc_commit_one(one, bar); };
        auto scores = [&](int w, int s) {
            const uint64_t qa = smem_desc(base + w * C::kQ, 16, 1024), kb = smem_desc(base + C::kOffRing + s * C::kTile, 16, 1024);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)                    // (descriptors count 16 bytes)
                mma_ss(one, tmem + C::kColS + w * 128, qa + (k / 4 * (kBM * 128) + k % 4 * 32) / 16, kb + (k / 4 * (kBN * 128) + k % 4 * 32) / 16, kDescS, k > 0);
            commit(s_full(w));
        };
        // the eight steps of 16 keys, [from, to) in the order in which P is written
        auto values = [&](int w, int s, bool add, auto from, auto to) {
            constexpr int order[8] = { 2, 3, 4, 5, 6, 7, 0, 1 };
            const uint64_t vb = smem_desc(base + C::kOffRing + s * C::kTile, kBN * 128, 1024);
#pragma unroll
            for (int i = decltype(from)::value; i < decltype(to)::value; ++i)
                mma_ts(one, tmem + C::kColO + w * D, tmem + C::kColS + w * 128 + C::kColP + order[i] * 8, vb + order[i] * 2048 / 16, kDescO, add || i > 0);
        };
        using std::integral_constant;
        while (ok && next()) {
            const int nw = __shfl_sync(0xffffffffu, g.two(sp) ? 2 : 1, 0), n = __shfl_sync(0xffffffffu, g.t1 - g.t0, 0);
            if (!(ok = WAIT(q_full, uint32_t(seg) & 1))) break;
            if (!(ok = WAIT(kv_full(int(it % C::kStages)), uint32_t(it / C::kStages) & 1))) break;
            tc_after();
            for (int w = 0; w < nw; ++w) scores(w, int(it % C::kStages));
            commit(kv_empty(int(it % C::kStages)));
            for (int j = 0; ok && j < n; ++j) {
                const uint32_t iv = it + 1, ik = it + 2;
                if (!(ok = WAIT(kQuant ? kv_full(int(iv % C::kStages)) : v_ready(int(iv % C::kStages)), uint32_t(iv / C::kStages) & 1))) break;
                for (int w = 0; ok && w < nw; ++w) {
                    if constexpr (!kQuant) {                    // the first half of P is worked on while the second is made
                        if (!(ok = WAIT(p_half(w), uint32_t(tiles_of[w]) & 1))) break;
                        tc_after();
                        values(w, int(iv % C::kStages), j > 0, integral_constant<int, 0>(), integral_constant<int, 4>());
                    }
                    if (!(ok = WAIT(p_full(w), uint32_t(tiles_of[w]) & 1))) break;
                    tc_after();
                    ++tiles_of[w];
                    values(w, int(iv % C::kStages), j > 0, integral_constant<int, kQuant ? 0 : 4>(), integral_constant<int, 8>());
                    commit(o_done(w));
                    if (j + 1 < n) {
                        if (w == 0 && !(ok = WAIT(kv_full(int(ik % C::kStages)), uint32_t(ik / C::kStages) & 1))) break;
                        scores(w, int(ik % C::kStages));
                    }
                    if (j + 2 >= n && w == nw - 1 && (j + 2 == n || n == 1)) commit(q_empty);      // the segment's last scores are issued
                }
                if (!ok) break;
                // both tiles' instructions up to here must be done before the stages are filled again
                commit(kv_empty(int(iv % C::kStages)));
                if (j + 1 < n) commit(kv_empty(int(ik % C::kStages)));
                it += 2;
            }
            ++seg;
        }
        // nor any matrix instruction, or its arrival at a barrier
        commit(drained);
        const long long t0 = clock64();
        while (!bar_try(drained, 0) && clock64() - t0 < 100000000ll) {}
    } else if (warp >= C::kWarpConvert && warp < C::kWarpMma) {
        // ---- widening: codes of a staged tile to the operand layout, scales beside them ----
        if constexpr (kQuant) {
            const int t = tid - C::kWarpConvert * 32;
            constexpr int kChunks = D / 16;                     // 16 codes each
            uint32_t it = 0, unit = 0;                          // unit: a power of two, as bits
            bool ok = true;
            while (ok && next()) {
                for (int tile = g.t0; ok && tile < g.t1; ++tile) {
                    const int key0 = g.tile_key(tile);
                    auto seen = [&](int key) { return key < g.hi && (!a.window || key >= g.lo || key < int(a.sinks)); };
                    // this thread's keys' scales
                    float scale[2][kBN / C::kConvert];
#pragma unroll
                    for (int e = 0; e < kBN / C::kConvert; ++e) {
                        scale[0][e] = scale[1][e] = 0.0f;
                        const int key = key0 + t + e * C::kConvert;
                        if (seen(key)) {
                            const uint32_t page = uint32_t(__ldg(a.b.page_table + uint64_t(g.seq) * a.b.table_stride + (uint32_t(key) >> a.p.page_shift)));
                            if (page < a.p.n_pages) {
                                const uint64_t cell = ((uint64_t(page) * Hkv + uint32_t(g.h)) << a.p.page_shift) + (key & ((1 << a.p.page_shift) - 1));
                                scale[0][e] = __ldg(a.p.k_scale + cell); scale[1][e] = __ldg(a.p.v_scale + cell);
                            }
                        }
                    }
                    float lift = C::kLift;
                    if constexpr (C::kRelative) {
                        uint32_t top = 0;
#pragma unroll
                        for (int e = 0; e < kBN / C::kConvert; ++e) { const uint32_t b = __float_as_uint(scale[1][e]) & 0x7fffffffu; if (b < 0x7f800000u) top = max(top, b); }
                        top = __reduce_max_sync(0xffffffffu, top);
                        const uint32_t n = it / 2 % 2;
                        if (lane == 0) largest[2 * n + warp - C::kWarpConvert] = top;
                        bar_arrive(widened);
                        if (!(ok = WAIT(widened, n))) break;
                        if (tile == g.t0) unit = 27u << 23;              // 2^-100: smaller values are zeros in f16 anyway, and its inverse can be lifted
                        unit = min(max(unit, max(largest[2 * n], largest[2 * n + 1]) & 0x7f800000u), 253u << 23);
                        lift *= __uint_as_float((254u << 23) - unit);
                    }
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        const int ss = int(it % C::kStaging), s = int(it % C::kStages);
                        if (!(ok = WAIT(st_full(ss), uint32_t(it / C::kStaging) & 1))) break;
                        if (it >= C::kStages && !(ok = WAIT(kv_empty(s), uint32_t(it / C::kStages - 1) & 1))) break;
                        const uint8_t* from = smem + C::kOffStaging + ss * C::kCodes;
                        uint8_t* to = smem + C::kOffRing + s * C::kTile;
#pragma unroll 4
                        for (int e = 0; e < kChunks * (kBN / C::kConvert); ++e) {
                            const int c = t % kChunks, r = t / kChunks + e * (C::kConvert / kChunks);
                            uint4 x = *reinterpret_cast<const uint4*>(from + r * D + c * 16);
                            if (!seen(key0 + r)) x = make_uint4(0, 0, 0, 0);
                            const uint4 lo = make_uint4(widen<BF, CACHE>(x.x & 0xffffu), widen<BF, CACHE>(x.x >> 16), widen<BF, CACHE>(x.y & 0xffffu), widen<BF, CACHE>(x.y >> 16));
                            const uint4 hi = make_uint4(widen<BF, CACHE>(x.z & 0xffffu), widen<BF, CACHE>(x.z >> 16), widen<BF, CACHE>(x.w & 0xffffu), widen<BF, CACHE>(x.w >> 16));
                            uint8_t* row = to + c / 4 * (kBN * 128) + r * 128;
                            const int p0 = ((2 * (c % 4)) ^ (r & 7)) * 16, p1 = ((2 * (c % 4) + 1) ^ (r & 7)) * 16;
                            if (c < 4) { *reinterpret_cast<uint4*>(row + p0) = lo; *reinterpret_cast<uint4*>(row + p1) = hi; }
                            else { *reinterpret_cast<uint4*>(row + p1) = hi; *reinterpret_cast<uint4*>(row + p0) = lo; }   // the other order: no bank twice
                        }
                        float* sc = reinterpret_cast<float*>(smem + C::kOffScales) + ((it / 2) % 4 * 2 + kv) * kBN;
#pragma unroll
                        for (int e = 0; e < kBN / C::kConvert; ++e) sc[t + e * C::kConvert] = kv ? scale[1][e] * lift : scale[0][e] * a.scale_log2;
                        if (C::kRelative && kv == 0 && t == 0) unit_of[it / 2 % 4] = __uint_as_float(unit);
                        fence_async_proxy();
                        bar_arrive(kv_full(s));
                        bar_arrive(st_empty(ss));
                        ++it;
                    }
                }
            }
        } else {
            // ---- 16-bit values: those that no row of the unit sees become zeros (a weight of 0 does not silence a NaN), and so do, where some rows see
            // them and others do not, those that are no numbers: the softmax warps add them to the rows that see them when the segment's sums are done.
            // (A warp of its own: in the softmax warps the same cost 512 tokens behind 5,489 2 % and two prompts of 8,192 tokens 3 to 7 %; here they lose
            // nothing.  A second such warp costs the former 4 %.)
            const int t = tid - C::kWarpConvert * 32;
            uint32_t it = 1;                                    // ring item of the values
            bool ok = true;
            while (ok && next()) {
                for (int tile = g.t0; tile < g.t1; ++tile, it += 2) {
                    const int key0 = g.tile_key(tile), s = int(it % C::kStages);
                    if (!(ok = WAIT(kv_full(s), uint32_t(it / C::kStages) & 1))) break;
                    if (g.mixed(a, sp, key0)) {
#pragma unroll 1
                        for (int r = t; r < kBN; r += C::kConvert) {
                            const int key = key0 + r;
                            const bool seen = key < g.hi && (!a.window || key >= g.lo || key < int(a.sinks));
                            uint8_t* row = smem + C::kOffRing + s * C::kTile + r * 128;
                            auto piece = [&](int e) { return reinterpret_cast<uint4*>(row + e / 8 * (kBN * 128) + ((e ^ r) & 7) * 16); };     // (neighbours meet no bank twice)
                            uint32_t top = 0;
                            if (seen) {
#pragma unroll
                                for (int e = 0; e < 8 * C::kSlabs; ++e) largest_halves(top, *piece(e));
                            }
                            if (!seen || unreal2<BF>(top)) {
#pragma unroll 1
                                for (int e = 0; e < 8 * C::kSlabs; ++e) {
                                    const uint4 x = *piece(e);
                                    *piece(e) = seen ? make_uint4(real2<BF>(x.x), real2<BF>(x.y), real2<BF>(x.z), real2<BF>(x.w)) : make_uint4(0, 0, 0, 0);
                                }
                                if (seen) atomicOr(words + 3, 2u);
                            }
                        }
                        fence_async_proxy();
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(v_ready(s));
                }
            }
        }
    } else if (warp < C::kSoftmaxWarps) {
        // ---- softmax of one row tile: kHalves threads per row, kCols columns each ----
        constexpr int kCols = kBN / C::kHalves;
        const int w = warp / (4 * C::kHalves), half = warp / 4 % C::kHalves, r = tid % 128;
        const uint32_t lanes = uint32_t(warp % 4 * 32) << 16;
        const uint32_t tS = tmem + C::kColS + w * 128 + half * kCols + lanes, tP = tmem + C::kColS + w * 128 + C::kColP + half * kCols / 2 + lanes;
        const uint32_t tO = tmem + C::kColO + w * D + half * (D / C::kHalves) + lanes;
        const uint32_t pair = pair_bar(w * 4 + warp % 4);                     // the two warps that share 32 rows
        float* mine = reinterpret_cast<float*>(smem + C::kOffExchange) + (w * 2 + half) * kBM + r;
        const float* theirs = reinterpret_cast<float*>(smem + C::kOffExchange) + (w * 2 + (half ^ 1)) * kBM + r;
        uint32_t it = 0, n_done = 0, joins = 0, pairs = 0;   // tiles of the block (ring items / 2), tiles of this row tile, joins, exchanges
        bool ok = true;
        while (ok && next()) {
            const int n = g.t1 - g.t0;
            const bool work = w == 0 || g.two(sp);
            const int tok = g.tok0(sp) + w * tq + r / int(G);
            const bool row_on = r < tq * int(G) && tok < g.q_len;
            const int place = (g.kv - g.q_len) + tok;
            // places of the row tile's first and last row
            const int place_a = (g.kv - g.q_len) + g.tok0(sp) + w * tq, place_b = (g.kv - g.q_len) + min(g.q_len - 1, g.tok0(sp) + w * tq + tq - 1);
            float m = kLow, l = 0.0f, unit = 1.0f;                           // unit: what O is relative to
            if (work) {
                for (int j = 0; j < n; ++j) {
                    const int key0 = g.tile_key(g.t0 + j), first = key0 + half * kCols;
                    const uint32_t iv = 2 * (it + j) + 1;                    // ring item of the tile's values
                    if (!(ok = WAIT(s_full(w), n_done & 1))) break;
                    tc_after();
                    uint32_t bad = 0;                                        // 16 keys each of this thread that lie in a page outside the pool: hidden
                    if (*static_cast<volatile uint32_t*>(words + 3)) {
#pragma unroll 1
                        for (int e = 0; e < kCols / 16; ++e) {
                            const int key = first + 16 * e;
                            if (key < g.hi && uint32_t(__ldg(a.b.page_table + uint64_t(g.seq) * a.b.table_stride + (uint32_t(key) >> a.p.page_shift))) >= a.p.n_pages) bad |= 1u << e;
                        }
                    }
                    const bool masked = bad || key0 + kBN - 1 > place_a || (a.window && key0 < place_b - int(a.window) + 1 && key0 + kBN > int(a.sinks));
                    const float* ks = reinterpret_cast<const float*>(smem + C::kOffScales) + ((it + j) % 4 * 2) * kBN + half * kCols;
                    if constexpr (kQuant) { if (!(ok = WAIT(kv_full(int(iv % C::kStages)), (iv / C::kStages) & 1))) break; }     // both scales are there
                    // the columns [c0, c0 + 32) of this thread that the row sees, a bit each
                    auto visible = [&](int c0) {
                        const int end = min(max(place - first - c0 + 1, 0), 32);                       // columns before `end` are not ahead of the row
                        uint32_t bits = end == 32 ? ~0u : (1u << end) - 1;
                        if (a.window) {
                            const int from = min(max(place - first - c0 + 1 - int(a.window), 0), 32);  // columns before `from` have left the window, unless they are sinks
                            const int sunk = min(max(int(a.sinks) - first - c0, 0), 32);
                            bits &= (from == 32 ? 0u : ~0u << from) | (sunk == 32 ? ~0u : (1u << sunk) - 1);
                        }
                        const uint32_t out = bad >> (c0 / 16);
                        return bits & ~((out & 1u) * 0xffffu | (out >> 1 & 1u) * 0xffff0000u);
                    };
                    const float f = kQuant ? 1.0f : a.scale_log2;
                    const uint32_t kHidden = f < 0.0f ? 0x7f800000u : 0xff800000u;                    // x f = -infinity
                    // 32 columns: times the key scales (which hold the softmax scale) where the cache has them, hidden ones put away
                    auto prepare = [&](uint32_t* v, int c0) {
                        if constexpr (kQuant) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                const ulonglong2 k4 = *reinterpret_cast<const ulonglong2*>(ks + c0 + e);
                                scale2(v + e, k4.x); scale2(v + e + 2, k4.y);
                            }
                        }
                        if (masked) {                            // (the same for the whole warp)
                            const uint32_t bits = visible(c0);
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = bits & (1u << e) ? v[e] : kHidden;
                        }
                    };
                    uint32_t x0[32], x[kCols - 32];
                    tm_ld32(tS, x0);
#pragma unroll
                    for (int c0 = 32; c0 < kCols; c0 += 32) tm_ld32(tS + c0, x + c0 - 32);
                    tm_wait_ld32(x0);
#pragma unroll
                    for (int c0 = 32; c0 < kCols; c0 += 32) tie32(x + c0 - 32);
                    prepare(x0, 0);
#pragma unroll
                    for (int c0 = 32; c0 < kCols; c0 += 32) prepare(x + c0 - 32, c0);
                    auto X = [&](int e) { return __uint_as_float(e < 32 ? x0[e] : x[e - 32]); };
                    float top, t0 = X(0), t1 = X(1), t2 = X(2), t3 = X(3);
                    if (f >= 0.0f) {
#pragma unroll
                        for (int e = 0; e < kCols; e += 8) { t0 = max3(t0, X(e), X(e + 1)); t1 = max3(t1, X(e + 2), X(e + 3)); t2 = max3(t2, X(e + 4), X(e + 5)); t3 = max3(t3, X(e + 6), X(e + 7)); }
                        top = fmaxf(max3(t0, t1, t2), t3) * f;
                    } else {
#pragma unroll
                        for (int e = 4; e < kCols; e += 4) { t0 = fminf(t0, X(e)); t1 = fminf(t1, X(e + 1)); t2 = fminf(t2, X(e + 2)); t3 = fminf(t3, X(e + 3)); }
                        top = fminf(fminf(t0, t1), fminf(t2, t3)) * f;
                    }
                    if constexpr (C::kHalves == 2) {
                        *mine = top;
                        bar_arrive(pair);
                        if (!(ok = WAIT(pair, pairs & 1))) break;
                        ++pairs;
                        top = fmaxf(top, *theirs);
                    }
                    if (!row_on) top = m;
                    const float unit_now = C::kRelative ? unit_of[(it + j) % 4] : 1.0f;
                    if (__any_sync(0xffffffffu, top > m + C::kLag) || unit_now != unit) {
                        const float mn = fmaxf(m, top), less = ex2(m - mn), shrink = C::kRelative ? less * __fdiv_rn(unit, unit_now) : less;
                        if (j > 0) {                            // O so far shrinks too, once the last product into it is done; each thread takes its share of the columns
                            if (!(ok = WAIT(o_done(w), (n_done - 1) & 1))) break;
                            tc_after();
#pragma unroll 1
                            for (int c0 = 0; c0 < D / C::kHalves; c0 += 16) {
                                uint32_t v[16];
                                tm_ld16(tO + c0, v);
                                tm_wait_ld16(v);
#pragma unroll
                                for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * shrink);
                                tm_st16(tO + c0, v);
                            }
                        }
                        l *= less; m = mn; unit = unit_now;
                    }
                    const uint64_t f2 = pack2(f, f), m2 = pack2(C::kRaise - m, C::kRaise - m);
                    uint64_t sum_a = pack2(0.0f, 0.0f), sum_b = sum_a;
                    auto weights = [&](const uint32_t* v, int c0) {
                        uint32_t p[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float y0, y1;
                            unpack2(fma2(pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), f2, m2), y0, y1);
                            y0 = ex2(y0); y1 = ex2(y1);
                            const uint64_t y = pack2(y0, y1);
                            if (e % 4) sum_b = add2(sum_b, y); else sum_a = add2(sum_a, y);
                            if constexpr (kQuant) {
                                const ulonglong2 v4 = *reinterpret_cast<const ulonglong2*>(ks + kBN + c0 + e / 4 * 4);
                                unpack2(mul2(y, e % 4 ? v4.y : v4.x), y0, y1);
                                if (masked) { y0 = v[e] == kHidden ? 0.0f : y0; y1 = v[e + 1] == kHidden ? 0.0f : y1; }      // a hidden value's scale may be NaN
                            }
                            p[e / 2] = A::pack(y0, y1);
                        }
                        tm_st16(tP + c0 / 2, p);
                    };
                    if constexpr (C::kHalves == 1) {
                        // the first 32 columns were dropped after the maximum and are read again (tensor memory is cheaper than 32 more registers)
                        weights(x, 32);
                        tm_ld32(tS, x0);
                        weights(x + 32, 64);
                        tm_wait_st();
                        tc_before();
                        bar_arrive(p_half(w));
                        weights(x + 64, 96);
                        tm_wait_ld32(x0);
                        prepare(x0, 0);
                        weights(x0, 0);
                    } else {
                        weights(x0, 0);
                        weights(x, 32);
                    }
                    float s0, s1;
                    unpack2(add2(sum_a, sum_b), s0, s1);
                    l += s0 + s1;
                    tm_wait_st();
                    tc_before();
                    bar_arrive(p_full(w));
                    ++n_done;
                }
            }
            if (!ok) break;
            it += n;
            if (work) {
                if constexpr (C::kHalves == 2) {
                    mine[4 * kBM] = l;                          // the row's sum is that of both halves
                    bar_arrive(pair);
                    if (!(ok = WAIT(pair, pairs & 1))) break;
                    ++pairs;
                    l = half ? theirs[4 * kBM] + l : l + theirs[4 * kBM];
                }
                if (!(ok = WAIT(o_done(w), uint32_t(n_done - 1) & 1))) break;
                tc_after();
                if constexpr (!kQuant) {
                    if (*static_cast<volatile uint32_t*>(words + 3) & 2) {
#pragma unroll 1
                        for (int j = 0; j < n; ++j)
                            if (const int key0 = g.tile_key(g.t0 + j); g.mixed(a, sp, key0))
                                add_unreal<BF, D>(a.b.page_table + uint64_t(g.seq) * a.b.table_stride, a.p.v, a.p.n_pages, a.p.page_shift, Hkv, uint32_t(g.h), key0, min(key0 + kBN, g.hi),
                                                  g.lo, int(a.window), int(a.sinks), row_on ? place : -1, tO);
                    }
                }
            }
            const bool whole = g.t0 == 0 && g.t1 == g.tiles;
            const long long x0 = begin + g.from;
            const uint32_t slot = 2 * blockIdx.x + (x0 == begin ? 0 : 1);
            uint8_t* dst = a.out + (uint64_t(g.q0 + (row_on ? tok : 0)) * a.out_stride + (uint64_t(g.h) * G + r % G) * D + half * (D / C::kHalves)) * 2;
            if (work) {
                const float inv = l > 0.0f ? (1.0f / C::kLift) / l * unit : l;
#pragma unroll
                for (int c0 = 0; c0 < D / C::kHalves; c0 += 32) {
                    uint32_t v[32];
                    tm_ld32(tO + c0, v);
                    tm_wait_ld32(v);
                    if (whole) {
                        if (row_on) {
#pragma unroll
                            for (int e = 0; e < 32; e += 8) {
                                uint32_t o[4];
#pragma unroll
                                for (int q = 0; q < 4; ++q) o[q] = A::pack(__uint_as_float(v[e + 2 * q]) * inv, __uint_as_float(v[e + 2 * q + 1]) * inv);
                                *reinterpret_cast<uint4*>(dst + (c0 + e) * 2) = make_uint4(o[0], o[1], o[2], o[3]);
                            }
                        }
                    } else if (row_on) {
                        float4* part = reinterpret_cast<float4*>(a.s.part_o) + ((uint64_t(slot) * 2 + w) * (D / 4) + half * (D / 4 / C::kHalves)) * kBM + r;      // [slot][row tile][D / 4][128] float4
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            part[(c0 / 4 + e) * kBM] = make_float4(__uint_as_float(v[4 * e]) * unit, __uint_as_float(v[4 * e + 1]) * unit, __uint_as_float(v[4 * e + 2]) * unit, __uint_as_float(v[4 * e + 3]) * unit);
                    }
                }
                if (!whole && row_on && half == 0) a.s.part_ml[(slot * 2 + w) * kBM + r] = make_float2(m, l);
                tc_before();
            }
            if (!whole) {
                // the unit's blocks are consecutive; the last to arrive joins their parts in that order
                const long long u0 = x0 - g.t0, u1 = u0 + g.tiles;
                const uint32_t blk0 = uint32_t(u0 / share), blk1 = uint32_t((u1 - 1) / share);
                const uint32_t first_slot = 2 * blk0 + (u0 % share ? 1 : 0);
                __threadfence();
                bar_arrive(join);
                if (!(ok = WAIT(join, uint32_t(joins) & 1))) break;
                ++joins;
                if (tid == 0) { __threadfence(); words[2] = atomicAdd(&a.s.ticket[first_slot], 1u) == blk1 - blk0; }
                __syncwarp();
                bar_arrive(join);
                if (!(ok = WAIT(join, uint32_t(joins) & 1))) break;
                ++joins;
                if (words[2]) {
                    __threadfence();
                    if (row_on && work) {
                        // what the parts' weights add up to, then 32 columns at a time, whose loads do not depend on one another
                        auto slot_of = [&](uint32_t b) { return (b == blk0 ? first_slot : 2 * b) * 2 + w; };
                        float mm = kLow, ll = 0.0f;
                        for (uint32_t b = blk0; b <= blk1; ++b) {
                            const float2 ml = __ldcg(a.s.part_ml + slot_of(b) * kBM + r);
                            const float mn = fmaxf(mm, ml.x);
                            ll = ll * ex2(mm - mn) + ml.y * ex2(ml.x - mn); mm = mn;
                        }
                        const float inv = ll > 0.0f ? (1.0f / C::kLift) / ll : ll;
#pragma unroll 1
                        for (int c = 0; c < D / 4 / C::kHalves; c += 8) {
                            float4 acc[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) acc[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
                            for (uint32_t b = blk0; b <= blk1; ++b) {
                                const uint32_t s = slot_of(b);
                                const float f = ex2(__ldcg(a.s.part_ml + s * kBM + r).x - mm);
                                const float4* part = reinterpret_cast<const float4*>(a.s.part_o) + (uint64_t(s) * (D / 4) + half * (D / 4 / C::kHalves) + c) * kBM + r;
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const float4 v = __ldcg(part + e * kBM);
                                    acc[e].x += v.x * f; acc[e].y += v.y * f; acc[e].z += v.z * f; acc[e].w += v.w * f;
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 8; e += 2)
                                *reinterpret_cast<uint4*>(dst + (c + e) * 8) = make_uint4(A::pack(acc[e].x * inv, acc[e].y * inv), A::pack(acc[e].z * inv, acc[e].w * inv),
                                                                                          A::pack(acc[e + 1].x * inv, acc[e + 1].y * inv), A::pack(acc[e + 1].z * inv, acc[e + 1].w * inv));
                        }
                    }
                    if (tid == 0) a.s.ticket[first_slot] = 0;
                }
            }
        }
    }
#undef WAIT
    __syncwarp();
    tc_before();
    __syncthreads();
    if (tid == 0 && words[1]) report(a.err, beTimeout);
    if (warp == 0) { tc_after(); tmem_free(tmem, C::kCols); }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder()
{
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) == cudaSuccess && r == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(p) : nullptr;
    }();
    return f;
}

}  // namespace

cudaError_t launch_attend_tile(const AttendArgs& a, uint32_t head_dim, int dtype, int cache, cudaStream_t s)
{
    const EncodeTiled encode = encoder();
    if (!encode) return cudaErrorNotSupported;
    const bool quant = cache != WWWS_CACHE_16;
    const CUtensorMapDataType act = dtype == WWWS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap maps[3];
    {
        const cuuint64_t dims[3] = { head_dim, uint64_t(a.p.n_kv_heads) * a.group, a.b.n_tokens };
        const cuuint64_t strides[2] = { head_dim * 2ull, a.q_stride * 2ull };
        const cuuint32_t box[3] = { 64, a.group, 128 / a.group }, ones[3] = { 1, 1, 1 };
        if (encode(&maps[0], act, 3, const_cast<uint8_t*>(a.q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) return cudaErrorInvalidValue;
    }
    for (int kv = 0; kv < 2; ++kv) {
        const cuuint64_t dims[2] = { head_dim, uint64_t(a.p.n_pages) * a.p.n_kv_heads << a.p.page_shift };
        const cuuint64_t strides[1] = { head_dim * (quant ? 1ull : 2ull) };
        const cuuint32_t box[2] = { quant ? head_dim : 64, 1u << a.p.page_shift }, ones[2] = { 1, 1 };
        if (encode(&maps[1 + kv], quant ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : act, 2, kv ? a.p.v : a.p.k, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   quant ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    auto go = [&](auto bf, auto kind, auto dim) -> cudaError_t {
        using C = Cfg<decltype(bf)::value, decltype(kind)::value, decltype(dim)::value>;
        static_assert(C::kSmem <= 232448 - 512, "shared memory of a block");
        static_assert(C::kOffBars >= 2048 * 8, "the prefix fits over the rings");
        constexpr auto kernel = k_attend_tile<decltype(bf)::value, decltype(kind)::value, decltype(dim)::value>;
        if (cudaError_t e = allow_smem<kernel>(C::kSmem); e != cudaSuccess) return e;
        // no more blocks than tiles the bounds allow
        const uint64_t step = 2 * (128 / a.group), units = a.b.n_tokens / step + a.b.n_seqs;
        const uint64_t tiles = units * a.p.n_kv_heads * ((a.b.max_kv_len + kBN - 1) / kBN);
        kernel<<<uint32_t(tiles < kTileBlocks ? (tiles ? tiles : 1) : kTileBlocks), C::kThreads, C::kSmem, s>>>(a, maps[0], maps[1], maps[2]);
        return cudaGetLastError();
    };
    using std::integral_constant;
    auto dim = [&](auto bf, auto kind) { return head_dim == 64 ? go(bf, kind, integral_constant<int, 64>()) : go(bf, kind, integral_constant<int, 128>()); };
    auto kind = [&](auto bf) {
        return cache == WWWS_CACHE_16 ? dim(bf, integral_constant<int, 0>()) : cache == WWWS_CACHE_INT8 ? dim(bf, integral_constant<int, 1>()) : dim(bf, integral_constant<int, 2>());
    };
    return dtype == WWWS_BF16 ? kind(std::true_type()) : kind(std::false_type());
}

}  // namespace wwws
