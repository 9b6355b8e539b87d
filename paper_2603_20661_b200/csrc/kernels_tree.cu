// Attention of a tree of drafted tokens with many rows per kv head over the paged cache: tcgen05 tiles fed by TMA.
//
// A row is a (drafted token, query head) pair; the query heads of a kv head lie side by side.  Per tile of 128 keys and 128 rows
//     S = Q K^T            into tensor memory, fp32
//     P = 2^(x - m)        x = scale * log2(e) * S, running maximum m and sum per row, a row per thread; P back into tensor memory, 16 bits
//     O = O + P V          O stays in tensor memory, fp32
// Bound by HBM: a tile of keys and values of head_dim 128 in 16 bits is 64 KB, 2,850 clocks of an SM's share of HBM, against 1,024 clocks of the tensor cores and as
// many of the exponential unit per 128 rows.  So what counts is that loads never wait for anything:
//   - Eight softmax warps, two S.  A unit of more than 128 rows (16-bit caches) is two row tiles, each with an S, an O and four of the warps: while the
//     tensor cores work for one, the other's softmax runs.  One of fewer rows has a single O and its key tiles take the two S in turn: the next scores are worked out while
//     all eight warps, 64 columns a thread, turn the last ones into weights.
//   - One warp issues the matrix instructions in the order PV(n), S(n + 2), n counting the S; one issues the copies of pages, into rings of their own for keys and values.
//   - Work is cut by key tiles: all (unit, tile) pairs laid end to end, an equal share for each of 148 blocks, found from a running sum over the
//     sequences; cut units are joined by the last of their blocks, in block order.  Every role works out its segments by itself.
//   - m is allowed to lag behind the true maximum by a factor (2^8, 2^4 over quantised caches), so that O is rescaled in the first few tiles only.
//   - Quantised caches: codes land in a staging ring, four warps widen them into the operands' layout, to f16 whatever the backend (exactly, and for e4m3 by the
//     hardware: widening to bf16 took three times the instructions); scales multiply the scores (keys) and the weights (values) in fp32.
//     bf16 queries become f16 by a power of two per row (exact down to 2^-28 of the row's largest); weights are kept relative to twice the largest value scale of
//     the segment when that last grew beyond it.
//   - Measured: 12 x 61 tokens behind 16,001 of 16 bits, 32 on 8 heads of 128: 208 us, 3,850 GB/s, bound by the chain scores - weights - product of a row tile (from some hundred calls
//     on end 229 to 247 us: the power cap, 1,460 MHz); 24 x 21 behind 3,001 on average in e4m3: 98 us, bound by widening, scales and exponentials (behind 16,000: 305 us, 2,700 GB/s).
//   - Pages that no row sees are read from page 0 and their values put to zero before they are used, as is everything else of a tile that no row sees.
#include <cuda.h>

#include <type_traits>

#include "backend.cuh"
#include "tcgen.cuh"

namespace wwws {
namespace {

constexpr int kBM = 128, kBN = 128;
constexpr float kLow = -3.0e38f;

template <bool BF, int CACHE, int D, bool kTwo> struct Cfg {
    static constexpr bool kQuant = CACHE != WWWS_CACHE_16;
    static constexpr int kSlabs = D / 64;
    static_assert(!(kQuant && kTwo), "a quantised cache's rings leave no room for two row tiles");
    static constexpr int kQTiles = kTwo ? 2 : 1;            // row tiles of a unit
    static constexpr int kTile = kBN * D * 2, kCodes = kBN * D;
    static constexpr int kQ = kBM * D * 2;
    static constexpr int kK = kQuant ? 2 : D == 128 ? 3 : 4, kV = kQuant || D == 128 ? 2 : 4, kStaging = kQuant ? (D == 128 ? 3 : 6) : 0;
    static constexpr int kOffK = kQTiles * kQ, kOffV = kOffK + kK * kTile, kOffStaging = kOffV + kV * kTile;
    // [keys, values][4 tiles][128]: the keys' of three more tiles may come while a tile's scores are weighted (the third's wait for that tile's product)
    static constexpr int kOffScales = kOffStaging + kStaging * kCodes;
    static constexpr int kOffMl = kOffScales + (kQuant ? 2 * 4 * kBN * 4 : 0);           // [2 halves][128] sums
    static constexpr int kOffTops = kOffMl + (kTwo ? 0 : 2 * kBM * 4);                  // [2 tiles][2 halves][128] maxima
    static constexpr int kOffRel = kOffTops + (kTwo ? 0 : 2 * 2 * kBM * 4);             // [8 warps][64] value scales relative to the largest
    static constexpr int kOffBars = kOffRel + (kQuant ? 8 * 64 * 4 : 0);                // the sequences' running sum lies behind
    static constexpr int kOffPrefix = kOffBars + 384;
    static constexpr int kFixed = kOffPrefix + 1024;                        // the rings start at a 1,024-byte boundary
    static constexpr int kConvert = kQuant ? 4 : 1;                         // warps that widen codes, or look through 16-bit values
    static constexpr int kWarpConvert = 8, kWarpMma = kWarpConvert + kConvert, kWarpLoad = kWarpMma + 1, kThreads = (kWarpLoad + 1) * 32;
    static constexpr bool kB = BF && !kQuant;                               // the operands' type
    // How far (log2) m may lag behind, and the factor that weights in f16 and their sums carry: 2^15 at most together.  Over a quantised cache bf16 backends are
    // held to bf16's range, so the factor is the larger part there: what is lost is 2^-35 of the row's largest weight times the largest value of any key so far, whether the row sees it or
    // not (a factor of 2^8 failed columns of faint weights alone; a lag of 2^1 would lose 2^-38 and took 24 x 21 over e4m3 from 100 to 103 us).
    static constexpr float kLag = kQuant ? 4.0f : 8.0f, kRaise = kQuant ? 11.0f : kB ? 0.0f : 7.0f;
    static constexpr uint32_t kColS = 0, kColO = 256, kColP = 64, kCols = 512;
    // P's step e of 16 keys: over the upper half of S or, where two threads have a row, each over the first half of its own columns.
    static __device__ constexpr uint32_t col_p(int e) { return kTwo ? kColP + e * 8 : e / 4 * 64 + e % 4 * 8; }
};

// The largest of three (NaN only if all are).
__device__ __forceinline__ float max3(float a, float b, float c) { float d; asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// 2^y of two numbers on the units that add and multiply (the one for 2^y takes eight clocks a warp): y = n + f, |f| <= 1/2, 2^f by the polynomial of degree 5 whose
// largest relative error is least, 2^-23.7, and 2^-22.8 with the coefficients in fp32.  For y < 127; what is below 2^-126.5 is 0 (an exponent field of 0).  A NaN stays one.
__device__ __forceinline__ uint64_t ex2_both(uint64_t y)
{
    float y0, y1;
    unpack2(y, y0, y1);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(y0) : "f"(-127.0f)); asm("max.NaN.f32 %0, %0, %1;" : "+f"(y1) : "f"(-127.0f));
    y = pack2(y0, y1);
    constexpr float kRound = 12582912.0f + 127.0f;             // 1.5 2^23, and the exponent's bias: the sum's low bits are 2^n's exponent
    const uint64_t j = add2(y, pack2(kRound, kRound)), f = fma2(add2(j, pack2(-kRound, -kRound)), pack2(-1.0f, -1.0f), y);
    auto both = [](float c) { return pack2(c, c); };
    uint64_t r = both(0.0013248048f);
    r = fma2(r, f, both(0.009675051f)); r = fma2(r, f, both(0.055507995f)); r = fma2(r, f, both(0.24022135f)); r = fma2(r, f, both(0.69314694f)); r = fma2(r, f, both(1.0000001f));
    float j0, j1;
    unpack2(j, j0, j1);
    return mul2(r, pack2(__uint_as_float(__float_as_uint(j0) << 23), __uint_as_float(__float_as_uint(j1) << 23)));
}

// Four codes to f16, exactly: e4m3 by the hardware; int8 with its sign turned is the low byte of 1,024 + 128 + code.
template <int CACHE> __device__ __forceinline__ void widen4(uint32_t four, uint32_t& lo, uint32_t& hi)
{
    if constexpr (CACHE == WWWS_CACHE_INT8) {
        four ^= 0x80808080u;
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(four, 0x64646464u, 0x4140)), "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(four, 0x64646464u, 0x4342)), "r"(0x64806480u));
    } else { lo = widen<false, CACHE>(four & 0xffffu); hi = widen<false, CACHE>(four >> 16); }
}

// A unit counts kUnitCost tiles more than it has: what bringing its queries and storing its result costs, in tiles.
constexpr uint32_t kUnitCost = 3;

// What a call's sequences and a block's share of them come to.
struct Plan {
    const uint32_t* prefix;              // [n_seqs + 1] tiles of all earlier sequences, per kv head
    uint32_t share, begin, end;
    int tq, step;                        // tokens of a row tile, of a unit
};
struct Seg {
    int q0, q_len, kv, place0, h, tok0;
    int t0, t1, tiles;                   // key tiles [t0, t1) of the unit's
    int lo, n_sink, lo_tile;             // first key that the window leaves to any row; tiles with sinks; first tile behind them
    uint32_t seq, x0;                    // sequence; position of tile t0
    __device__ __forceinline__ int key_of(int t) const { return (t < n_sink ? t : lo_tile + t - n_sink) * kBN; }
    // whether a tile has keys that some row of the unit may not see
    __device__ __forceinline__ bool mixed(const AttendArgs& a, int key0) const
    {
        return key0 + kBN > place0 || (a.window && key0 < place0 + q_len - int(a.window) && key0 + kBN > int(a.sinks));
    }
    // whether any row of the unit may see a key
    __device__ __forceinline__ bool seen(const AttendArgs& a, int key) const { return key < kv && (!a.window || key >= lo || key < int(a.sinks)); }
};

__device__ __forceinline__ void span(const AttendArgs& a, int q_len, int kv, int& lo, int& lo_tile, int& n_sink, int& tiles)
{
    lo = a.window ? max(0, kv - q_len - int(a.window) + 1) : 0;
    const int all = (max(kv, 0) + kBN - 1) / kBN;
    lo_tile = min(lo / kBN, all);
    n_sink = a.window ? min((min(int(a.sinks), kv) + kBN - 1) / kBN, lo_tile) : 0;
    tiles = max(1, n_sink + all - lo_tile);                  // one (empty) tile even where nothing is seen: the rows get zeros
}

// The segment that begins at position x or, where a unit's last tile lies before it, the next one; x becomes the position behind it.  False: the share has no more.
__device__ __forceinline__ bool segment(const AttendArgs& a, const Plan& p, uint32_t& x, Seg& s)
{
    const uint32_t hkv = a.p.n_kv_heads;
    while (x < p.end) {
        const uint32_t per_head = x / hkv;
        uint32_t i = 0, hi = a.b.n_seqs;
        while (hi - i > 1) { const uint32_t mid = (i + hi) >> 1; if (p.prefix[mid] <= per_head) i = mid; else hi = mid; }
        s.seq = i;
        s.q0 = __ldg(a.b.q_start + i); s.q_len = __ldg(a.b.q_start + i + 1) - s.q0; s.kv = __ldg(a.b.kv_len + i); s.place0 = s.kv - s.q_len;
        span(a, s.q_len, s.kv, s.lo, s.lo_tile, s.n_sink, s.tiles);
        const uint32_t each = uint32_t(s.tiles) + kUnitCost, rel = x - p.prefix[i] * hkv, unit = rel / each, t0 = rel - unit * each;
        if (t0 >= uint32_t(s.tiles)) { x += each - t0; continue; }
        s.x0 = x; s.t0 = int(t0);
        s.t1 = int(min(uint32_t(s.tiles), t0 + (p.end - x)));
        s.h = int(unit % hkv); s.tok0 = int(unit / hkv) * p.step;
        x += uint32_t(s.t1) - t0;
        return true;
    }
    return false;
}

// The power of two that brings the largest of a row of bf16 into [2^14, 2^15); returns its inverse.  (A row of zeros, subnormals or with a NaN or an infinity stays.)
template <int N> __device__ __forceinline__ float lifted(const uint4 (&q)[N], float& mul)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) largest_halves(top, q[e]);
    const uint32_t ex = max(top & 0xffffu, top >> 16) >> 7;
    const uint32_t me = ex == 0 || ex == 255 ? 127 : min(max(127 + 127 + 14 - int(ex), 1), 253);
    mul = __uint_as_float(me << 23);
    return __uint_as_float((254 - me) << 23);
}

template <bool BF, int CACHE, int D, bool kTwo>
__global__ void __launch_bounds__(Cfg<BF, CACHE, D, kTwo>::kThreads, 1)
k_tree(AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using C = Cfg<BF, CACHE, D, kTwo>;
    using A = Act<BF>;
    using W = Act<C::kB>;
    constexpr bool kQuant = C::kQuant;
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t warp_sum[C::kThreads / 32], words[4];        // words: [0] tensor memory, [1] dead, [2] last to arrive, [3] bit 0: a bad page was met, bit 1: a value that is no number was taken out
    uint8_t* smem = raw + ((1024 - (smem_at(raw) & 1023)) & 1023);
    const uint32_t base = smem_at(smem), bars = base + C::kOffBars;
    volatile uint32_t* dead = words + 1;
    auto k_full = [&](uint32_t s) { return bars + 8 * s; };
    auto k_empty = [&](uint32_t s) { return bars + 8 * (C::kK + s); };
    auto v_full = [&](uint32_t s) { return bars + 8 * (2 * C::kK + s); };
    auto v_empty = [&](uint32_t s) { return bars + 8 * (2 * C::kK + C::kV + s); };
    constexpr int kRest = 2 * (C::kK + C::kV);
    auto st_full = [&](uint32_t s) { return bars + 8 * (kRest + s); };
    auto st_empty = [&](uint32_t s) { return bars + 8 * (kRest + C::kStaging + s); };
    auto v_ready = [&](uint32_t s) { return bars + 8 * (kRest + s); };              // 16-bit values, looked through
    constexpr int kMore = kRest + (kQuant ? 2 * C::kStaging : C::kV);
    const uint32_t q_full = bars + 8 * kMore, done = q_full + 8, drained = q_full + 16;
    auto s_full = [&](int w) { return q_full + 24 + 8 * w; };
    auto p_full = [&](int w) { return q_full + 40 + 8 * w; };
    const uint32_t meeting = q_full + 56, o_done = q_full + 64;
    auto p_both = [&](uint32_t b) { return q_full + 72 + 8 * b; };
    auto pair = [&](int q) { return q_full + 88 + 8 * q; };          // the two warps that share 32 rows
    auto p_half = [&](int w) { return q_full + 120 + 8 * w; };       // the weights of columns 64 to 127 are there
    static_assert(8 * (kMore + 17) <= 384, "barriers fit");
    uint32_t* prefix = reinterpret_cast<uint32_t*>(smem + C::kOffPrefix);

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
    const uint32_t hkv = a.p.n_kv_heads, G = a.group;
    Plan plan;
    plan.prefix = prefix; plan.tq = kBM / int(G); plan.step = C::kQTiles * plan.tq;

    // ---- the block's share ----
    uint32_t carry = 0;
    for (uint32_t b0 = 0; b0 < a.b.n_seqs; b0 += C::kThreads) {
        uint32_t v = 0;
        if (b0 + tid < a.b.n_seqs) {
            int q0, q_len, kv, lo, lt, ns, tiles;
            if (sequence(a.b, b0 + tid, q0, q_len, kv, a.err) && q_len) { span(a, q_len, kv, lo, lt, ns, tiles); v = uint32_t((q_len + plan.step - 1) / plan.step) * (uint32_t(tiles) + kUnitCost); }
        }
        uint32_t inc = v;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, inc, m); if (lane >= m) inc += y; }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        uint32_t before = carry;
        for (int k = 0; k < C::kThreads / 32; ++k) { if (k < warp) before += warp_sum[k]; carry += warp_sum[k]; }
        if (b0 + tid < a.b.n_seqs) prefix[b0 + tid] = before + inc - v;
        __syncthreads();
    }
    const uint32_t total = carry * hkv;
    plan.share = max((total + gridDim.x - 1) / gridDim.x, 2u);
    plan.begin = min(blockIdx.x * plan.share, total); plan.end = min(total, plan.begin + plan.share);
    if (tid == 0) {
        words[1] = words[3] = 0;
        for (int s = 0; s < C::kK; ++s) { bar_init(k_full(s), kQuant ? C::kConvert * 32 : 1); bar_init(k_empty(s), 1); }
        for (int s = 0; s < C::kV; ++s) { bar_init(v_full(s), kQuant ? C::kConvert * 32 : 1); bar_init(v_empty(s), 1); if (!kQuant) bar_init(v_ready(s), 1); }
        for (int s = 0; s < C::kStaging; ++s) { bar_init(st_full(s), 1); bar_init(st_empty(s), C::kConvert * 32); }
        bar_init(q_full, 256); bar_init(done, 1); bar_init(drained, 1); bar_init(meeting, 256); bar_init(o_done, 1);
        for (int w = 0; w < 2; ++w) { bar_init(s_full(w), 1); bar_init(p_full(w), 128); bar_init(p_both(w), 256); bar_init(p_half(w), 128); }
        for (int q = 0; q < 4; ++q) bar_init(pair(q), 64);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 0) tmem_alloc(smem_at(words), C::kCols);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, words[0], 0);
#define WAIT(bar, parity) __all_sync(0xffffffffu, bar_wait(bar, parity, dead))

    if (warp == C::kWarpLoad) {
        // ---- copies: a key and a value tile in turn, a lane per box of a page ----
        const uint32_t page_tokens = 1u << a.p.page_shift;
        constexpr int kBoxSlabs = kQuant ? 1 : C::kSlabs;
        const int n_box = kBN / int(page_tokens) * kBoxSlabs;
        uint32_t it = 0, staged = 0, k_sent = 0, v_sent = 0;        // tiles before the segment; copies so far
        bool ok = true;
        uint32_t x = plan.begin;
        for (Seg g; ok && segment(a, plan, x, g);) {
            // the unit's queries and masks will be read by others in some tiles' time
            for (int r = lane; r < C::kQTiles * kBM; r += 32)
                if (const int tok = g.tok0 + r / int(G); r < plan.step * int(G) && tok < g.q_len) {
                    const uint8_t* q = a.q + (uint64_t(g.q0 + tok) * a.q_stride + (uint64_t(g.h) * G + r % int(G)) * D) * 2;
                    for (int e = 0; e < D * 2; e += 128) asm volatile("prefetch.global.L1 [%0];" :: "l"(q + e));
                    if (r % int(G) == 0) asm volatile("prefetch.global.L1 [%0];" :: "l"(a.tree + uint64_t(uint32_t(g.q0 + tok)) * a.tree_words));
                }
            // keys of a tile, then the values of the one before: the next scores do not wait for a place among the values
            int row = 0;
            for (int t = g.t0; ok && t <= g.t1; ++t) {
                const int b = lane / kBoxSlabs, values_row = row;
                if (t < g.t1) {
                    const int key = g.key_of(t) + b * int(page_tokens);
                    row = int(uint32_t(g.h) << a.p.page_shift);     // page 0
                    if (lane < n_box && key < g.kv && (!a.window || key + int(page_tokens) > g.lo || key < int(a.sinks))) {
                        const uint32_t page = uint32_t(__ldg(a.b.page_table + uint64_t(g.seq) * a.b.table_stride + (uint32_t(key) >> a.p.page_shift)));
                        if (page < a.p.n_pages) row = int((page * hkv + uint32_t(g.h)) << a.p.page_shift);
                        else { report(a.err, bePage); atomicOr(words + 3, 1u); }        // (the others see it by way of the barriers below)
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (kv ? t == g.t0 : t == g.t1) continue;
                    const uint32_t tile = it + uint32_t(t - g.t0) - kv;
                    uint32_t full, dst;
                    if constexpr (kQuant) {
                        const uint32_t s = staged % C::kStaging;
                        if (staged >= C::kStaging && !(ok = WAIT(st_empty(s), (staged / C::kStaging - 1) & 1))) break;
                        ++staged;
                        full = st_full(s); dst = base + C::kOffStaging + s * C::kCodes + b * int(page_tokens) * D;
                    } else {
                        const uint32_t s = tile % (kv ? C::kV : C::kK), turn = tile / (kv ? C::kV : C::kK);
                        if (turn && !(ok = WAIT(kv ? v_empty(s) : k_empty(s), (turn - 1) & 1))) break;
                        ++(kv ? v_sent : k_sent);
                        full = kv ? v_full(s) : k_full(s);
                        dst = base + (kv ? C::kOffV : C::kOffK) + s * C::kTile + lane % kBoxSlabs * (kBN * 128) + b * int(page_tokens) * 128;
                    }
                    if (lane == 0) bar_expect(full, kQuant ? C::kCodes : C::kTile);
                    __syncwarp();
                    if (lane < n_box) tma_2d(dst, kv ? &v_map : &k_map, kQuant ? 0 : lane % kBoxSlabs * 64, kv ? values_row : row, full);
                    __syncwarp();
                }
            }
            it += uint32_t(g.t1 - g.t0);
        }
        // leave no copy in flight behind: where all went well they have landed long ago; otherwise the waits end after 1e8 cycles
        const long long t0 = clock64();
        auto landed = [&](uint32_t bar, uint32_t parity) { while (!bar_try(bar, parity) && clock64() - t0 < 100000000ll) {} };
        if constexpr (kQuant) {
            for (uint32_t n = staged > C::kStaging ? staged - C::kStaging : 0; n < staged; ++n) landed(st_full(n % C::kStaging), (n / C::kStaging) & 1);
        } else {
            for (uint32_t n = k_sent > C::kK ? k_sent - C::kK : 0; n < k_sent; ++n) landed(k_full(n % C::kK), (n / C::kK) & 1);
            for (uint32_t n = v_sent > C::kV ? v_sent - C::kV : 0; n < v_sent; ++n) landed(v_full(n % C::kV), (n / C::kV) & 1);
        }
    } else if (warp == C::kWarpMma) {
        // ---- matrix instructions ----
        constexpr uint32_t kDescS = mma_desc(C::kB, false, kBN), kDescO = mma_desc(C::kB, true, D);
        const uint32_t one = elect_one();
        uint32_t it = 0, seg = 0, jobs_of[2] = { 0, 0 };            // tiles before the segment; segments; jobs of each pipeline or S
        bool ok = true;
        auto commit = [&](uint32_t bar) { tc_commit_one(one, bar); };
        uint32_t x = plan.begin;
        for (Seg g; ok && segment(a, plan, x, g); ++seg) {
            const uint32_t n = uint32_t(g.t1 - g.t0);
            const int jobs = int(n) * (kTwo ? 2 : 1);
            // job k: tile k or k / 2 of the segment, row tile 0 or k % 2
            auto scores = [&](int k) {
                const int w = k & 1;
                const uint32_t item = it + uint32_t(kTwo ? k >> 1 : k), s = item % C::kK;
                if (!kTwo || w == 0) { if (!(ok = WAIT(k_full(s), (item / C::kK) & 1))) return; tc_after(); }
                const uint64_t qa = smem_desc(base + (kTwo ? w : 0) * C::kQ, 16, 1024), kb = smem_desc(base + C::kOffK + s * C::kTile, 16, 1024);
#pragma unroll
                for (int e = 0; e < D / 16; ++e)                    // (descriptors count 16 bytes)
                    mma_ss(one, tmem + C::kColS + w * 128, qa + (e / 4 * (kBM * 128) + e % 4 * 32) / 16, kb + (e / 4 * (kBN * 128) + e % 4 * 32) / 16, kDescS, e > 0);
                commit(s_full(w));
                if (!kTwo || w == 1) commit(k_empty(s));
            };
            if (!(ok = WAIT(q_full, seg & 1))) break;
            tc_after();
            scores(0);
            if (ok && jobs > 1) scores(1);
            for (int k = 0; ok && k < jobs; ++k) {
                const int w = k & 1;
                const uint32_t item = it + uint32_t(kTwo ? k >> 1 : k), s = item % C::kV;
                if (!kTwo || w == 0) { if (!(ok = WAIT(kQuant ? v_full(s) : v_ready(s), (item / C::kV) & 1))) break; }
                const uint64_t vb = smem_desc(base + C::kOffV + s * C::kTile, kBN * 128, 1024);
                auto product = [&](int e, bool more) { mma_ts(one, tmem + C::kColO + (kTwo ? w : 0) * D, tmem + C::kColS + w * 128 + C::col_p(e), vb + e * 2048 / 16, kDescO, more); };
                if constexpr (kTwo) {                               // the second half's weights come first: its product runs while the first's are worked out
                    if (!(ok = WAIT(p_half(w), jobs_of[w] & 1))) break;
                    tc_after();
#pragma unroll
                    for (int e = 4; e < 8; ++e) product(e, k >= 2 || e > 4);
                }
                if (!(ok = WAIT(kTwo ? p_full(w) : p_both(w), jobs_of[w] & 1))) break;
                ++jobs_of[w];
                tc_after();
#pragma unroll
                for (int e = 0; e < (kTwo ? 4 : 8); ++e) product(e, kTwo || k > 0 || e > 0);
                if (!kTwo) commit(o_done);
                if (!kTwo || w == 1) commit(v_empty(s));
                if (k + 2 < jobs) scores(k + 2);
            }
            if (ok) commit(done);
            it += n;
        }
        commit(drained);                                            // nor any matrix instruction, or its arrival at a barrier
        const long long t0 = clock64();
        while (!bar_try(drained, 0) && clock64() - t0 < 100000000ll) {}
    } else if (warp >= C::kWarpConvert) {
        const int t = tid - C::kWarpConvert * 32;
        uint32_t it = 0, staged = 0, next_page = ~0u;
        bool ok = true, next_on = false;
        float next_scale[2] = { 0.0f, 0.0f };
        // of a quantised cache: this thread's key's page of a tile; its scales, whose page has been looked up
        auto look_up = [&](const Seg& g, int tile) {
            const int key = g.key_of(tile) + t;
            next_page = tile < g.t1 && g.seen(a, key) ? uint32_t(__ldg(a.b.page_table + uint64_t(g.seq) * a.b.table_stride + (uint32_t(key) >> a.p.page_shift))) : ~0u;
        };
        auto scales_of = [&](const Seg& g, int tile) {
            const int key = g.key_of(tile) + t;
            next_on = next_page < a.p.n_pages;
            next_scale[0] = next_scale[1] = 0.0f;
            if (next_on) {
                const uint64_t cell = ((uint64_t(next_page) * hkv + uint32_t(g.h)) << a.p.page_shift) + (key & ((1 << a.p.page_shift) - 1));
                next_scale[0] = __ldg(a.p.k_scale + cell); next_scale[1] = __ldg(a.p.v_scale + cell);
            }
        };
        uint32_t x = plan.begin;
        for (Seg g; ok && segment(a, plan, x, g);) {
            const int32_t* table = a.b.page_table + uint64_t(g.seq) * a.b.table_stride;
            auto page_of = [&](int key) { return uint32_t(__ldg(table + (uint32_t(key) >> a.p.page_shift))); };
            if constexpr (kQuant) {
                // ---- codes of a staged tile to the operand layout, scales beside them: a key per thread; keys of a tile, then the values of the one before ----
                static_assert(C::kConvert * 32 == kBN, "a thread per key");
                constexpr int kChunks = D / 16;                     // 16 codes each
                uint32_t rows_on = 0;
                float v_scale = 0.0f;
                look_up(g, g.t0); scales_of(g, g.t0); look_up(g, g.t0 + 1);
                for (int tile = g.t0; ok && tile <= g.t1; ++tile) {
                    // (the scales of the next tile and the page of the one behind it are on their way meanwhile: three waits for memory a tile cost more than the widening)
                    const uint32_t values_on = rows_on;
                    const float scale[2] = { next_scale[0], v_scale };
                    if (tile < g.t1) {
                        rows_on = __ballot_sync(0xffffffffu, next_on);      // (the rows of a warp are its threads' keys)
                        v_scale = next_scale[1];
                        scales_of(g, tile + 1); look_up(g, tile + 2);
                    }
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv) {
                        if (kv ? tile == g.t0 : tile == g.t1) continue;
                        const uint32_t item = it + uint32_t(tile - g.t0) - uint32_t(kv), ss = staged % C::kStaging, s = item % (kv ? C::kV : C::kK), turn = item / (kv ? C::kV : C::kK);
                        if (!(ok = WAIT(st_full(ss), (staged / C::kStaging) & 1))) break;
                        if (turn && !(ok = WAIT(kv ? v_empty(s) : k_empty(s), (turn - 1) & 1))) break;
                        ++staged;
                        const uint32_t on = kv ? values_on : rows_on;
                        const uint8_t* from = smem + C::kOffStaging + ss * C::kCodes;
                        uint8_t* to = smem + (kv ? C::kOffV : C::kOffK) + s * C::kTile;
                        // a warp takes its 32 rows, neighbouring lanes neighbouring pieces of a row; all of a lane's pieces are read before the first is written
                        uint4 codes[kChunks];
#pragma unroll
                        for (int e = 0; e < kChunks; ++e) codes[e] = *reinterpret_cast<const uint4*>(from + t / 32 * 32 * D + (e * 32 + lane) * 16);
#pragma unroll
                        for (int e = 0; e < kChunks; ++e) {
                            const int c = lane % kChunks, r = t / 32 * 32 + e * (32 / kChunks) + lane / kChunks;
                            uint4 v = codes[e];
                            if (!(on >> (r & 31) & 1)) v = make_uint4(0, 0, 0, 0);
                            uint4 lo, hi;
                            widen4<CACHE>(v.x, lo.x, lo.y); widen4<CACHE>(v.y, lo.z, lo.w); widen4<CACHE>(v.z, hi.x, hi.y); widen4<CACHE>(v.w, hi.z, hi.w);
                            uint8_t* row = to + c / 4 * (kBN * 128) + r * 128;
                            const int p0 = ((2 * (c % 4)) ^ (r & 7)) * 16, p1 = ((2 * (c % 4) + 1) ^ (r & 7)) * 16;
                            if (c < 4) { *reinterpret_cast<uint4*>(row + p0) = lo; *reinterpret_cast<uint4*>(row + p1) = hi; }
                            else { *reinterpret_cast<uint4*>(row + p1) = hi; *reinterpret_cast<uint4*>(row + p0) = lo; }     // the other order: no bank twice
                        }
                        reinterpret_cast<float*>(smem + C::kOffScales)[(kv * 4 + item % 4) * kBN + t] = scale[kv];
                        fence_async_proxy();
                        bar_arrive(st_empty(ss));                   // (not before the codes have been used: right behind their loads, the next copy overtook some of those)
                        bar_arrive(kv ? v_full(s) : k_full(s));
                    }
                }
                it += uint32_t(g.t1 - g.t0);
            } else {
                for (int tile = g.t0; ok && tile < g.t1; ++tile, ++it) {
                    const int key0 = g.key_of(tile);
                    // ---- 16-bit values: those that no row of the unit sees become zeros (a weight of 0 does not silence a NaN), and so do, where some rows see them
                    // and others do not (mixed tiles alone), those that are no numbers: they are added to the rows that see them at the segment's end ----
                    const uint32_t s = it % C::kV;
                    if (!(ok = WAIT(v_full(s), (it / C::kV) & 1))) break;
                    const bool bad = *static_cast<volatile uint32_t*>(words + 3) & 1, mixed = g.mixed(a, key0);
                    if (bad || mixed) {
#pragma unroll 1
                        for (int r = t; r < kBN; r += 32) {
                            const int key = key0 + r;
                            const bool seen = g.seen(a, key) && (!bad || page_of(key) < a.p.n_pages);
                            uint8_t* row = smem + C::kOffV + s * C::kTile + r * 128;
                            auto piece = [&](int e) { return reinterpret_cast<uint4*>(row + e / 8 * (kBN * 128) + ((e ^ r) & 7) * 16); };     // (neighbours meet no bank twice)
                            uint32_t top = 0;
                            if (seen && mixed) {
#pragma unroll
                                for (int e = 0; e < 8 * C::kSlabs; ++e) largest_halves(top, *piece(e));
                            }
                            if (!seen || unreal2<BF>(top)) {
#pragma unroll 1
                                for (int e = 0; e < 8 * C::kSlabs; ++e) {
                                    const uint4 v = *piece(e);
                                    *piece(e) = seen ? make_uint4(real2<BF>(v.x), real2<BF>(v.y), real2<BF>(v.z), real2<BF>(v.w)) : make_uint4(0, 0, 0, 0);
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
    } else {
        // ---- softmax: pipeline w, a row per thread ----
        const int w = warp / 4, r = tid % 128;
        const uint32_t lanes = uint32_t(warp % 4 * 32) << 16;
        float f = a.scale_log2;                                     // what turns a product into x (over a quantised cache, of this row, and times the key's scale)
        const bool falling = a.scale_log2 < 0.0f;
        const uint32_t kHidden = falling ? 0x7f800000u : 0xff800000u;               // x f = -infinity
        uint32_t it = 0, seg = 0, scored[2] = { 0, 0 }, products = 0, meetings = 0, pairs = 0;      // tiles before the segment, segments, scores in each S so far, products of both halves, meetings
        bool ok = true;
        auto meet = [&] { bar_arrive(meeting); ok = WAIT(meeting, meetings & 1); ++meetings; return ok; };      // of both pipelines (bounded, as every wait here)
        auto token_of = [&](const Seg& g) { return g.tok0 + (kTwo ? w : 0) * plan.tq + r / int(G); };
        auto on_of = [&](const Seg& g) { return r < plan.tq * int(G) && token_of(g) < g.q_len; };
        // Brings the queries of the pipeline's row tile (where the pipelines share one, the first brings it), zeros where there is no row, and returns f.
        auto bring = [&](const Seg& g) {
            const bool on = on_of(g);
            float f = a.scale_log2;
            if (kTwo || w == 0 || (kQuant && BF)) {
                const uint4* from = reinterpret_cast<const uint4*>(a.q + (uint64_t(g.q0 + (on ? token_of(g) : 0)) * a.q_stride + (uint64_t(g.h) * G + r % int(G)) * D) * 2);
                uint8_t* row = smem + (kTwo ? w : 0) * C::kQ + r * 128;
                uint4 q[D / 8];
#pragma unroll
                for (int e = 0; e < D / 8; ++e) q[e] = on ? __ldg(from + e) : make_uint4(0, 0, 0, 0);
                if constexpr (kQuant && BF) {
                    float mul;
                    f *= lifted(q, mul);
                    // an infinity at a hidden key times f has to stay one (f rounded to 0 made NaN rows of faint queries at scales near 0); sums are below 2^128, so x moves by 2^-21 at most
                    if (f == 0.0f) f = copysignf(0x1p-149f, a.scale_log2);
#pragma unroll
                    for (int e = 0; e < D / 8; ++e)
                        q[e] = make_uint4(W::pack(A::lo(q[e].x) * mul, A::hi(q[e].x) * mul), W::pack(A::lo(q[e].y) * mul, A::hi(q[e].y) * mul),
                                          W::pack(A::lo(q[e].z) * mul, A::hi(q[e].z) * mul), W::pack(A::lo(q[e].w) * mul, A::hi(q[e].w) * mul));
                }
                if (kTwo || w == 0) {
#pragma unroll
                    for (int e = 0; e < D / 8; ++e) *reinterpret_cast<uint4*>(row + e / 8 * (kBM * 128) + ((e ^ r) & 7) * 16) = q[e];
                    fence_async_proxy();
                }
            }
            bar_arrive(q_full);
            return f;
        };
        uint32_t x = plan.begin;
        Seg g;
        bool more = segment(a, plan, x, g);
        if (more) f = bring(g);
        for (; ok && more; ++seg) {
            const int n = g.t1 - g.t0;
            const int rt = kTwo ? w : 0;                           // row tile of this pipeline
            const int tok = token_of(g);
            const bool row_on = on_of(g);
            const bool any_on = __any_sync(0xffffffffu, row_on);
            const int tree_row = g.q0 + min(tok, g.q_len - 1);
            // the row's masks, up to itself, where two words hold them (looked up tile by tile they cost a fifth of a call over short contexts)
            const bool short_tree = g.q_len <= 64;
            unsigned long long mask = 0;
            if (short_tree && row_on) {
                const uint32_t* from = a.tree + uint64_t(uint32_t(tree_row)) * a.tree_words;
                mask = __ldg(from) | (unsigned long long)(a.tree_words > 1 ? __ldg(from + 1) : 0u) << 32;
                mask &= tok < 63 ? (2ull << tok) - 1 : ~0ull;
            }
            const int depth_place = a.window && row_on ? g.place0 + tree_depth(a.tree, a.tree_words, tree_row, tok) : 0;      // where the window counts from
            const int32_t* table = a.b.page_table + uint64_t(g.seq) * a.b.table_stride;
            float m = kLow, l = 0.0f, unit = 0.0f, unit_inv = 0.0f; // unit: what the values' scales and so O are relative to, at least the largest of the segment's tiles so far
            bool bad_met = false;
                                auto visible = [&](int first) {        // the columns of keys [first, first + 32) that the row sees, a bit each
                                    const int rel = first - g.place0;
                                    uint32_t bits;
                                    if (short_tree) bits = rel <= -32 ? ~0u : rel >= 64 ? 0u : uint32_t(rel >= 0 ? mask >> rel : mask << -rel | ((1ull << -rel) - 1));
                                    else {
                                        const int end = min(max(tok - rel + 1, 0), 32);        // columns before `end` are not ahead of the row
                                        bits = (end == 32 ? ~0u : (1u << end) - 1) & tree_bits(a.tree, a.tree_words, tree_row, rel);
                                    }
                                    if (a.window) {
                                        const int from = min(max(depth_place - first + 1 - int(a.window), 0), min(max(-rel, 0), 32));      // context before `from` has left the window, unless it is a sink
                                        const int sunk = min(max(int(a.sinks) - first, 0), 32);
                                        bits &= (from == 32 ? 0u : ~0u << from) | (sunk == 32 ? ~0u : (1u << sunk) - 1);
                                    }
                                    if (bad_met)
            #pragma unroll 1
                                        for (int e = 0; e < 2; ++e)
                                            if (const int key = first + 16 * e; key >= 0 && key < g.kv && bits >> (16 * e) & 0xffffu && uint32_t(__ldg(table + (uint32_t(key) >> a.p.page_shift))) >= a.p.n_pages) bits &= ~(0xffffu << (16 * e));
                                    return row_on ? bits : 0u;
                                };
            // The scores of one S to weights: all 128 columns by one thread (kHalf false, S and O of the pipeline), or 64 by each of two, who tell one another their maxima.
            auto weigh = [&](auto masked_one, int key0, uint32_t item, uint32_t buffer, int tile) {
                constexpr bool kMasked = decltype(masked_one)::value, kHalf = !kTwo;
                const int cb = kHalf ? w * 64 : 0;
                const uint32_t tS = tmem + C::kColS + buffer * 128 + cb + lanes, tP = tmem + C::kColS + buffer * 128 + (kHalf ? cb : int(C::kColP)) + lanes;
                const uint32_t tO = tmem + C::kColO + w * (kHalf ? D / 2 : D) + lanes;
                const float* ks = reinterpret_cast<const float*>(smem + C::kOffScales) + item % 4 * kBN + cb;
                [[maybe_unused]] const float* vs = ks + 4 * kBN;
                // 32 columns: times the keys' scales where the cache has them, hidden ones put away
                auto fetch = [&](uint32_t* v, int c0) {
                    if constexpr (kQuant) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const ulonglong2 k4 = *reinterpret_cast<const ulonglong2*>(ks + c0 + e);
                            float y0, y1, y2, y3;
                            unpack2(mul2(pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), k4.x), y0, y1);
                            unpack2(mul2(pack2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), k4.y), y2, y3);
                            v[e] = __float_as_uint(y0); v[e + 1] = __float_as_uint(y1); v[e + 2] = __float_as_uint(y2); v[e + 3] = __float_as_uint(y3);
                        }
                    }
                    if constexpr (kMasked) {
                        const uint32_t bits = visible(key0 + cb + c0);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = bits & (1u << e) ? v[e] : kHidden;
                    }
                };
                uint32_t v0[32];
                [[maybe_unused]] uint32_t v1[32];
                float top = falling ? INFINITY : -INFINITY;
                auto widest = [&](const uint32_t* v) {
                    if (!falling) {
                        float t0 = top, t1 = -INFINITY;
#pragma unroll
                        for (int e = 0; e < 32; e += 4) { t0 = max3(t0, __uint_as_float(v[e]), __uint_as_float(v[e + 1])); t1 = max3(t1, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])); }
                        top = fmaxf(t0, t1);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) top = fminf(top, __uint_as_float(v[e]));
                    }
                };
                __syncwarp();
                if constexpr (kQuant) {                             // (the upper columns are read again: there are no registers to hold them, and spilling them cost more)
                    tm_ld32(tS + 32, v0);
                    tm_wait_ld32(v0);
                    fetch(v0, 32); widest(v0);
                    tm_ld32(tS, v0);
                    tm_wait_ld32(v0);
                    fetch(v0, 0); widest(v0);
                } else {
                    tm_ld32(tS, v0); tm_ld32(tS + 32, v1);
                    tm_wait_ld32(v0); tie32(v1);
                    fetch(v0, 0); widest(v0);
                    fetch(v1, 32); widest(v1);
                }
                if constexpr (!kHalf) {
                    __syncwarp();
                    tm_ld32(tS + 64, v0); tm_ld32(tS + 96, v1);
                    tm_wait_ld32(v0); tie32(v1);
                    fetch(v0, 64); widest(v0);
                    fetch(v1, 96); widest(v1);
                }
                top *= f;
                if constexpr (kHalf) {
                    float* tops = reinterpret_cast<float*>(smem + C::kOffTops) + (tile & 1) * 2 * kBM + r;
                    tops[w * kBM] = top;
                    bar_arrive(pair(warp % 4));                      // (both have read S as well: weights may go over it)
                    if (!(ok = WAIT(pair(warp % 4), pairs & 1))) return;
                    ++pairs;
                    top = fmaxf(top, tops[(w ^ 1) * kBM]);
                }
                if (!row_on) top = m;
                float largest = 0.0f;
                if constexpr (kQuant) {
                    if (!(ok = WAIT(v_full(item % C::kV), (item / C::kV) & 1))) return;       // the values' scales are there (the next turn of this stage waits for the product)
                    const float4 v4 = *reinterpret_cast<const float4*>(vs - cb + lane * 4);
                    largest = fmaxf(fmaxf(v4.x, v4.y), fmaxf(v4.z, v4.w));
                    largest = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(largest, unit))));      // (scales are not negative; a NaN is none here)
                }
                if (__any_sync(0xffffffffu, top > m + C::kLag) || largest > unit) {            // O so far shrinks
                    const float mn = fmaxf(m, top);
                    float less = ex2(m - mn);
                    l *= less; m = mn;
                    if (kQuant && largest > unit) { largest *= largest < 0x1p126f ? 2.0f : 1.0f; less *= __fdiv_rn(unit, largest); unit = largest; unit_inv = __fdiv_rn(1.0f, largest); }
                    if (tile > 0) {
                        // one S and O: the products into it were issued before these scores; two S and an O: the last product may be under way
                        if constexpr (kHalf) { if (!(ok = WAIT(o_done, (products + uint32_t(tile) - 1) & 1))) return; tc_after(); }
#pragma unroll 1
                        for (int c0 = 0; c0 < (kHalf ? D / 2 : D); c0 += 32) {
                            uint32_t o[32];
                            tm_ld32(tO + c0, o);
                            tm_wait_ld32(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * less);
                            tm_st16(tO + c0, o); tm_st16(tO + c0 + 16, o + 16);
                        }
                    }
                }
                // (by every thread for itself they cost 32 multiplications a tile)
                [[maybe_unused]] float* rel = reinterpret_cast<float*>(smem + C::kOffRel) + (kQuant ? warp * 64 : 0);
                if constexpr (kQuant) {
                    const float2 v2 = *reinterpret_cast<const float2*>(vs + lane * 2);
                    __syncwarp();
                    *reinterpret_cast<float2*>(rel + lane * 2) = make_float2(v2.x * unit_inv, v2.y * unit_inv);
                    __syncwarp();
                }
                const uint64_t f2 = pack2(f, f), m2 = pack2(C::kRaise - m, C::kRaise - m);
                uint64_t sum_a = pack2(0.0f, 0.0f), sum_b = sum_a;
                auto weights = [&](const uint32_t* v, int c0) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float y0, y1;
                        uint64_t y = fma2(pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), f2, m2);
                        // every fourth pair by a polynomial (12 x 61 tokens behind 16,001: 212 -> 207 us, every second one 214; quantised caches have no registers left for it)
                        if (kTwo && e % 8 == 6) { y = ex2_both(y); unpack2(y, y0, y1); }
                        else { unpack2(y, y0, y1); y0 = ex2(y0); y1 = ex2(y1); y = pack2(y0, y1); }
                        if (e % 4) sum_b = add2(sum_b, y); else sum_a = add2(sum_a, y);
                        if constexpr (kQuant) {
                            const ulonglong2 v4 = *reinterpret_cast<const ulonglong2*>(rel + c0 + e / 4 * 4);
                            unpack2(mul2(y, e % 4 ? v4.y : v4.x), y0, y1);
                            if constexpr (kMasked) { y0 = v[e] == kHidden ? 0.0f : y0; y1 = v[e + 1] == kHidden ? 0.0f : y1; }      // a hidden value's scale may be NaN
                        }
                        p[e / 2] = W::pack(y0, y1);
                    }
                    tm_st16(tP + c0 / 2, p);
                };
                if constexpr (kHalf) {
                    weights(v0, 0);
                    if constexpr (kQuant) {
                        tm_ld32(tS + 32, v0);
                        tm_wait_ld32(v0);
                        fetch(v0, 32); weights(v0, 32);
                    } else weights(v1, 32);
                } else {
                    weights(v0, 64);
                    tm_ld32(tS, v0);                                // read again: registers for one half only
                    weights(v1, 96);
                    tm_wait_st();
                    __syncwarp();
                    tc_before();
                    bar_arrive(p_half(w));
                    tm_ld32(tS + 32, v1);
                    tm_wait_ld32(v0); tie32(v1);
                    fetch(v0, 0); weights(v0, 0);
                    fetch(v1, 32); weights(v1, 32);
                }
                float s0, s1;
                unpack2(add2(sum_a, sum_b), s0, s1);
                l += s0 + s1;
                tm_wait_st();
            };
            for (int tile = 0; tile < n; ++tile) {
                const int key0 = g.key_of(g.t0 + tile);
                const uint32_t item = it + uint32_t(tile), buffer = kTwo ? uint32_t(w) : uint32_t(tile) & 1;
                if (!(ok = WAIT(s_full(buffer), (buffer ? scored[1] : scored[0]) & 1))) break;
                if (kTwo) { ++scored[0]; ++scored[1]; } else ++(buffer ? scored[1] : scored[0]);
                tc_after();
                if (any_on) {
                    bad_met = *static_cast<volatile uint32_t*>(words + 3) & 1;
                    const bool masked = bad_met || g.mixed(a, key0);
                    // (versions with and without masks: asking for every pair of weights cost a quantised cache more than the pairs)
                    using std::bool_constant;
                    if (masked) weigh(bool_constant<true>(), key0, item, buffer, tile); else weigh(bool_constant<false>(), key0, item, buffer, tile);
                    if (!ok) break;
                } else if (kTwo) bar_arrive(p_half(w));
                __syncwarp();
                tc_before();
                bar_arrive(kTwo ? p_full(w) : p_both(buffer));
            }
            if (!ok) break;
            it += uint32_t(n);
            if (!(ok = WAIT(done, seg & 1))) break;
            tc_after();
            // ---- the segment's result: of this thread's row, or, where the pipelines shared the rows, of half its columns ----
            constexpr bool joined = !kTwo;
            if (joined) products += uint32_t(n);
            float ll = l;
            if (joined) {
                reinterpret_cast<float*>(smem + C::kOffMl)[w * kBM + r] = l;
                if (!meet()) break;
                const float other = reinterpret_cast<const float*>(smem + C::kOffMl)[(w ^ 1) * kBM + r];
                ll = w ? other + l : l + other;
            }
            // the next segment's queries: its first scores are on their way while this one's result is written (before the last product was awaited it took no less)
            Seg after;
            more = segment(a, plan, x, after);
            if (more) f = bring(after);
            const uint32_t tO = tmem + C::kColO + (joined ? 0 : w) * D + lanes;
            const int c_from = joined ? w * (D / 2) : 0, c_to = joined ? c_from + D / 2 : D;
            const bool whole = g.t0 == 0 && g.t1 == g.tiles;
            const uint32_t slot = 2 * blockIdx.x + (g.x0 == plan.begin ? 0 : 1);
            uint8_t* dst = a.out + (uint64_t(g.q0 + (row_on ? tok : 0)) * a.out_stride + (uint64_t(g.h) * G + r % int(G)) * D) * 2;
            const float inv = ll > 0.0f ? 1.0f / ll : ll;           // 0: nothing seen; NaN stays NaN
            const bool unreal_met = !kQuant && (*static_cast<volatile uint32_t*>(words + 3) & 2);
#pragma unroll 1
            for (int c0 = c_from; c0 < c_to; c0 += 32) {
                uint32_t v[32];
                tm_ld32(tO + c0, v);
                tm_wait_ld32(v);
                float y[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) y[e] = kQuant ? __uint_as_float(v[e]) * unit : __uint_as_float(v[e]);
                if constexpr (!kQuant) {
                    if (unreal_met && row_on) {                     // values that are no numbers, to the rows that see them
#pragma unroll 1
                        for (int t = g.t0; t < g.t1; ++t) {
                            const int key0 = g.key_of(t);
                            if (!g.mixed(a, key0)) continue;
#pragma unroll 1
                            for (int key = key0; key < min(key0 + kBN, g.place0 + tok + 1); ++key) {
                                if (key < 0) continue;
                                const bool sees = key >= g.place0 ? (tree_bits(a.tree, a.tree_words, tree_row, key - g.place0) & 1u) != 0 : !a.window || key > depth_place - int(a.window) || key < int(a.sinks);
                                const uint32_t page = sees ? uint32_t(__ldg(table + (uint32_t(key) >> a.p.page_shift))) : ~0u;
                                if (page >= a.p.n_pages) continue;
                                const uint4* from = reinterpret_cast<const uint4*>(a.p.v + (((uint64_t(page) * hkv + uint32_t(g.h)) << a.p.page_shift) + (key & ((1 << a.p.page_shift) - 1))) * (D * 2) + c0 * 2);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint4 q = __ldg(from + e);
                                    const uint32_t u[4] = { q.x, q.y, q.z, q.w };
#pragma unroll
                                    for (int j = 0; j < 8; ++j) { const uint32_t half = u[j / 2] >> (j % 2 * 16) & 0xffffu; if (unreal<BF>(half)) y[8 * e + j] += A::lo(half); }
                                }
                            }
                        }
                    }
                    __syncwarp();
                }
                if (row_on) {
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            *reinterpret_cast<uint4*>(dst + (c0 + e) * 2) = make_uint4(A::pack(y[e] * inv, y[e + 1] * inv), A::pack(y[e + 2] * inv, y[e + 3] * inv),
                                                                                      A::pack(y[e + 4] * inv, y[e + 5] * inv), A::pack(y[e + 6] * inv, y[e + 7] * inv));
                    } else {
                        float4* part = reinterpret_cast<float4*>(a.s.part_o) + ((uint64_t(slot) * 2 + rt) * (D / 4) + c0 / 4) * kBM + r;      // [slot][row tile][D / 4][128] float4
#pragma unroll
                        for (int e = 0; e < 8; ++e) part[e * kBM] = make_float4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
                    }
                }
                __syncwarp();
            }
            if (!whole && row_on && (kTwo || w == 0)) a.s.part_ml[(slot * 2 + rt) * kBM + r] = make_float2(m, ll);
            tc_before();
            if (!whole) {
                // the unit's blocks are consecutive; the last to arrive joins their parts in that order
                const uint32_t u0 = g.x0 - uint32_t(g.t0), u1 = u0 + uint32_t(g.tiles);
                const uint32_t blk0 = u0 / plan.share, blk1 = (u1 - 1) / plan.share, first_slot = 2 * blk0 + (u0 % plan.share ? 1 : 0);
                if (!meet()) break;
                if (tid == 0) { __threadfence(); words[2] = atomicAdd(&a.s.ticket[first_slot], 1u) == blk1 - blk0; }
                __syncwarp();
                if (!meet()) break;
                if (words[2]) {
                    __threadfence();
                    if (row_on) {
                        auto slot_of = [&](uint32_t b) { return (b == blk0 ? first_slot : 2 * b) * 2 + rt; };
                        float tm = kLow, tl = 0.0f;
                        for (uint32_t b = blk0; b <= blk1; ++b) {
                            const float2 p = __ldcg(a.s.part_ml + slot_of(b) * kBM + r);
                            const float mn = fmaxf(tm, p.x);
                            tl = tl * ex2(tm - mn) + p.y * ex2(p.x - mn); tm = mn;
                        }
                        const float part_inv = tl > 0.0f ? 1.0f / tl : tl;
#pragma unroll 1
                        for (int c = c_from / 4; c < c_to / 4; c += 8) {
                            float4 acc[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) acc[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
                            for (uint32_t b = blk0; b <= blk1; ++b) {
                                const uint32_t s = slot_of(b);
                                const float by = ex2(__ldcg(a.s.part_ml + s * kBM + r).x - tm);
                                const float4* part = reinterpret_cast<const float4*>(a.s.part_o) + (uint64_t(s) * (D / 4) + c) * kBM + r;
#pragma unroll
                                for (int e = 0; e < 8; ++e) { const float4 v = __ldcg(part + e * kBM); acc[e].x += v.x * by; acc[e].y += v.y * by; acc[e].z += v.z * by; acc[e].w += v.w * by; }
                            }
#pragma unroll
                            for (int e = 0; e < 8; e += 2)
                                *reinterpret_cast<uint4*>(dst + (c + e) * 8) = make_uint4(A::pack(acc[e].x * part_inv, acc[e].y * part_inv), A::pack(acc[e].z * part_inv, acc[e].w * part_inv),
                                                                                          A::pack(acc[e + 1].x * part_inv, acc[e + 1].y * part_inv), A::pack(acc[e + 1].z * part_inv, acc[e + 1].w * part_inv));
                        }
                    }
                    if (tid == 0) a.s.ticket[first_slot] = 0;
                }
            }
            g = after;
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

cudaError_t launch_tree(const AttendArgs& a, uint32_t head_dim, int dtype, int cache, cudaStream_t s)
{
    const EncodeTiled encode = encoder();
    if (!encode) return cudaErrorNotSupported;
    const bool quant = cache != WWWS_CACHE_16;
    CUtensorMap maps[2];
    for (int kv = 0; kv < 2; ++kv) {
        const cuuint64_t dims[2] = { head_dim, uint64_t(a.p.n_pages) * a.p.n_kv_heads << a.p.page_shift };
        const cuuint64_t strides[1] = { head_dim * (quant ? 1ull : 2ull) };
        const cuuint32_t box[2] = { quant ? head_dim : 64, 1u << a.p.page_shift }, ones[2] = { 1, 1 };
        if (encode(&maps[kv], quant ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : dtype == WWWS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, kv ? a.p.v : a.p.k, dims, strides, box, ones,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, quant ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    // Two row tiles where the longest sequence has more than 128 rows (its shorter ones then leave the second empty).
    const bool two = !quant && uint64_t(a.b.max_q_len) * a.group > uint64_t(kBM / a.group * a.group);
    auto go = [&](auto bf, auto kind, auto dim, auto tiles) -> cudaError_t {
        constexpr bool kTwo = decltype(tiles)::value && decltype(kind)::value == WWWS_CACHE_16;
        using C = Cfg<decltype(bf)::value, decltype(kind)::value, decltype(dim)::value, kTwo>;
        static_assert(C::kFixed + (kTreeSeqs + 1) * 4 <= 232448 - 256, "shared memory of a block");
        constexpr auto kernel = k_tree<decltype(bf)::value, decltype(kind)::value, decltype(dim)::value, kTwo>;
        const uint32_t smem = C::kFixed + (a.b.n_seqs + 1) * 4;
        if (cudaError_t e = allow_smem<kernel>(C::kFixed + (kTreeSeqs + 1) * 4); e != cudaSuccess) return e;
        kernel<<<kTileBlocks, C::kThreads, smem, s>>>(a, maps[0], maps[1]);
        return cudaGetLastError();
    };
    using std::integral_constant;
    auto row_tiles = [&](auto bf, auto kind, auto dim) { return two ? go(bf, kind, dim, std::true_type()) : go(bf, kind, dim, std::false_type()); };
    auto dim = [&](auto bf, auto kind) { return head_dim == 64 ? row_tiles(bf, kind, integral_constant<int, 64>()) : row_tiles(bf, kind, integral_constant<int, 128>()); };
    auto kind = [&](auto bf) {
        return cache == WWWS_CACHE_16 ? dim(bf, integral_constant<int, 0>()) : cache == WWWS_CACHE_INT8 ? dim(bf, integral_constant<int, 1>()) : dim(bf, integral_constant<int, 2>());
    };
    return dtype == WWWS_BF16 ? kind(std::true_type()) : kind(std::false_type());
}

}  // namespace wwws
