// Attention of few rows per kv head over the paged cache (single tokens, a few drafted tokens).
//
// out_r = sum_j 2^(x_rj - m_r) v_j / sum_j 2^(x_rj - m_r),  x = scale * log2(e) * q_r . k_j,  m_r = max_j x_rj, computed in one pass over
// the keys with a running maximum and sum.  The query heads that share a kv head, times the sequence's new tokens, are the rows of one unit, so a
// key is read once for all of them.  Bound by HBM: a key and its value are head_dim * 2 (or 1) * 2 bytes for 4 * head_dim * rows operations, two
// orders of magnitude below the tensor peak, so the warp-level mma.sync does: what matters is how many bytes are in flight and how few instructions
// each costs.
//   - Keys are the 16 rows of the operand, query rows its 8 columns (S^T = K Q^T, O^T = V^T P^T): no half-empty 16-row tile of queries, and
//     kGroups = 1 or 2 groups of 8 rows share the fragments of a key.  (Up to 32 rows come here, 48 over a quantised cache, as units of 16, or of 8 where no
//     sequence has more.  One unit of 32 took 82 us where two of 16 take 66, five drafted tokens of 24 requests,
//     since it has registers for no more than half the warps' work in flight.)
//   - Work is cut by keys, not by sequences: all (sequence, row tile, kv head) units laid end to end in tiles of kTK keys, and block i takes
//     the i-th equal share (the lengths are read on the device: no plan, no host copy of them).  A unit cut by a share boundary leaves a
//     partial result (m, sum, weighted values) in the workspace; the last of its blocks to arrive joins them in block order,
//     so the result does not depend on who arrives last.
//   - Within a block the warps take every fourth tile of a segment, each with its own ring of cp.async stages (no block barrier
//     inside a segment), and join through shared memory at its end.
//   - A quantised tile is widened in registers on its way into the operand; its scales multiply the score (keys) and the softmax weight
//     (values), so the codes themselves, which f16 holds exactly, are the operands, whatever the activation type: bf16 queries become f16 by a
//     power of two per row (exact down to 2^-28 of the row's largest), and weights times value scales are kept relative to the largest value
//     scale so far.  Weights in f16 carry a factor 2^15, which cancels in the quotient and keeps small ones out of the subnormals.
// Fragments: mma.m16n8k16 leaves the order of the k index free as long as both operands agree.  For K Q^T a thread takes 16 consecutive bytes of
// its key's row (8 or 16 elements = 2 or 4 k-steps) and the query fragments follow that order; for 8-bit values, where no transposing load
// fits, a thread takes head_dim / 8 consecutive columns of four keys' rows and row tile i of V^T is columns 2i and 2i + 1 of each thread's.
// With WWWS_TREE the new tokens are a tree (kernels_attend_tree.cu): one of them sees another where its mask has a bit, the context as before.
#include "backend.cuh"

#ifndef WWWS_TREE
#define WWWS_TREE 0
#endif

namespace wwws {
namespace {

constexpr bool kTree = WWWS_TREE;

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr float kLow = -3.0e38f;            // below every score: 2^(x - kLow) is never formed, 2^(-inf - kLow) is 0

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

template <bool BF> __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2])
{
    if constexpr (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on)     // 16 bytes, or zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool on)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}

// Four codes to two pairs of f16: int8 by 0x6400 | (code ^ 0x80), which is 1024 + 128 + code, less 1152; e4m3 by the hardware's conversion.
template <int CACHE> __device__ __forceinline__ void widen4(uint32_t four, uint32_t& lo, uint32_t& hi)
{
    if constexpr (CACHE == WWWS_CACHE_INT8) {
        const uint32_t u = four ^ 0x80808080u;
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0x64806480u));
    } else {
        asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}" : "=r"(lo), "=r"(hi) : "r"(four));
    }
}

template <int CACHE, int D, int kGroups> struct Shape {
    static constexpr int kElem = CACHE == WWWS_CACHE_16 ? 2 : 1;
    static constexpr int kRow = D * kElem;              // bytes of a cached row
    static constexpr int kChunks = kRow / 16;
    static constexpr int kTK = kRow == 256 ? 16 : 32;   // keys per tile: 4 KB of keys where rows allow it
    static constexpr int kTile = kTK * kRow;
    static constexpr int kScales = CACHE == WWWS_CACHE_16 ? 0 : kTK * 8;
    static constexpr int kStage = 2 * kTile + kScales;
    // blocks of an SM: as many as registers allow; stages: what their shared memory allows
    static constexpr int kBlocks = kRow <= 128 && kGroups == 1 ? 3 : 2;
    static constexpr int kStages = kRow == 64 ? (kBlocks == 3 ? 4 : 5) : kBlocks == 3 ? 2 : 3;
    static constexpr int kRing = kStages * kStage;
    static constexpr int kSmem = kWarps * kRing;
    // where chunk c of key's row lies, so that the fragment loads below meet no bank twice
    static __device__ __forceinline__ int k_at(int key, int c) { return key * kRow + ((kChunks >= 8 ? c ^ ((key & 1) << 2) : c) << 4); }
    static __device__ __forceinline__ int v_at(int key, int c) { return key * kRow + ((CACHE == WWWS_CACHE_16 ? c ^ (key & 7) : kChunks == 8 ? c ^ (key & 6) : c ^ (key & 2)) << 4); }
};

// What a unit's rows can see of a sequence, in tiles: the first n_sink tiles, then those from lo_tile on.
struct Span { int n_sink, lo_tile, tiles; };
template <int TK> __device__ __forceinline__ Span span_of(int q_len, int kv, uint32_t window, uint32_t sinks)
{
    Span s;
    const int lo = window ? max(0, kv - q_len - int(window) + 1) : 0;
    s.lo_tile = min(lo / TK, (kv + TK - 1) / TK);
    s.n_sink = window ? min((min(int(sinks), kv) + TK - 1) / TK, s.lo_tile) : 0;
    s.tiles = max(1, s.n_sink + (kv + TK - 1) / TK - s.lo_tile);     // one (empty) tile even where nothing is seen: the rows get zeros
    return s;
}

template <bool BF, int CACHE, int D, int kGroups>
__global__ void __launch_bounds__(kThreads, Shape<CACHE, D, kGroups>::kBlocks) k_attend_rows(AttendArgs a)
{
    constexpr bool kQuant = CACHE != WWWS_CACHE_16;
    constexpr bool kB = BF && !kQuant;                       // the operands' type
    using A = Act<BF>;
    using W = Act<kB>;
    using S = Shape<CACHE, D, kGroups>;
    constexpr int TK = S::kTK, KT = TK / 16, kRows = 8 * kGroups;
    constexpr float kLift = kB ? 0.0f : 15.0f;               // log2 of the weights' common factor
    extern __shared__ __align__(128) uint8_t smem[];
    unsigned long long* prefix = reinterpret_cast<unsigned long long*>(smem + S::kSmem);   // [n_seqs + 1] tiles of all earlier sequences, per kv head
    __shared__ unsigned long long warp_sum[kWarps];
    __shared__ uint32_t last_flag;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, n = lane / 4, c = lane % 4;
    const uint32_t Hkv = a.p.n_kv_heads, G = a.group;

    // tiles of every sequence, and their running sum
    unsigned long long carry = 0;
    for (uint32_t base = 0; base < a.b.n_seqs; base += kThreads) {
        unsigned long long x = 0;
        if (base + tid < a.b.n_seqs) {
            int q0, q_len, kv;
            if (sequence(a.b, base + tid, q0, q_len, kv, a.err) && q_len)
                x = (unsigned long long)((uint32_t(q_len) * G + kRows - 1) / kRows) * (a.pad ? a.pad : span_of<TK>(q_len, kv, a.window, a.sinks).tiles);
        }
        const unsigned long long own = x;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) { const unsigned long long y = __shfl_up_sync(0xffffffffu, x, m); if (lane >= m) x += y; }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        unsigned long long before = carry;
        for (int w = 0; w < kWarps; ++w) { if (w < warp) before += warp_sum[w]; carry += warp_sum[w]; }
        if (base + tid < a.b.n_seqs) prefix[base + tid] = before + x - own;
        __syncthreads();
    }
    if (tid == 0) prefix[a.b.n_seqs] = carry;
    __syncthreads();
    const unsigned long long total = carry * Hkv;
    unsigned long long share = (total + gridDim.x - 1) / gridDim.x;
    if (share < kWarps) share = kWarps;
    if (a.pad) share = (share + a.pad - 1) / a.pad * a.pad;
    const unsigned long long begin = blockIdx.x * share, end = min(total, begin + share);

    const uint32_t ring = uint32_t(__cvta_generic_to_shared(smem)) + warp * S::kRing;
    const uint8_t* ring_g = smem + warp * S::kRing;
    float* comb_o = reinterpret_cast<float*>(smem);                                   // [kWarps][kRows][D], over the drained rings
    float2* comb_ml = reinterpret_cast<float2*>(comb_o + kWarps * kRows * D);   // [kWarps][kRows]

    for (unsigned long long x = begin; x < end;) {
        // the segment: unit (sequence i, row tile r, kv head h), its tiles [t0, t1)
        const unsigned long long per_head = x / Hkv;
        uint32_t i = 0, hi_seq = a.b.n_seqs;
        while (hi_seq - i > 1) { const uint32_t mid = (i + hi_seq) >> 1; if (prefix[mid] <= per_head) i = mid; else hi_seq = mid; }
        const int q0 = a.b.q_start[i], q_len = a.b.q_start[i + 1] - q0, kv = a.b.kv_len[i];
        const Span sp = span_of<TK>(q_len, kv, a.window, a.sinks);
        const unsigned long long rel = x - prefix[i] * Hkv;
        const uint32_t counted = a.pad ? a.pad : uint32_t(sp.tiles), unit = uint32_t(rel / counted);
        const int t0 = int(rel - (unsigned long long)unit * counted);
        const int t1 = a.pad ? sp.tiles : int(min((unsigned long long)sp.tiles, t0 + (end - x)));
        const uint32_t h = unit % Hkv, row0 = unit / Hkv * kRows;
        const int n_rows = min(int(kRows), q_len * int(G) - int(row0));
        const int place0 = kv - q_len;                                   // place of the sequence's first new token
        const int first_place = place0 + int(row0 / G), last_place = place0 + int((row0 + n_rows - 1) / G);
        const int lo_key = a.window ? max(0, (kTree ? place0 : first_place) - int(a.window) + 1) : 0, hi_key = min(kv, last_place + 1);

        // Query fragments (columns are rows n + 8 g), in the order in which the keys' chunks are taken.  Quantised: f16 times 2^e of the row, whose
        // largest element then lies in [2^14, 2^15); rm is what turns a product into x.
        uint32_t qb[kGroups][D / 16][2];
        float rm[kGroups][2];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int r = n + 8 * g;
            const uint4* from = reinterpret_cast<const uint4*>(a.q + (uint64_t(q0 + int((row0 + min(r, n_rows - 1)) / G)) * a.q_stride + (uint64_t(h) * G + (row0 + min(r, n_rows - 1)) % G) * D) * 2);
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const uint4 u = __ldg(from + (kQuant ? (4 * (s / 2) + c) * 2 + s % 2 : 4 * s + c));
                qb[g][2 * s][0] = u.x; qb[g][2 * s][1] = u.y; qb[g][2 * s + 1][0] = u.z; qb[g][2 * s + 1][1] = u.w;
            }
            float mine = a.scale_log2;
            if constexpr (kQuant && BF) {
                uint32_t top = 0;
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
#pragma unroll
                    for (int e = 0; e < 2; ++e) top = max(top, max(qb[g][s][e] << 16 & 0x7fffffffu, qb[g][s][e] & 0x7fff0000u));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1)); top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const uint32_t ex = top >> 23;                // 0: all zero or subnormal, 255: a NaN or an infinity
                const uint32_t me = ex == 0 || ex == 255 ? 127 : min(max(127 + 127 + 14 - int(ex), 1), 253);
                const float mul = __uint_as_float(me << 23);
                mine *= __uint_as_float((254 - me) << 23);
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
#pragma unroll
                    for (int e = 0; e < 2; ++e) qb[g][s][e] = W::pack(A::lo(qb[g][s][e]) * mul, A::hi(qb[g][s][e]) * mul);
            }
            rm[g][0] = __shfl_sync(0xffffffffu, mine, 8 * c); rm[g][1] = __shfl_sync(0xffffffffu, mine, 8 * c + 4);
        }
        // this thread's rows are the columns 2 c and 2 c + 1 of each group
        auto place_of = [&](int g, int e) { return place0 + int((row0 + min(8 * g + 2 * c + e, n_rows - 1)) / G); };

        float o[kGroups][D / 16][4], m[kGroups][2], l[kGroups][2], unit_v = 0.0f, unit_inv = 0.0f;      // largest value scale so far, its inverse
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            m[g][0] = m[g][1] = kLow; l[g][0] = l[g][1] = 0.0f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[g][d][0] = o[g][d][1] = o[g][d][2] = o[g][d][3] = 0.0f;
        }

        const int32_t* table = a.b.page_table + uint64_t(i) * a.b.table_stride;
        const int page_mask = (1 << a.p.page_shift) - 1;
        auto key_of = [&](int t) { return (t < sp.n_sink ? t : sp.lo_tile + t - sp.n_sink) * TK; };
        // whether a row of the unit sees any of 16 keys; a page of which none is seen may be someone else's by now and is not looked up
        auto some = [&](int kg) { return kg < hi_key && (kg + 16 > lo_key || kg < int(a.sinks)); };
        auto pages_of = [&](int t, uint32_t (&pg)[KT]) {
#pragma unroll
            for (int g = 0; g < KT; ++g) {
                const int key = key_of(t) + 16 * g;
                pg[g] = t < t1 && some(key) ? uint32_t(__ldg(table + (key >> a.p.page_shift))) : 0u;
            }
        };
        bool bad = false;                                    // this warp has met a page outside the pool: such keys are looked for, and hidden
        // copies one tile of keys and values (zeros for keys that no row of the unit sees)
        auto issue = [&](int t, int stage, const uint32_t (&pg)[KT]) {
            if (t < t1) {
                const int key0 = key_of(t);
                const uint32_t dst = ring + stage * S::kStage;
#pragma unroll
                for (int g = 0; g < KT; ++g) {
                    const int kg = key0 + 16 * g;
                    bool ok = some(kg);
                    if (ok && pg[g] >= a.p.n_pages) { report(a.err, bePage); ok = false; bad = true; }
                    const int64_t cell = ok ? (((int64_t(pg[g]) * Hkv + h) << a.p.page_shift) + (kg & page_mask)) : 0;
                    constexpr int kPer = 16 * S::kChunks / 32;
                    const uint8_t* ksrc = a.p.k + cell * S::kRow + lane * 16;
                    const uint8_t* vsrc = a.p.v + cell * S::kRow + lane * 16;
                    if (ok && kg + 16 <= hi_key && (kg >= lo_key || kg + 16 <= int(a.sinks))) {      // 16 keys that some row sees
#pragma unroll
                        for (int e = 0; e < kPer; ++e) {
                            const int ci = lane + 32 * e, kk = 16 * g + ci / S::kChunks, ch = ci % S::kChunks;
                            cp16(dst + S::k_at(kk, ch), ksrc + e * 512);
                            cp16(dst + S::kTile + S::v_at(kk, ch), vsrc + e * 512);
                        }
                        if constexpr (kQuant) cp4(dst + 2 * S::kTile + (lane / 16 * TK + 16 * g + lane % 16) * 4, (lane < 16 ? a.p.k_scale : a.p.v_scale) + cell + lane % 16, true);
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const int ci = lane + 32 * e, kk = ci / S::kChunks, ch = ci % S::kChunks, key = kg + kk;
                        const bool on = ok && key < hi_key && (key >= lo_key || key < int(a.sinks));
                        cp16(dst + S::k_at(16 * g + kk, ch), on ? ksrc + e * 512 : a.p.k, on);
                        cp16(dst + S::kTile + S::v_at(16 * g + kk, ch), on ? vsrc + e * 512 : a.p.v, on);
                    }
                    if constexpr (kQuant) {
                        const int kk = lane % 16, key = kg + kk;
                        const bool on = ok && key < hi_key && (key >= lo_key || key < int(a.sinks));
                        cp4(dst + 2 * S::kTile + (lane / 16 * TK + 16 * g + kk) * 4, (lane < 16 ? a.p.k_scale : a.p.v_scale) + cell + (on ? kk : 0), on);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };

        uint32_t pg[KT];
        pages_of(t0 + warp, pg);
#pragma unroll
        for (int s = 0; s < S::kStages - 1; ++s) {
            uint32_t next[KT];
            pages_of(t0 + warp + kWarps * (s + 1), next);
            issue(t0 + warp + kWarps * s, s, pg);
#pragma unroll
            for (int g = 0; g < KT; ++g) pg[g] = next[g];
        }
        int stage = 0;
        for (int t = t0 + warp; t < t1; t += kWarps) {
            asm volatile("cp.async.wait_group %0;" :: "n"(S::kStages - 2) : "memory");
            __syncwarp();
            {   // refill the stage that the previous turn emptied
                const int ahead = t + kWarps * (S::kStages - 1);
                uint32_t next[KT];
                pages_of(ahead + kWarps, next);
                issue(ahead, stage == 0 ? S::kStages - 1 : stage - 1, pg);
#pragma unroll
                for (int g = 0; g < KT; ++g) pg[g] = next[g];
            }
            const uint8_t* kt = ring_g + stage * S::kStage;
            const uint8_t* vt = kt + S::kTile;
            const int key0 = key_of(t);

            // S^T: keys n, n + 8 of each 16, columns 2 c, 2 c + 1 of each group
            float s[kGroups][KT][4];
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int k = 0; k < KT; ++k) s[g][k][0] = s[g][k][1] = s[g][k][2] = s[g][k][3] = 0.0f;
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int u = 0; u < S::kChunks / 4; ++u) {
                    const uint4 x = *reinterpret_cast<const uint4*>(kt + S::k_at(k * 16 + n, 4 * u + c)), y = *reinterpret_cast<const uint4*>(kt + S::k_at(k * 16 + n + 8, 4 * u + c));
                    if constexpr (!kQuant) {
#pragma unroll
                        for (int g = 0; g < kGroups; ++g) {
                            mma<kB>(s[g][k], x.x, y.x, x.y, y.y, qb[g][2 * u]);
                            mma<kB>(s[g][k], x.z, y.z, x.w, y.w, qb[g][2 * u + 1]);
                        }
                    } else {
                        const uint32_t xs[4] = { x.x, x.y, x.z, x.w }, ys[4] = { y.x, y.y, y.z, y.w };
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t x0, x1, y0, y1;
                            widen4<CACHE>(xs[e], x0, x1); widen4<CACHE>(ys[e], y0, y1);
#pragma unroll
                            for (int g = 0; g < kGroups; ++g) mma<kB>(s[g][k], x0, y0, x1, y1, qb[g][4 * u + e]);
                        }
                    }
                }
            const float* scales = reinterpret_cast<const float*>(vt + S::kTile);
            const bool masked = bad || key0 + TK - 1 > (kTree ? place0 - 1 : first_place) || (a.window && key0 < last_place - int(a.window) + 1 && key0 + TK > int(a.sinks));
            // value scales relative to the largest so far
            float vs[KT][2];
            if constexpr (kQuant) {
                float top = 0.0f;
#pragma unroll
                for (int k = 0; k < KT; ++k) { vs[k][0] = scales[TK + k * 16 + n]; vs[k][1] = scales[TK + k * 16 + n + 8]; top = fmaxf(top, fmaxf(vs[k][0], vs[k][1])); }
                if (__any_sync(0xffffffffu, top > unit_v)) {
#pragma unroll
                    for (int e = 4; e < 32; e <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, e));
                    const float f = __fdiv_rn(unit_v, top);
                    unit_v = top; unit_inv = __fdiv_rn(1.0f, top);
#pragma unroll
                    for (int g = 0; g < kGroups; ++g)
#pragma unroll
                        for (int d = 0; d < D / 16; ++d) { o[g][d][0] *= f; o[g][d][1] *= f; o[g][d][2] *= f; o[g][d][3] *= f; }
                }
#pragma unroll
                for (int k = 0; k < KT; ++k) { vs[k][0] *= unit_inv; vs[k][1] *= unit_inv; }
            }
            uint32_t pf[kGroups][KT][2];                     // P^T fragments
            bool moved = false;
            float top[kGroups][2];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    float f0 = 1.0f, f1 = 1.0f;
                    if constexpr (kQuant) { f0 = scales[k * 16 + n]; f1 = scales[k * 16 + n + 8]; }
                    s[g][k][0] *= rm[g][0] * f0; s[g][k][1] *= rm[g][1] * f0; s[g][k][2] *= rm[g][0] * f1; s[g][k][3] *= rm[g][1] * f1;
                }
                if (masked) {
                    uint32_t drafted[2] = { 0, 0 };
                    int left[2] = { 0, 0 };                  // context up to here has left the window
                    if constexpr (kTree) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int tok = place_of(g, e) - place0;
                            drafted[e] = tree_bits(a.tree, a.tree_words, q0 + tok, key0 - place0);
                            if (a.window) left[e] = place0 + tree_depth(a.tree, a.tree_words, q0 + tok, tok) - int(a.window);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < KT; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if constexpr (kTree) {
                                const int at = k * 16 + n + 8 * (e >> 1), key = key0 + at;
                                if (key > place_of(g, e & 1) || !(drafted[e & 1] >> at & 1u) || (a.window && key < place0 && key <= left[e & 1] && key >= int(a.sinks))) s[g][k][e] = -INFINITY;
                                continue;
                            }
                            const int key = key0 + k * 16 + n + 8 * (e >> 1), p = place_of(g, e & 1);
                            if (key > p || (a.window && key <= p - int(a.window) && key >= int(a.sinks))) s[g][k][e] = -INFINITY;
                        }
                    if (bad) {
#pragma unroll
                        for (int k = 0; k < KT; ++k)
                            if (const int kg = key0 + 16 * k; some(kg) && uint32_t(__ldg(table + (kg >> a.p.page_shift))) >= a.p.n_pages)
                                s[g][k][0] = s[g][k][1] = s[g][k][2] = s[g][k][3] = -INFINITY;
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float t = fmaxf(s[g][0][e], s[g][0][e + 2]);
#pragma unroll
                    for (int k = 1; k < KT; ++k) t = fmaxf(t, fmaxf(s[g][k][e], s[g][k][e + 2]));
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
                    top[g][e] = t;
                    moved = moved || t > m[g][e];
                }
            }
            if (__any_sync(0xffffffffu, moved)) {            // a maximum moved: earlier sums shrink
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const float x0 = fmaxf(top[g][0], m[g][0]), x1 = fmaxf(top[g][1], m[g][1]), c0 = ex2(m[g][0] - x0), c1 = ex2(m[g][1] - x1);
                    m[g][0] = x0; m[g][1] = x1; l[g][0] *= c0; l[g][1] *= c1;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) { o[g][d][0] *= c0; o[g][d][1] *= c1; o[g][d][2] *= c0; o[g][d][3] *= c1; }
                }
            }
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const float m0 = m[g][0] - kLift, m1 = m[g][1] - kLift;
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    float p0 = ex2(s[g][k][0] - m0), p1 = ex2(s[g][k][1] - m1), p2 = ex2(s[g][k][2] - m0), p3 = ex2(s[g][k][3] - m1);
                    l[g][0] += p0 + p2; l[g][1] += p1 + p3;
                    if constexpr (kQuant) {
                        p0 *= vs[k][0]; p1 *= vs[k][0]; p2 *= vs[k][1]; p3 *= vs[k][1];
                        if (masked) {                        // a hidden value's scale may be NaN
                            p0 = s[g][k][0] == -INFINITY ? 0.0f : p0; p1 = s[g][k][1] == -INFINITY ? 0.0f : p1;
                            p2 = s[g][k][2] == -INFINITY ? 0.0f : p2; p3 = s[g][k][3] == -INFINITY ? 0.0f : p3;
                        }
                    }
                    // 8 keys x 8 rows, transposed: row n, keys 2 c and 2 c + 1
                    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(pf[g][k][0]) : "r"(W::pack(p0, p1)));
                    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(pf[g][k][1]) : "r"(W::pack(p2, p3)));
                }
            }
            if constexpr (!kQuant) {
                if (masked && (kTree || first_place != last_place)) {   // (rows of one token see the same keys; five drafted tokens of 24 requests: 74.4 -> 76.9 us)
                    uint8_t* values = smem + (vt - smem);
                    uint32_t top_half = 0;
#pragma unroll
                    for (int e = 0; e < S::kTile / 512; ++e) largest_halves(top_half, *reinterpret_cast<const uint4*>(values + e * 512 + lane * 16));
                    if (__any_sync(0xffffffffu, unreal2<BF>(top_half))) {
#pragma unroll 1
                        for (int kk = 0; kk < TK; ++kk) {
                            auto value = [&](int d) { return uint32_t(*reinterpret_cast<const uint16_t*>(values + S::v_at(kk, d / 8) + d % 8 * 2)); };
                            auto sees = [&](int g, int e) {
                                const int key = key0 + kk, p = place_of(g, e);
                                if constexpr (kTree) {
                                    const int tok = p - place0;
                                    if (key >= place0) return key <= p && (tree_bits(a.tree, a.tree_words, q0 + tok, key - place0) & 1u) != 0;
                                    return !a.window || key > place0 + tree_depth(a.tree, a.tree_words, q0 + tok, tok) - int(a.window) || key < int(a.sinks);
                                }
                                return key <= p && (!a.window || key > p - int(a.window) || key < int(a.sinks));
                            };
#pragma unroll
                            for (int d = 0; d < D / 16; ++d) {
                                const uint32_t v0 = value(16 * d + n), v1 = value(16 * d + n + 8);
#pragma unroll
                                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        if (unreal<BF>(v0) && sees(g, e)) o[g][d][e] += A::lo(v0);
                                        if (unreal<BF>(v1) && sees(g, e)) o[g][d][e + 2] += A::lo(v1);
                                    }
                            }
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int e = 0; e < S::kTile / 512; ++e) {
                            uint4* x = reinterpret_cast<uint4*>(values + e * 512 + lane * 16);
                            *x = make_uint4(real2<BF>(x->x), real2<BF>(x->y), real2<BF>(x->z), real2<BF>(x->w));
                        }
                        __syncwarp();
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                if constexpr (!kQuant) {
                    // blocks (keys 0-7, columns 0-7), (keys 0-7, columns 8-15), (keys 8-15, ...) of 16 keys x 16 columns, transposed
                    const int key = 16 * k + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        uint32_t r0, r1, r2, r3;
                        const uint32_t at = uint32_t(__cvta_generic_to_shared(vt)) + S::v_at(key, 2 * d + ((lane >> 3) & 1));
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(at) : "memory");
#pragma unroll
                        for (int g = 0; g < kGroups; ++g) mma<kB>(o[g][d], r0, r1, r2, r3, pf[g][k]);
                    }
                } else {
                    constexpr int kWords = D / 32;           // words of a thread's columns of one key
                    uint32_t v[4][kWords];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = 16 * k + 2 * c + (e & 1) + (e >> 1) * 8;
                        if constexpr (kWords == 4) {
                            const uint4 x = *reinterpret_cast<const uint4*>(vt + S::v_at(key, n));
                            v[e][0] = x.x; v[e][1] = x.y; v[e][2] = x.z; v[e][3] = x.w;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2*>(vt + S::v_at(key, n >> 1) + (n & 1) * 8);
                            v[e][0] = x.x; v[e][1] = x.y;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kWords; ++i) {
                        // columns 4 i .. 4 i + 3 of keys (0, 1) and (8, 9), side by side
                        uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
                        widen4<CACHE>(__byte_perm(v[0][i], v[1][i], 0x5140), a0, a1); widen4<CACHE>(__byte_perm(v[0][i], v[1][i], 0x7362), a2, a3);
                        widen4<CACHE>(__byte_perm(v[2][i], v[3][i], 0x5140), b0, b1); widen4<CACHE>(__byte_perm(v[2][i], v[3][i], 0x7362), b2, b3);
#pragma unroll
                        for (int g = 0; g < kGroups; ++g) {
                            mma<kB>(o[g][2 * i], a0, a1, b0, b1, pf[g][k]);
                            mma<kB>(o[g][2 * i + 1], a2, a3, b2, b3, pf[g][k]);
                        }
                    }
                }
            }
            __syncwarp();
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();                       // every warp is done with its ring
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float t = l[g][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
                const int r = 8 * g + 2 * c + e;
                if (n == 0) comb_ml[warp * kRows + r] = make_float2(m[g][e], t);
                float* ow = comb_o + (warp * kRows + r) * D;
                const float back = kQuant ? unit_v : 1.0f;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
                    // columns of row tile d: 16 d + n and + 8 (values as given), n D / 8 + 2 d and + 1 (8-bit values)
                    const int d0 = kQuant ? n * (D / 8) + 2 * d : 16 * d + n;
                    ow[d0] = o[g][d][e] * back; ow[d0 + (kQuant ? 1 : 8)] = o[g][d][e + 2] * back;
                }
            }
        }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == sp.tiles;
        // a segment at the start of the block's share goes to the block's slot 0, another to slot 1
        const uint32_t slot = 2 * blockIdx.x + (x == begin ? 0 : 1);
        auto store = [&](int r, int d, float v0, float v1, float l) {
            const float f = l > 0.0f ? 1.0f / l : l;       // l = 0: nothing seen; l = NaN stays NaN
            const uint32_t row = row0 + r;
            *reinterpret_cast<uint32_t*>(a.out + (uint64_t(q0 + int(row / G)) * a.out_stride + (uint64_t(h) * G + row % G) * D + d) * 2) = A::pack(v0 * f, v1 * f);
        };
        for (int e = tid; e < n_rows * (D / 2); e += kThreads) {
            const int r = e / (D / 2), d = e % (D / 2) * 2;
            float m = kLow, l = 0.0f, v0 = 0.0f, v1 = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, comb_ml[w * kRows + r].x);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 ml = comb_ml[w * kRows + r];
                const float f = ex2(ml.x - m);
                const float2 v = *reinterpret_cast<const float2*>(comb_o + (w * kRows + r) * D + d);
                l += ml.y * f; v0 += v.x * f; v1 += v.y * f;
            }
            if (whole) store(r, d, v0, v1, l);
            else {
                *reinterpret_cast<float2*>(a.s.part_o + (uint64_t(slot) * kDecodeRows + r) * D + d) = make_float2(v0, v1);
                if (d == 0) a.s.part_ml[slot * kDecodeRows + r] = make_float2(m, l);
            }
        }
        if (!whole) {
            // the unit's blocks are consecutive; the last to arrive joins their partial results in that order
            const unsigned long long u0 = x - t0, u1 = u0 + sp.tiles;
            const uint32_t blk0 = uint32_t(u0 / share), blk1 = uint32_t((u1 - 1) / share);
            const uint32_t first_slot = 2 * blk0 + (u0 % share ? 1 : 0);
            __threadfence();
            __syncthreads();
            if (tid == 0) last_flag = atomicAdd(&a.s.ticket[first_slot], 1u) == blk1 - blk0;
            __syncthreads();
            if (last_flag) {
                __threadfence();
                for (int e = tid; e < n_rows * (D / 2); e += kThreads) {
                    const int r = e / (D / 2), d = e % (D / 2) * 2;
                    float m = kLow, l = 0.0f, v0 = 0.0f, v1 = 0.0f;
                    constexpr uint32_t kAtOnce = 8;             // parts whose loads are in flight together
                    for (uint32_t k0 = blk0; k0 <= blk1; k0 += kAtOnce) {
                        float2 ml[kAtOnce], v[kAtOnce];
#pragma unroll
                        for (uint32_t k = 0; k < kAtOnce; ++k) {
                            ml[k] = make_float2(kLow, 0.0f); v[k] = make_float2(0.0f, 0.0f);
                            if (k0 + k <= blk1) {
                                const uint32_t s = k0 + k == blk0 ? first_slot : 2 * (k0 + k);
                                ml[k] = __ldcg(a.s.part_ml + s * kDecodeRows + r);
                                v[k] = __ldcg(reinterpret_cast<const float2*>(a.s.part_o + (uint64_t(s) * kDecodeRows + r) * D + d));
                            }
                        }
#pragma unroll
                        for (uint32_t k = 0; k < kAtOnce; ++k) {
                            const float mn = fmaxf(m, ml[k].x), f0 = ex2(m - mn), f1 = ex2(ml[k].x - mn);
                            l = l * f0 + ml[k].y * f1; v0 = v0 * f0 + v[k].x * f1; v1 = v1 * f0 + v[k].y * f1;
                            m = mn;
                        }
                    }
                    store(r, d, v0, v1, l);
                }
                if (tid == 0) a.s.ticket[first_slot] = 0;
            }
        }
        __syncthreads();                       // the joined rows are read before the rings fill again
        x += a.pad ? a.pad : t1 - t0;
    }
}

}  // namespace

// `rows`: rows per kv head of the longest sequence that comes here.
#if WWWS_TREE
#define launch_attend_rows launch_attend_rows_tree
#endif
cudaError_t launch_attend_rows(const AttendArgs& a, uint32_t rows, uint32_t head_dim, int dtype, int cache, cudaStream_t s)
{
    auto go = [&](auto bf, auto kind, auto dim, auto groups) -> cudaError_t {
        constexpr int D = decltype(dim)::value, CACHE = decltype(kind)::value, kGroups = decltype(groups)::value;
        using S = Shape<CACHE, D, kGroups>;
        static_assert(S::kSmem >= kWarps * 8 * kGroups * (D + 2) * 4, "the joined rows fit the rings");
        constexpr auto kernel = k_attend_rows<decltype(bf)::value, CACHE, D, kGroups>;
        const uint32_t smem = S::kSmem + (a.b.n_seqs + 1) * 8;
        if (cudaError_t e = allow_smem<kernel>(S::kSmem + 2049 * 8); e != cudaSuccess) return e;
        const uint64_t row_tiles = (rows + 8 * kGroups - 1) / (8 * kGroups);
        const uint64_t units = uint64_t(a.b.n_seqs) * row_tiles * a.p.n_kv_heads, most = 148 * S::kBlocks;
        uint64_t tiles = (a.b.max_kv_len + S::kTK - 1) / S::kTK;             // of a unit, at most
        const uint64_t seen = (a.sinks + S::kTK - 1) / S::kTK + (uint64_t(a.window) + a.b.max_q_len) / S::kTK + 2;
        if (a.window && seen < tiles) tiles = seen;
        // Units of at most 16 tiles are not cut: each counts the same number of tiles and shares end between units, which saves the parts and their
        // joining (one request of 300 tokens: 8.7 us on the GPU cut, 5.8 uncut) and costs some balance, little against it at this size.
        AttendArgs args = a;
        args.pad = tiles <= 16 ? uint32_t(tiles ? tiles : 1) : 0;
        // (one at least: where max_q_len is 0 it reports the sequences that have tokens)
        const uint64_t blocks = args.pad ? units : (units * (tiles + 1) + kWarps - 1) / kWarps;
        kernel<<<uint32_t(blocks < 1 ? 1 : blocks < most ? blocks : most), kThreads, smem, s>>>(args);
        return cudaGetLastError();
    };
    using std::integral_constant;
    auto group = [&](auto bf, auto kind, auto dim) {
        return rows <= 8 ? go(bf, kind, dim, integral_constant<int, 1>()) : go(bf, kind, dim, integral_constant<int, 2>());
    };
    auto dim = [&](auto bf, auto kind) { return head_dim == 64 ? group(bf, kind, integral_constant<int, 64>()) : group(bf, kind, integral_constant<int, 128>()); };
    auto kind = [&](auto bf) {
        return cache == WWWS_CACHE_16 ? dim(bf, integral_constant<int, 0>()) : cache == WWWS_CACHE_INT8 ? dim(bf, integral_constant<int, 1>()) : dim(bf, integral_constant<int, 2>());
    };
    return dtype == WWWS_BF16 ? kind(std::true_type()) : kind(std::false_type());
}

}  // namespace wwws
