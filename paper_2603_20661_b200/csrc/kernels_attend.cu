// Attention of few rows per kv head over the paged cache (single tokens, a few drafted tokens).
//
// out_r = sum_j 2^(x_rj - m_r) v_j / sum_j 2^(x_rj - m_r),  x = scale * log2(e) * q_r . k_j,  m_r = max_j x_rj, computed in one pass over
// the keys with a running maximum and sum.  The query heads that share a kv head, times the sequence's new tokens, are the rows of one
// 16-row tile, so a key is read once for all of them.  Bound by HBM: a key and its value are head_dim * 2 (or 1) * 2 bytes for
// 4 * head_dim * rows operations, two orders of magnitude below the tensor peak, so the warp-level mma.sync does: what matters
// is how many bytes are in flight.
//   - Work is cut by keys, not by sequences: all (sequence, row tile, kv head) units laid end to end in tiles of kTK keys, and block i takes
//     the i-th equal share (the lengths are read on the device: no plan, no host copy of them).  A unit cut by a share boundary leaves a
//     partial result (m, sum, weighted values) in the workspace; the last of its blocks to arrive joins them in block order,
//     so the result does not depend on who arrives last.
//   - Within a block the warps take every fourth tile of a segment, each with its own ring of cp.async stages (no block barrier
//     inside a segment), and join through shared memory at its end.
//   - A quantised tile is widened in registers on its way into the tensor operand; its scales multiply the score (keys) and the
//     softmax weight (values), so the codes themselves, which 16-bit floats hold exactly, are the operands.
// Fragments: mma.m16n8k16 leaves the order of the k index free as long as both operands agree.  For q.k a thread takes 16 consecutive bytes of
// its key's row (8 or 16 elements = 2 or 4 k-steps) and the query fragments follow that order; for 8-bit values, where no transposing load
// fits, a thread takes head_dim / 8 consecutive columns of four keys' rows and n-tile i is column i of each thread's.
#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kBlocksPerSM = 2;
constexpr float kLow = -3.0e38f;            // below every score: 2^(x - kLow) is never formed, 2^(-inf - kLow) is 0

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

template <bool BF> __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on)     // 16 bytes, or zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool on)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}

template <int CACHE, int D> struct Shape {
    static constexpr int kElem = CACHE == WWWS_CACHE_16 ? 2 : 1;
    static constexpr int kRow = D * kElem;              // bytes of a cached row
    static constexpr int kChunks = kRow / 16;
    static constexpr int kTK = kRow == 256 ? 16 : 32;   // keys per tile: 4 KB of keys where rows allow it
    static constexpr int kTile = kTK * kRow;
    static constexpr int kScales = CACHE == WWWS_CACHE_16 ? 0 : kTK * 8;
    static constexpr int kStage = 2 * kTile + kScales;
    static constexpr int kStages = kRow == 64 ? 5 : 3;
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

template <bool BF, int CACHE, int D>
__global__ void __launch_bounds__(kThreads, kBlocksPerSM) k_attend_rows(AttendArgs a)
{
    using A = Act<BF>;
    using S = Shape<CACHE, D>;
    constexpr int TK = S::kTK, NT = TK / 8, KT = TK / 16;
    constexpr bool kQuant = CACHE != WWWS_CACHE_16;
    constexpr float kLift = kQuant && !BF ? 64.0f : 1.0f;    // keeps f16 weights times small value scales out of the subnormals (a scale of f16 values is at most 516, so the product stays finite)
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
            if (sequence(a.b, base + tid, q0, q_len, kv, a.err) && q_len && uint32_t(q_len) * G <= a.few_rows)
                x = (unsigned long long)((uint32_t(q_len) * G + kDecodeRows - 1) / kDecodeRows) * span_of<TK>(q_len, kv, a.window, a.sinks).tiles;
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
    const unsigned long long begin = blockIdx.x * share, end = min(total, begin + share);

    const uint32_t ring = uint32_t(__cvta_generic_to_shared(smem)) + warp * S::kRing;
    const uint8_t* ring_g = smem + warp * S::kRing;
    float* comb_o = reinterpret_cast<float*>(smem);                                   // [kWarps][16][D], over the drained rings
    float2* comb_ml = reinterpret_cast<float2*>(comb_o + kWarps * kDecodeRows * D);   // [kWarps][16]

    for (unsigned long long x = begin; x < end;) {
        // the segment: unit (sequence i, row tile r, kv head h), its tiles [t0, t1)
        const unsigned long long per_head = x / Hkv;
        uint32_t i = 0, hi_seq = a.b.n_seqs;
        while (hi_seq - i > 1) { const uint32_t mid = (i + hi_seq) >> 1; if (prefix[mid] <= per_head) i = mid; else hi_seq = mid; }
        const int q0 = a.b.q_start[i], q_len = a.b.q_start[i + 1] - q0, kv = a.b.kv_len[i];
        const Span sp = span_of<TK>(q_len, kv, a.window, a.sinks);
        const unsigned long long rel = x - prefix[i] * Hkv;
        const uint32_t unit = uint32_t(rel / uint32_t(sp.tiles));
        const int t0 = int(rel - (unsigned long long)unit * uint32_t(sp.tiles));
        const int t1 = int(min((unsigned long long)sp.tiles, t0 + (end - x)));
        const uint32_t h = unit % Hkv, row0 = unit / Hkv * kDecodeRows;
        const int n_rows = min(int(kDecodeRows), q_len * int(G) - int(row0));
        const int place0 = kv - q_len;                                   // place of the sequence's first new token
        const int first_place = place0 + int(row0 / G), last_place = place0 + int((row0 + n_rows - 1) / G);
        const int lo_key = a.window ? max(0, first_place - int(a.window) + 1) : 0, hi_key = min(kv, last_place + 1);

        // query fragments, in the order in which the keys' chunks are taken
        uint32_t qa[D / 16][4];
        {
            const int ra = n, rb = n + 8;
            auto at = [&](int r) { return reinterpret_cast<const uint4*>(a.q + (uint64_t(q0 + int((row0 + r) / G)) * a.q_stride + (uint64_t(h) * G + (row0 + r) % G) * D) * 2); };
            constexpr int kPer = kQuant ? 2 : 1;         // 8-element pieces of a thread's chunk
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const int piece = kQuant ? (4 * (s / 2) + c) * kPer + s % 2 : 4 * s + c;
                const uint4 z = make_uint4(0, 0, 0, 0);
                const uint4 u = ra < n_rows ? __ldg(at(ra) + piece) : z, w = rb < n_rows ? __ldg(at(rb) + piece) : z;
                qa[2 * s][0] = u.x; qa[2 * s][1] = w.x; qa[2 * s][2] = u.y; qa[2 * s][3] = w.y;
                qa[2 * s + 1][0] = u.z; qa[2 * s + 1][1] = w.z; qa[2 * s + 1][2] = u.w; qa[2 * s + 1][3] = w.w;
            }
        }
        const int pa = place0 + int((row0 + min(n, n_rows - 1)) / G), pb = place0 + int((row0 + min(n + 8, n_rows - 1)) / G);

        float o[D / 8][4];
#pragma unroll
        for (int d = 0; d < D / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.0f;
        float ma = kLow, mb = kLow, la = 0.0f, lb = 0.0f;

        const int32_t* table = a.b.page_table + uint64_t(i) * a.b.table_stride;
        const int page_mask = (1 << a.p.page_shift) - 1;
        auto key_of = [&](int t) { return (t < sp.n_sink ? t : sp.lo_tile + t - sp.n_sink) * TK; };
        auto pages_of = [&](int t, uint32_t (&pg)[KT]) {
#pragma unroll
            for (int g = 0; g < KT; ++g) {
                const int key = key_of(t) + 16 * g;
                pg[g] = t < t1 && key < hi_key ? uint32_t(__ldg(table + (key >> a.p.page_shift))) : 0u;
            }
        };
        // copies one tile of keys and values (zeros for keys that no row of the unit sees)
        auto issue = [&](int t, int stage, const uint32_t (&pg)[KT]) {
            if (t < t1) {
                const int key0 = key_of(t);
                const uint32_t dst = ring + stage * S::kStage;
#pragma unroll
                for (int g = 0; g < KT; ++g) {
                    const int kg = key0 + 16 * g;
                    bool ok = kg < hi_key;
                    if (ok && pg[g] >= a.p.n_pages) { report(a.err, bePage); ok = false; }
                    const int64_t cell = ok ? (((int64_t(pg[g]) * Hkv + h) << a.p.page_shift) + (kg & page_mask)) : 0;
                    constexpr int kPer = 16 * S::kChunks / 32;
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const int ci = lane + 32 * e, kk = ci / S::kChunks, ch = ci % S::kChunks, key = kg + kk;
                        const bool on = ok && key < hi_key && (key >= lo_key || key < int(a.sinks));
                        cp16(dst + S::k_at(16 * g + kk, ch), a.p.k + cell * S::kRow + (on ? ci * 16 : 0), on);
                        cp16(dst + S::kTile + S::v_at(16 * g + kk, ch), a.p.v + cell * S::kRow + (on ? ci * 16 : 0), on);
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

            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.0f;
#pragma unroll
            for (int u = 0; u < S::kChunks / 4; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 w = *reinterpret_cast<const uint4*>(kt + S::k_at(nt * 8 + n, 4 * u + c));
                    if constexpr (!kQuant) {
                        mma<BF>(s[nt], qa[2 * u], w.x, w.y);
                        mma<BF>(s[nt], qa[2 * u + 1], w.z, w.w);
                    } else {
                        const uint32_t ws[4] = { w.x, w.y, w.z, w.w };
#pragma unroll
                        for (int e = 0; e < 4; ++e) mma<BF>(s[nt], qa[4 * u + e], widen<BF, CACHE>(ws[e] & 0xffffu), widen<BF, CACHE>(ws[e] >> 16));
                    }
                }
            const float* scales = reinterpret_cast<const float*>(vt + S::kTile);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float f0 = a.scale_log2, f1 = f0;
                if constexpr (kQuant) { const float2 k2 = *reinterpret_cast<const float2*>(scales + nt * 8 + 2 * c); f0 = f0 * k2.x; f1 = f1 * k2.y; }
                s[nt][0] *= f0; s[nt][1] *= f1; s[nt][2] *= f0; s[nt][3] *= f1;
            }
            // hidden keys, where the tile has any
            const bool masked = key0 + TK - 1 > first_place || (a.window && key0 < last_place - int(a.window) + 1 && key0 + TK > int(a.sinks));
            if (masked) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + nt * 8 + 2 * c + (e & 1), p = e < 2 ? pa : pb;
                        if (key > p || (a.window && key <= p - int(a.window) && key >= int(a.sinks))) s[nt][e] = -INFINITY;
                    }
            }
            float xa = fmaxf(s[0][0], s[0][1]), xb = fmaxf(s[0][2], s[0][3]);
#pragma unroll
            for (int nt = 1; nt < NT; ++nt) { xa = fmaxf(xa, fmaxf(s[nt][0], s[nt][1])); xb = fmaxf(xb, fmaxf(s[nt][2], s[nt][3])); }
#pragma unroll
            for (int m = 1; m < 4; m <<= 1) { xa = fmaxf(xa, __shfl_xor_sync(0xffffffffu, xa, m)); xb = fmaxf(xb, __shfl_xor_sync(0xffffffffu, xb, m)); }
            if (__any_sync(0xffffffffu, xa > ma || xb > mb)) {       // the maximum moved: earlier sums shrink
                xa = fmaxf(xa, ma); xb = fmaxf(xb, mb);
                const float ca = ex2(ma - xa), cb = ex2(mb - xb);
                ma = xa; mb = xb; la *= ca; lb *= cb;
#pragma unroll
                for (int d = 0; d < D / 8; ++d) { o[d][0] *= ca; o[d][1] *= ca; o[d][2] *= cb; o[d][3] *= cb; }
            }
            uint32_t pf[KT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p0 = ex2(s[nt][0] - ma), p1 = ex2(s[nt][1] - ma), p2 = ex2(s[nt][2] - mb), p3 = ex2(s[nt][3] - mb);
                la += p0 + p1; lb += p2 + p3;
                if constexpr (kQuant) {
                    const float2 v2 = *reinterpret_cast<const float2*>(scales + TK + nt * 8 + 2 * c);
                    const float f0 = v2.x * kLift, f1 = v2.y * kLift;
                    p0 *= f0; p1 *= f1; p2 *= f0; p3 *= f1;
                    if (masked) {               // a hidden value's scale may be NaN
                        p0 = s[nt][0] == -INFINITY ? 0.0f : p0; p1 = s[nt][1] == -INFINITY ? 0.0f : p1;
                        p2 = s[nt][2] == -INFINITY ? 0.0f : p2; p3 = s[nt][3] == -INFINITY ? 0.0f : p3;
                    }
                }
                pf[nt / 2][(nt & 1) * 2] = A::pack(p0, p1);
                pf[nt / 2][(nt & 1) * 2 + 1] = A::pack(p2, p3);
            }
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                if constexpr (!kQuant) {
                    const int key = 16 * k + (lane & 15);
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        uint32_t r0, r1, r2, r3;
                        const uint32_t at = uint32_t(__cvta_generic_to_shared(vt)) + S::v_at(key, 2 * d + (lane >> 4));
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(at) : "memory");
                        mma<BF>(o[2 * d], pf[k], r0, r1);
                        mma<BF>(o[2 * d + 1], pf[k], r2, r3);
                    }
                } else {
                    constexpr int W = D / 32;        // words of a thread's columns of one key
                    uint32_t v[4][W];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = 16 * k + 2 * c + (e & 1) + (e >> 1) * 8;
                        if constexpr (W == 4) {
                            const uint4 w = *reinterpret_cast<const uint4*>(vt + S::v_at(key, n));
                            v[e][0] = w.x; v[e][1] = w.y; v[e][2] = w.z; v[e][3] = w.w;
                        } else {
                            const uint2 w = *reinterpret_cast<const uint2*>(vt + S::v_at(key, n >> 1) + (n & 1) * 8);
                            v[e][0] = w.x; v[e][1] = w.y;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        const uint32_t a0 = __byte_perm(v[0][w], v[1][w], 0x5140), a1 = __byte_perm(v[0][w], v[1][w], 0x7362);
                        const uint32_t b0 = __byte_perm(v[2][w], v[3][w], 0x5140), b1 = __byte_perm(v[2][w], v[3][w], 0x7362);
                        mma<BF>(o[4 * w + 0], pf[k], widen<BF, CACHE>(a0 & 0xffffu), widen<BF, CACHE>(b0 & 0xffffu));
                        mma<BF>(o[4 * w + 1], pf[k], widen<BF, CACHE>(a0 >> 16), widen<BF, CACHE>(b0 >> 16));
                        mma<BF>(o[4 * w + 2], pf[k], widen<BF, CACHE>(a1 & 0xffffu), widen<BF, CACHE>(b1 & 0xffffu));
                        mma<BF>(o[4 * w + 3], pf[k], widen<BF, CACHE>(a1 >> 16), widen<BF, CACHE>(b1 >> 16));
                    }
                }
            }
            __syncwarp();
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
        for (int m = 1; m < 4; m <<= 1) { la += __shfl_xor_sync(0xffffffffu, la, m); lb += __shfl_xor_sync(0xffffffffu, lb, m); }
        __syncthreads();                       // every warp is done with its ring
        {
            float* ow = comb_o + warp * kDecodeRows * D;
#pragma unroll
            for (int d = 0; d < D / 8; ++d) {
                // columns of n-tile d: 8 d + column (values as given), column * D / 8 + d (8-bit values)
                const int c0 = kQuant ? 2 * c * (D / 8) + d : 8 * d + 2 * c, c1 = kQuant ? c0 + D / 8 : c0 + 1;
                ow[n * D + c0] = o[d][0]; ow[n * D + c1] = o[d][1];
                ow[(n + 8) * D + c0] = o[d][2]; ow[(n + 8) * D + c1] = o[d][3];
            }
            if (c == 0) { comb_ml[warp * kDecodeRows + n] = make_float2(ma, la); comb_ml[warp * kDecodeRows + n + 8] = make_float2(mb, lb); }
        }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == sp.tiles;
        // a segment at the start of the block's share goes to the block's slot 0, another to slot 1
        const uint32_t slot = 2 * blockIdx.x + (x == begin ? 0 : 1);
        auto store = [&](int r, int d, float v0, float v1, float l) {
            const float f = l > 0.0f ? (1.0f / kLift) / l : l;       // l = 0: nothing seen; l = NaN stays NaN
            const uint32_t row = row0 + r;
            *reinterpret_cast<uint32_t*>(a.out + (uint64_t(q0 + int(row / G)) * a.out_stride + (uint64_t(h) * G + row % G) * D + d) * 2) = A::pack(v0 * f, v1 * f);
        };
        for (int e = tid; e < n_rows * (D / 2); e += kThreads) {
            const int r = e / (D / 2), d = e % (D / 2) * 2;
            float m = kLow, l = 0.0f, v0 = 0.0f, v1 = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, comb_ml[w * kDecodeRows + r].x);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 ml = comb_ml[w * kDecodeRows + r];
                const float f = ex2(ml.x - m);
                const float2 v = *reinterpret_cast<const float2*>(comb_o + (w * kDecodeRows + r) * D + d);
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
                    for (uint32_t k = blk0; k <= blk1; ++k) {
                        const uint32_t s = k == blk0 ? first_slot : 2 * k;
                        const float2 ml = __ldcg(a.s.part_ml + s * kDecodeRows + r);
                        const float2 v = __ldcg(reinterpret_cast<const float2*>(a.s.part_o + (uint64_t(s) * kDecodeRows + r) * D + d));
                        const float mn = fmaxf(m, ml.x), f0 = ex2(m - mn), f1 = ex2(ml.x - mn);
                        l = l * f0 + ml.y * f1; v0 = v0 * f0 + v.x * f1; v1 = v1 * f0 + v.y * f1;
                        m = mn;
                    }
                    store(r, d, v0, v1, l);
                }
                if (tid == 0) a.s.ticket[first_slot] = 0;
            }
        }
        __syncthreads();                       // the joined rows are read before the rings fill again
        x += t1 - t0;
    }
}

}  // namespace

cudaError_t launch_attend_rows(const AttendArgs& a, uint32_t head_dim, int dtype, int cache, cudaStream_t s)
{
    auto go = [&](auto bf, auto kind, auto dim) -> cudaError_t {
        constexpr bool BF = decltype(bf)::value;
        constexpr int CACHE = decltype(kind)::value, D = decltype(dim)::value;
        using S = Shape<CACHE, D>;
        static_assert(S::kSmem >= kWarps * int(kDecodeRows) * (D + 2) * 4, "the joined rows fit the rings");
        auto kernel = k_attend_rows<BF, CACHE, D>;
        const uint32_t smem = S::kSmem + (a.b.n_seqs + 1) * 8;
        if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem + 2049 * 8); e != cudaSuccess) return e;
        const uint64_t row_tiles = (uint64_t(a.b.max_q_len) * a.group + kDecodeRows - 1) / kDecodeRows;
        const uint64_t tiles = uint64_t(a.b.n_seqs) * row_tiles * a.p.n_kv_heads * ((a.b.max_kv_len + S::kTK - 1) / S::kTK + 1);
        const uint64_t blocks = (tiles + kWarps - 1) / kWarps;
        kernel<<<uint32_t(blocks < 148 * kBlocksPerSM ? blocks : 148 * kBlocksPerSM), kThreads, smem, s>>>(a);
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
