// Norms of queries and keys for each head and their rotation by position in one pass, with the write of keys and values to the paged cache.
//
//   n = x w / sqrt(mean(x^2) + eps),   (a, b) -> (a cos p f - b sin p f, b cos p f + a sin p f) for the pairs (a, b) of n, in fp32, rounded once
// (for a quantised cache not even once before the code is made).  Bound by HBM: every element is read once and written once, and nothing is read
// twice but the positions.
//   - Angles are kept as fractions of a turn in 64-bit whole numbers: position * turns wraps around exactly, so a position of 2^30 costs no
//     precision that one of 2 does not, without 64-bit floating point; cos and sin are then of an argument in [-1, 1) half turns.
//   - A lane holds 16 elements of a head as two 16-byte pieces that contain both halves of its 8 pairs: elements 8 j and dim / 2 + 8 j on where the halves
//     of a head are paired, 16 neighbours where neighbours are.  So head_dim / 16 lanes share a head, a warp turns 4 or 8 heads at once, its 8 angles a lane
//     are worked out once a token and the norm is a shuffle over 3 or 2 steps.
//   - A warp takes one token, or a part of its heads where there are too few tokens to fill the GPU: the angles are then worked out more than once.
#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 128;
constexpr int kNone = -1;                // no cache: turned keys are given back

struct Pieces { uint4 a, b; };

template <bool BF, int CACHE, int D, bool kNeighbours>
__global__ void __launch_bounds__(kThreads) k_rotate(RotateArgs g)
{
    using A = Act<BF>;
    constexpr int L = D / 16, R = 32 / L;                // lanes of a head, heads of a warp at once
    constexpr bool kAppend = CACHE != kNone, kQuant = CACHE == WWWS_CACHE_INT8 || CACHE == WWWS_CACHE_E4M3;
    extern __shared__ int32_t start[];                   // [n_seqs + 1], append alone
    if constexpr (kAppend) {
        for (uint32_t i = threadIdx.x; i <= g.b.n_seqs; i += kThreads) start[i] = g.b.q_start[i];
        __syncthreads();
    }
    const uint32_t lane = threadIdx.x % 32, j = lane % L, sub = lane / L;
    const wwws_rotation& r = g.r;
    // this lane's pieces of a head, and its pairs: (a[e], b[e]) or, for neighbours, of each piece
    const bool turned = j * 16 < r.dim;
    const uint32_t off_a = turned && !kNeighbours ? 8 * j : 16 * j, off_b = turned && !kNeighbours ? r.dim / 2 + 8 * j : 16 * j + 8;
    const uint32_t groups_q = (g.n_heads + R - 1) / R, groups_k = (g.n_kv_heads + R - 1) / R;
    const uint32_t groups = groups_q + (kAppend ? 2 : 1) * groups_k;
    const uint64_t tasks = uint64_t(g.n_tokens) * g.parts;
    const uint64_t warps = uint64_t(gridDim.x) * (kThreads / 32);
    for (uint64_t task = (uint64_t(blockIdx.x) * kThreads + threadIdx.x) / 32; task < tasks; task += warps) {
        const uint32_t tok = uint32_t(task / g.parts), part = uint32_t(task - uint64_t(tok) * g.parts);
        const uint32_t g0 = uint32_t(uint64_t(groups) * part / g.parts), g1 = uint32_t(uint64_t(groups) * (part + 1) / g.parts);
        int64_t cell = -1;                               // of kv head 0
        int place = 0;
        if constexpr (kAppend) {
            uint32_t i = 0, hi = g.b.n_seqs;
            while (hi - i > 1) { const uint32_t mid = (i + hi) >> 1; if (start[mid] <= int(tok)) i = mid; else hi = mid; }
            const int q_len = start[i + 1] - start[i], kv = __ldg(g.b.kv_len + i);
            if (uint32_t(q_len) > g.b.max_q_len || uint32_t(kv) > g.b.max_kv_len || start[i] < 0 || start[i] > int(tok) || start[i + 1] <= int(tok)) { report(g.err, beOffset); continue; }
            place = kv - q_len + int(tok) - start[i];
            if (place >= 0) {
                const uint32_t page = uint32_t(__ldg(g.b.page_table + uint64_t(i) * g.b.table_stride + (uint32_t(place) >> g.p.page_shift)));
                if (page >= g.p.n_pages) report(g.err, bePage);
                else cell = (int64_t(page) * g.p.n_kv_heads << g.p.page_shift) + (place & ((1 << g.p.page_shift) - 1));
            }
        }
        float cs[8], sn[8];
        if (turned && g0 < groups_q + groups_k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t pair = 8 * j + e;
                uint32_t axis = r.axis ? __ldg(r.axis + pair) : 0;
                if (axis >= r.n_axes) { report(g.err, beOffset); axis = 0; }
                const int pos = g.positions ? __ldg(g.positions + uint64_t(tok) * r.n_axes + axis) : place;
                const uint64_t phase = uint64_t(int64_t(pos)) * __ldg(reinterpret_cast<const unsigned long long*>(r.turns) + pair);
                sincospif(float(int32_t(phase >> 32)) * 0x1p-31f, &sn[e], &cs[e]);
            }
        }
        const uint8_t* q = g.q + uint64_t(tok) * g.q_stride * 2; uint8_t* qo = g.q_out + uint64_t(tok) * g.q_out_stride * 2;
        const uint8_t* k = g.k + uint64_t(tok) * g.k_stride * 2; uint8_t* ko = kAppend ? nullptr : g.k_out + uint64_t(tok) * g.k_out_stride * 2;
        const uint8_t* v = kAppend ? g.v + uint64_t(tok) * g.v_stride * 2 : nullptr;
        for (uint32_t at = g0; at < g1; ++at) {
            const int kind = at < groups_q ? 0 : at < groups_q + groups_k ? 1 : 2;                  // queries, keys, values
            const uint32_t h = (kind == 0 ? at : kind == 1 ? at - groups_q : at - groups_q - groups_k) * R + sub;
            const bool on = h < (kind == 0 ? g.n_heads : g.n_kv_heads);
            Pieces x{ make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0) };
            if (on) {
                const uint8_t* from = (kind == 0 ? q : kind == 1 ? k : v) + h * (D * 2);
                x.a = *reinterpret_cast<const uint4*>(from + off_a * 2); x.b = *reinterpret_cast<const uint4*>(from + off_b * 2);
            }
            float a[8], b[8];
            {
                const uint32_t wa[4] = { x.a.x, x.a.y, x.a.z, x.a.w }, wb[4] = { x.b.x, x.b.y, x.b.z, x.b.w };
#pragma unroll
                for (int e = 0; e < 4; ++e) { a[2 * e] = A::lo(wa[e]); a[2 * e + 1] = A::hi(wa[e]); b[2 * e] = A::lo(wb[e]); b[2 * e + 1] = A::hi(wb[e]); }
            }
            if (const float* w = kind == 0 ? r.q_weight : kind == 1 ? r.k_weight : nullptr) {       // (the same for the whole warp)
                float ss = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = __fmaf_rn(a[e], a[e], __fmaf_rn(b[e], b[e], ss));
#pragma unroll
                for (int m = 1; m < L; m <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                const float inv = rsqrtf(__fmaf_rn(ss, 1.0f / D, r.eps));
                const float4* wa = reinterpret_cast<const float4*>(w + off_a);
                const float4* wb = reinterpret_cast<const float4*>(w + off_b);
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const float4 y = __ldg(wa + e / 4), z = __ldg(wb + e / 4);
                    a[e] *= inv * y.x; a[e + 1] *= inv * y.y; a[e + 2] *= inv * y.z; a[e + 3] *= inv * y.w;
                    b[e] *= inv * z.x; b[e + 1] *= inv * z.y; b[e + 2] *= inv * z.z; b[e + 3] *= inv * z.w;
                }
            }
            if (kind < 2 && turned) {
                auto turn = [&](float& p, float& q2, int e) {
                    const float y = __fmaf_rn(p, cs[e], -(q2 * sn[e]));
                    q2 = __fmaf_rn(q2, cs[e], p * sn[e]); p = y;
                };
                if constexpr (kNeighbours) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) { turn(a[2 * e], a[2 * e + 1], e); turn(b[2 * e], b[2 * e + 1], 4 + e); }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) turn(a[e], b[e], e);
                }
            }
            if (!kQuant || kind == 0) {
                uint8_t* to;
                bool put = on;
                if (kind == 0) to = qo + h * (D * 2);
                else if constexpr (!kAppend) to = ko + h * (D * 2);
                else { to = (kind == 1 ? g.p.k : g.p.v) + (cell + (int64_t(h) << g.p.page_shift)) * (D * 2); put = on && cell >= 0; }
                if (put && kind == 2) {                  // values go as they are
                    *reinterpret_cast<uint4*>(to + off_a * 2) = x.a; *reinterpret_cast<uint4*>(to + off_b * 2) = x.b;
                } else if (put) {
                    *reinterpret_cast<uint4*>(to + off_a * 2) = make_uint4(A::pack(a[0], a[1]), A::pack(a[2], a[3]), A::pack(a[4], a[5]), A::pack(a[6], a[7]));
                    *reinterpret_cast<uint4*>(to + off_b * 2) = make_uint4(A::pack(b[0], b[1]), A::pack(b[2], b[3]), A::pack(b[4], b[5]), A::pack(b[6], b[7]));
                }
            } else {
                // the largest magnitude as bits: NaN > infinity > every finite value
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, max(__float_as_uint(a[e]) & 0x7fffffffu, __float_as_uint(b[e]) & 0x7fffffffu));
#pragma unroll
                for (int m = 1; m < L; m <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
                constexpr float kTop = CACHE == WWWS_CACHE_INT8 ? 127.0f : 448.0f;
                const float amax = __uint_as_float(top);
                const bool finite = top < 0x7f800000u;
                const float scale = !finite ? __uint_as_float(0x7fffffffu) : amax < 0x1p-100f ? 0.0f : amax * (1.0f / kTop);
                const float inv = finite && scale > 0.0f ? __fdiv_rn(1.0f, scale) : 0.0f;
                uint32_t code[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float* x4 = (w < 2 ? a : b) + w % 2 * 4;
                    const float y0 = x4[0] * inv, y1 = x4[1] * inv, y2 = x4[2] * inv, y3 = x4[3] * inv;
                    if constexpr (CACHE == WWWS_CACHE_INT8) {
                        constexpr float kShift = 12582912.0f;       // 1.5 * 2^23 + y has round-to-even(y) in its low byte
                        const uint32_t lo = __byte_perm(__float_as_uint(y0 + kShift), __float_as_uint(y1 + kShift), 0x0040), hi = __byte_perm(__float_as_uint(y2 + kShift), __float_as_uint(y3 + kShift), 0x0040);
                        code[w] = __byte_perm(lo, hi, 0x5410);
                    } else {
                        uint16_t lo, hi;
                        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y1), "f"(y0));
                        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y3), "f"(y2));
                        code[w] = uint32_t(lo) | uint32_t(hi) << 16;
                    }
                    if (!finite) code[w] = 0;
                }
                if (on && cell >= 0) {
                    const int64_t c = cell + (int64_t(h) << g.p.page_shift);
                    uint8_t* to = (kind == 1 ? g.p.k : g.p.v) + c * D;
                    *reinterpret_cast<uint2*>(to + off_a) = make_uint2(code[0], code[1]);
                    *reinterpret_cast<uint2*>(to + off_b) = make_uint2(code[2], code[3]);
                    if (j == 0) (kind == 1 ? g.p.k_scale : g.p.v_scale)[c] = scale;
                }
            }
        }
    }
}

}  // namespace

cudaError_t launch_rotate(RotateArgs a, bool append, uint32_t head_dim, int dtype, int cache, cudaStream_t s)
{
    const uint32_t at_once = 32 * 16 / head_dim;
    const uint32_t groups = (a.n_heads + at_once - 1) / at_once + (append ? 2 : 1) * ((a.n_kv_heads + at_once - 1) / at_once);
    // A warp per token, unless that leaves the GPU with fewer than 16 warps an SM: then its heads are shared out.
    a.parts = 1;
    while (a.parts < groups && uint64_t(a.n_tokens) * a.parts < 148 * 16) ++a.parts;
    const uint64_t blocks = (uint64_t(a.n_tokens) * a.parts * 32 + kThreads - 1) / kThreads;
    const uint32_t grid = uint32_t(blocks < 148 * 64 ? blocks : 148 * 64), smem = append ? (a.b.n_seqs + 1) * 4 : 0;
    auto go = [&](auto bf, auto kind, auto dim) {
        constexpr int D = decltype(dim)::value, CACHE = decltype(kind)::value;
        if (a.r.interleaved) k_rotate<decltype(bf)::value, CACHE, D, true><<<grid, kThreads, smem, s>>>(a);
        else k_rotate<decltype(bf)::value, CACHE, D, false><<<grid, kThreads, smem, s>>>(a);
        return cudaGetLastError();
    };
    using std::integral_constant;
    auto dim = [&](auto bf, auto kind) { return head_dim == 64 ? go(bf, kind, integral_constant<int, 64>()) : go(bf, kind, integral_constant<int, 128>()); };
    auto kind = [&](auto bf) {
        return !append ? dim(bf, integral_constant<int, kNone>()) : cache == WWWS_CACHE_16 ? dim(bf, integral_constant<int, WWWS_CACHE_16>())
             : cache == WWWS_CACHE_INT8 ? dim(bf, integral_constant<int, WWWS_CACHE_INT8>()) : dim(bf, integral_constant<int, WWWS_CACHE_E4M3>());
    };
    return dtype == WWWS_BF16 ? kind(std::true_type()) : kind(std::false_type());
}

}  // namespace wwws
