// Norms of queries and keys for each head and their rotation by position in one pass, with the write of keys and values to the paged cache.
//
//   n = x w / sqrt(mean(x^2) + eps),   (a, b) -> (a cos p f - b sin p f, b cos p f + a sin p f) for the pairs (a, b) of n, in fp32, rounded once
// (for a quantised cache not even once before the code is made).  Bound by HBM: every element is read once and written once, and nothing is read
// twice but the positions.
//   - Angles are kept as fractions of a turn in 64-bit whole numbers: position * turns wraps around exactly, so a position of 2^30 costs no
//     precision that one of 2 does not, without 64-bit floating point.  cos and sin are then of an argument in [-pi, pi), where the hardware's are within
//     2^-21 (absolute; a rounding to f16 is off by up to 2^-12 of a result of size 1, to bf16 by 2^-9), and take a tenth of the exact ones' instructions.
//   - A lane holds 16 elements of a head as two 16-byte pieces that contain both halves of its 8 pairs: elements 8 j and dim / 2 + 8 j on (head_dim / 2 + 8 j where
//     neighbours are paired).  So head_dim / 16 lanes share a head, a warp turns 4 or 8 heads at once, its 8 angles a lane
//     are worked out once a token and the norm is a shuffle over 3 or 2 steps.
//   - 6 x 4,097 tokens of 28 + 4 heads of 128 in f16, three axes: 76 us, 5,300 GB/s; 24 prompts of 900 tokens on average to int8 with norms: 112 us.
//   - A warp takes one token, or a part of its heads where there are too few tokens to fill the GPU: the angles are then worked out more than once.
#include "backend.cuh"
#include "tcgen.cuh"

namespace wwws {
namespace {

constexpr int kThreads = 128;
constexpr int kNone = -1;                // no cache: turned keys are given back

struct Pieces { uint4 a, b; };

template <bool BF, int CACHE, int D, bool kNeighbours>
__global__ void __launch_bounds__(kThreads, 5) k_rotate(RotateArgs g)
{
    using A = Act<BF>;
    using std::integral_constant;
    constexpr int L = D / 16, R = 32 / L;                // lanes of a head, heads of a warp at once
    constexpr bool kAppend = CACHE != kNone, kQuant = CACHE == WWWS_CACHE_INT8 || CACHE == WWWS_CACHE_E4M3;
    extern __shared__ int32_t start[];                   // [n_seqs + 1], append alone
    if constexpr (kAppend) {
        for (uint32_t i = threadIdx.x; i <= g.b.n_seqs; i += kThreads) start[i] = g.b.q_start[i];
        __syncthreads();
        if (blockIdx.x == 0 && threadIdx.x == 0 && (start[0] != 0 || uint32_t(start[g.b.n_seqs]) != g.n_tokens)) report(g.err, beOffset);
    }
    const uint32_t lane = threadIdx.x % 32, j = lane % L, sub = lane / L;
    const wwws_rotation& r = g.r;
    // This lane's pieces of a head: its pairs are (a[e], b[e]); or, for neighbours, lie within a piece, and the lanes' pieces side by side (16 neighbours a lane
    // wrote half sectors).
    const bool turned = j * 16 < r.dim;
    const uint32_t off_a = kNeighbours ? 8 * j : turned ? 8 * j : 16 * j, off_b = kNeighbours ? D / 2 + 8 * j : turned ? r.dim / 2 + 8 * j : 16 * j + 8;
    const bool turned_a = kNeighbours ? off_a < r.dim : turned, turned_b = kNeighbours ? off_b < r.dim : turned;
    const uint32_t groups_q = (g.n_heads + R - 1) / R, groups_k = (g.n_kv_heads + R - 1) / R;
    const uint32_t groups = groups_q + (kAppend ? 2 : 1) * groups_k;
    const uint32_t tasks = g.n_tokens * g.parts, warps = gridDim.x * (kThreads / 32);
    for (uint32_t task = (blockIdx.x * kThreads + threadIdx.x) / 32; task < tasks; task += warps) {
        uint32_t tok = task, g0 = 0, g1 = groups;        // a token, or a part of its heads
        if (g.parts > 1) {
            tok = task / g.parts;
            const uint32_t part = task - tok * g.parts;
            g0 = groups * part / g.parts; g1 = groups * (part + 1) / g.parts;
        }
        if (g.parts == 1) {                              // all of the token is on its way while its angles are worked out (6 x 4,097 tokens 88 -> 76 us, 24 prompts to int8 125 -> 112)
            auto lines = [&](const uint8_t* in, uint32_t heads) { for (uint32_t e = lane * 128; e < heads * D * 2; e += 32 * 128) asm volatile("prefetch.global.L1 [%0];" :: "l"(in + e)); };
            lines(g.q + uint64_t(tok) * g.q_stride * 2, g.n_heads); lines(g.k + uint64_t(tok) * g.k_stride * 2, g.n_kv_heads);
            if (kAppend) lines(g.v + uint64_t(tok) * g.v_stride * 2, g.n_kv_heads);
        }
        int64_t cell = -1;                               // of kv head 0
        int place = 0;
        if constexpr (kAppend) {
            uint32_t i = 0, hi = g.b.n_seqs;
            while (hi - i > 1) { const uint32_t mid = (i + hi) >> 1; if (start[mid] <= int(tok)) i = mid; else hi = mid; }
            const int q_len = start[i + 1] - start[i], kv = __ldg(g.b.kv_len + i);
            if (uint32_t(q_len) > g.b.max_q_len || uint32_t(kv) > g.b.max_kv_len || start[i] < 0 || start[i] > int(tok) || start[i + 1] <= int(tok) || uint32_t(start[i + 1]) > g.n_tokens) { report(g.err, beOffset); continue; }
            place = kv - q_len + int(tok) - start[i];
            if (place >= 0) {
                const uint32_t page = uint32_t(__ldg(g.b.page_table + uint64_t(i) * g.b.table_stride + (uint32_t(place) >> g.p.page_shift)));
                if (page >= g.p.n_pages) report(g.err, bePage);
                else cell = (int64_t(page) * g.p.n_kv_heads << g.p.page_shift) + (place & ((1 << g.p.page_shift) - 1));
            }
        }
        // halves: cos, sin and -sin of two pairs side by side; neighbours: of a pair
        uint64_t cs[4], sn[4], minus[4];
        float c1[8], s1[8];
        if (turned_a && g0 < groups_q + groups_k) {
            const int32_t* from = g.positions ? g.positions + uint64_t(tok) * r.n_axes : nullptr;
            const unsigned long long* turns = reinterpret_cast<const unsigned long long*>(r.turns);
            int pos = from ? __ldg(from) : place;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t pair = !kNeighbours ? 8 * j + e : e < 4 ? off_a / 2 + e : off_b / 2 + e - 4;
                if (kNeighbours && e >= 4 && !turned_b) break;
                if (r.axis && from) {                    // (with places for positions every axis has the same)
                    uint32_t axis = __ldg(r.axis + pair);
                    if (axis >= r.n_axes) { report(g.err, beOffset); axis = 0; }
                    pos = __ldg(from + axis);
                }
                const uint64_t phase = uint64_t(int64_t(pos)) * __ldg(turns + pair);
                const float x = float(int32_t(phase >> 32)) * (0x1p-31f * 3.14159274f);
                c1[e] = __cosf(x); s1[e] = __sinf(x);
            }
            if constexpr (!kNeighbours)
#pragma unroll
                for (int e = 0; e < 4; ++e) { cs[e] = pack2(c1[2 * e], c1[2 * e + 1]); sn[e] = pack2(s1[2 * e], s1[2 * e + 1]); minus[e] = pack2(-s1[2 * e], -s1[2 * e + 1]); }
        }
        // The heads [R (from - first), R (to - first)) of queries (0), keys (1) or values (2), two groups' loads in flight.
        auto pass = [&](auto which, const uint8_t* in, uint8_t* out, float* scales, uint32_t heads, uint32_t first, uint32_t last, const float* weight) {
            constexpr int kKind = decltype(which)::value;
            constexpr bool kCodes = kQuant && kKind > 0, kCell = kAppend && kKind > 0;
            const uint32_t from = g0 > first ? g0 : first, to = g1 < last ? g1 : last;
            if (from >= to) return;
            uint64_t wa[4], wb[4];                       // this lane's weights
            if (kKind < 2 && weight) {
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const ulonglong2 y = __ldg(reinterpret_cast<const ulonglong2*>(weight + off_a) + e / 2), z = __ldg(reinterpret_cast<const ulonglong2*>(weight + off_b) + e / 2);
                    wa[e] = y.x; wa[e + 1] = y.y; wb[e] = z.x; wb[e + 1] = z.y;
                }
            }
            auto work = [&](const Pieces& x, uint32_t h, bool on) {
                // two elements at a time
                uint64_t a[4], b[4];
                const uint32_t w0[4] = { x.a.x, x.a.y, x.a.z, x.a.w }, w1[4] = { x.b.x, x.b.y, x.b.z, x.b.w };
                if (kKind < 2 || kCodes) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) { a[e] = pack2(A::lo(w0[e]), A::hi(w0[e])); b[e] = pack2(A::lo(w1[e]), A::hi(w1[e])); }
                }
                if (kKind < 2 && weight) {               // (the same for the whole warp)
                    uint64_t sq = mul2(a[0], a[0]);
#pragma unroll
                    for (int e = 1; e < 4; ++e) sq = fma2(a[e], a[e], sq);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sq = fma2(b[e], b[e], sq);
                    float s0, ss;
                    unpack2(sq, s0, ss);
                    ss += s0;
#pragma unroll
                    for (int m = 1; m < L; m <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                    const float inv = rsqrtf(__fmaf_rn(ss, 1.0f / D, r.eps));
                    const uint64_t by = pack2(inv, inv);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { a[e] = mul2(mul2(a[e], by), wa[e]); b[e] = mul2(mul2(b[e], by), wb[e]); }
                }
                if (kKind < 2 && turned_a) {
                    if constexpr (kNeighbours) {
                        auto turn = [&](uint64_t& p, int e) {
                            float y0, y1;
                            unpack2(p, y0, y1);
                            p = pack2(__fmaf_rn(y0, c1[e], -(y1 * s1[e])), __fmaf_rn(y1, c1[e], y0 * s1[e]));
                        };
#pragma unroll
                        for (int e = 0; e < 4; ++e) turn(a[e], e);
                        if (turned_b) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) turn(b[e], 4 + e);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint64_t y = fma2(a[e], cs[e], mul2(b[e], minus[e]));
                            b[e] = fma2(b[e], cs[e], mul2(a[e], sn[e])); a[e] = y;
                        }
                    }
                }
                const bool put = on && (!kCell || cell >= 0);
                const int64_t row = kCell ? cell + (int64_t(h) << g.p.page_shift) : int64_t(h);
                if constexpr (!kCodes) {
                    uint8_t* to = out + row * (D * 2);
                    auto packed = [](uint64_t v) { float y0, y1; unpack2(v, y0, y1); return A::pack(y0, y1); };
                    const uint4 ya = kKind == 2 ? x.a : make_uint4(packed(a[0]), packed(a[1]), packed(a[2]), packed(a[3]));        // values go as they are
                    const uint4 yb = kKind == 2 ? x.b : make_uint4(packed(b[0]), packed(b[1]), packed(b[2]), packed(b[3]));
                    if (put) { *reinterpret_cast<uint4*>(to + off_a * 2) = ya; *reinterpret_cast<uint4*>(to + off_b * 2) = yb; }
                } else {
                    // the largest magnitude as bits: NaN > infinity > every finite value
                    uint32_t top = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        top = max(top, max(uint32_t(a[e]) & 0x7fffffffu, uint32_t(a[e] >> 32) & 0x7fffffffu));
                        top = max(top, max(uint32_t(b[e]) & 0x7fffffffu, uint32_t(b[e] >> 32) & 0x7fffffffu));
                    }
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
                        float y0, y1, y2, y3;
                        unpack2(mul2((w < 2 ? a : b)[w % 2 * 2], pack2(inv, inv)), y0, y1);
                        unpack2(mul2((w < 2 ? a : b)[w % 2 * 2 + 1], pack2(inv, inv)), y2, y3);
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
                    if (put) {
                        uint8_t* to = out + row * D;
                        *reinterpret_cast<uint2*>(to + off_a) = make_uint2(code[0], code[1]);
                        *reinterpret_cast<uint2*>(to + off_b) = make_uint2(code[2], code[3]);
                        if (j == 0) scales[row] = scale;
                    }
                }
            };
            auto fetch = [&](uint32_t h) {
                Pieces x{ make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0) };
                if (h < heads) { x.a = *reinterpret_cast<const uint4*>(in + h * (D * 2) + off_a * 2); x.b = *reinterpret_cast<const uint4*>(in + h * (D * 2) + off_b * 2); }
                return x;
            };
            const uint32_t end = (to - first) * R;
            for (uint32_t h = (from - first) * R + sub; h - sub < end; h += 2 * R) {
                const bool more = h - sub + R < end;
                const Pieces x0 = fetch(h), x1 = fetch(more ? h + R : heads);
                work(x0, h, h < heads);
                if (more) work(x1, h + R, h + R < heads);
            }
        };
        pass(integral_constant<int, 0>(), g.q + uint64_t(tok) * g.q_stride * 2, g.q_out + uint64_t(tok) * g.q_out_stride * 2, nullptr, g.n_heads, 0, groups_q, r.q_weight);
        if constexpr (kAppend) {
            pass(integral_constant<int, 1>(), g.k + uint64_t(tok) * g.k_stride * 2, g.p.k, g.p.k_scale, g.n_kv_heads, groups_q, groups_q + groups_k, r.k_weight);
            pass(integral_constant<int, 2>(), g.v + uint64_t(tok) * g.v_stride * 2, g.p.v, g.p.v_scale, g.n_kv_heads, groups_q + groups_k, groups, nullptr);
        } else
            pass(integral_constant<int, 1>(), g.k + uint64_t(tok) * g.k_stride * 2, g.k_out + uint64_t(tok) * g.k_out_stride * 2, nullptr, g.n_kv_heads, groups_q, groups_q + groups_k, r.k_weight);
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
