// Types and launchers of the backend operators (internal to the library).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/wwws_backend.h"

namespace wwws {

// Kinds of device-side problems, kept as a bit mask in the workspace's error word.
enum BackendError : uint32_t { bePage = 1, beToken = 2, beMask = 4, beOffset = 8, beTimeout = 16, bePool = 32 };

struct SeqBatch {
    const int32_t* q_start; const int32_t* kv_len; const int32_t* page_table;
    uint32_t n_seqs, n_tokens, max_q_len, max_kv_len, table_stride;
    uint32_t ends;       // bit 0: the call's first sequence is among these, bit 1: its last
};

struct Pages {
    uint8_t* k; uint8_t* v; float* k_scale; float* v_scale;
    uint32_t n_pages, n_kv_heads, page_shift;
};

// Partial attention results (running maximum, sum and weighted values of a row) of the blocks that share a unit; all of the
// kernels use the same memory, one call after the other.
struct AttendScratch {
    float* part_o;       // [slots][rows][head_dim]
    float2* part_ml;     // [slots][rows]
    uint32_t* ticket;    // [kTickets], zero between calls
};

struct AttendArgs {
    SeqBatch b; Pages p; AttendScratch s;
    const uint8_t* q; uint8_t* out; uint64_t q_stride, out_stride;   // strides in elements
    uint32_t group;      // query heads per kv head
    float scale_log2;    // softmax scale * log2(e)
    uint32_t window, sinks;
    uint32_t pad;        // row kernel: 0, or the tiles that every unit counts (see kernels_attend.cu)
    uint32_t* err;
    const uint32_t* tree; uint32_t tree_words;      // bits of the new tokens that each new token sees (see wwws_attend_tree); not read by the kernels without trees
};

struct RotateArgs {
    wwws_rotation r;
    SeqBatch b; Pages p;                             // with the write to the cache alone
    const int32_t* positions;                        // NULL: the tokens' places
    const uint8_t* q; const uint8_t* k; const uint8_t* v; uint8_t* q_out; uint8_t* k_out;
    uint64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;      // in elements
    uint32_t n_tokens, n_heads, n_kv_heads;
    uint32_t parts;                                  // warps of a token
    uint32_t* err;
};

struct ForkArgs {
    const int32_t* refs; int32_t* refs_out;
    const int32_t* table; const int32_t* held; const int32_t* source; const int32_t* keep; const int32_t* room;
    int32_t* table_out; int32_t* held_out; int32_t* moves;
    uint32_t n_old, n_new, n_pages, max_pages, page_shift;
    uint32_t* owner; uint32_t* need;                 // workspace: [n_pages], [max_seqs]
    uint32_t* err;
};

constexpr uint32_t kMaxLayers = 64;                  // layers of a launch: their records are parameters of the kernel
struct Layer { uint8_t* k; uint8_t* v; float* k_scale; float* v_scale; };
struct LayerArgs {
    Layer layer[kMaxLayers];
    uint32_t n_pages, n_kv_heads, page_shift, row_bytes;
    uint32_t* err;
};

constexpr uint32_t kMaxBeams = 256, kMaxKeep = 128;
struct BeamArgs {
    const uint8_t* in; uint64_t stride;
    const float* total;
    float2* stat; float4* top; unsigned long long* heads;      // scratch, per row: [slices] maximum and sum, [chunks] maxima of four pieces, [chunks] best keys
    uint32_t* ticket;                                // [requests], zero between calls
    float* score; int32_t* parent; int32_t* token;
    uint32_t beams, vocab, keep, slices, chunks, per_slice;    // chunks of a row and of a slice
};

struct ShapeArgs {
    wwws_shaping s;
    const uint8_t* in; uint8_t* out; uint64_t in_stride, out_stride;
    uint32_t n_rows, vocab;
    int32_t* token; unsigned long long* best; uint32_t* ticket;     // best, ticket: [n_rows], zero between calls
    uint32_t* err;
};

constexpr uint32_t kDecodeSlots = 2 * 148 * 3;      // partial results of the row kernel: two per block of its largest grid
constexpr uint32_t kDecodeRows = 16;                 // most rows of its units
constexpr uint32_t kFewRows = 32, kFewRowsQuant = 48;     // most rows per kv head (new tokens * group) of the sequences of a call that goes to it (see wwws_attend)
constexpr uint32_t kTileBlocks = 148, kTileSlots = 2 * kTileBlocks;   // blocks of the tile kernel: one per SM

constexpr uint32_t kTileSeqs = 32;                    // sequences of a launch of the tile kernel, at most (see wwws_attend)
constexpr uint32_t kTreeSeqs = 256;                   // sequences of a launch of the tree kernel, at most: their running sum has to fit beside the rings
constexpr uint32_t kTickets = kDecodeSlots > kTileSlots ? kDecodeSlots : kTileSlots;

// Raises a kernel's limit of dynamic shared memory, the first time on each device.
template <auto kKernel> cudaError_t allow_smem(int bytes)
{
    static std::atomic<uint64_t> done{ 0 };          // a bit per device
    int device = 0;
    if (cudaError_t e = cudaGetDevice(&device); e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    if (cudaError_t e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_relaxed);
    return cudaSuccess;
}

cudaError_t launch_cache_append(const SeqBatch& b, const Pages& p, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride,
                                uint32_t head_dim, int dtype, int cache, uint32_t* err, cudaStream_t s);
cudaError_t launch_cache_read(const SeqBatch& b, const Pages& p, const int32_t* row_start, uint64_t n_rows, void* k_out, void* v_out,
                              uint32_t head_dim, int dtype, int cache, uint32_t* err, cudaStream_t s);
cudaError_t launch_attend_rows(const AttendArgs& a, uint32_t rows, uint32_t head_dim, int dtype, int cache, cudaStream_t s);
cudaError_t launch_attend_tile(const AttendArgs& a, uint32_t head_dim, int dtype, int cache, cudaStream_t s);
cudaError_t launch_attend_rows_tree(const AttendArgs& a, uint32_t rows, uint32_t head_dim, int dtype, int cache, cudaStream_t s);
cudaError_t launch_tree(const AttendArgs& a, uint32_t head_dim, int dtype, int cache, cudaStream_t s);
cudaError_t launch_shape_logits(const ShapeArgs& a, int dtype, cudaStream_t s);
cudaError_t launch_rotate(RotateArgs a, bool append, uint32_t head_dim, int dtype, int cache, cudaStream_t s);
cudaError_t launch_fork(const ForkArgs& a, cudaStream_t s);
cudaError_t launch_copy_pages(const LayerArgs& a, uint32_t n_layers, const int32_t* moves, uint32_t n_moves, cudaStream_t s);
cudaError_t launch_compact(const LayerArgs& a, uint32_t n_layers, const SeqBatch& b, const int32_t* path, const int32_t* path_len, uint32_t path_stride, cudaStream_t s);
uint64_t beams_scratch(uint32_t rows, uint32_t vocab, int dtype);
cudaError_t launch_beams(BeamArgs a, uint32_t rows, int dtype, void* scratch, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ void report(uint32_t* err, uint32_t bit) { atomicOr(err, bit); }

// The place of sequence i of the batch's new tokens; false (and reported) when its offsets or lengths break the batch's bounds, and
// the sequence is then skipped.
__device__ __forceinline__ bool sequence(const SeqBatch& b, uint32_t i, int& q0, int& q_len, int& kv, uint32_t* err)
{
    q0 = b.q_start[i]; q_len = b.q_start[i + 1] - q0; kv = b.kv_len[i];
    const bool ok = q0 >= 0 && q_len >= 0 && uint32_t(q_len) <= b.max_q_len && uint32_t(q0) + uint32_t(q_len) <= b.n_tokens &&
                    kv >= 0 && uint32_t(kv) <= b.max_kv_len;
    // tokens before the first sequence or behind the last are nobody's: reported, since no block will come by them
    if (!ok || (b.ends & 1 && i == 0 && q0 != 0) || (b.ends & 2 && i + 1 == b.n_seqs && uint32_t(q0) + uint32_t(q_len) != b.n_tokens)) report(err, beOffset);
    return ok;
}

// The new tokens rel .. rel + 31 (places behind the context) that the token of row `row` sees, a bit each; what lies before them is context: ones.
__device__ __forceinline__ uint32_t tree_bits(const uint32_t* tree, uint32_t words, int row, int rel)
{
    const uint32_t* w = tree + uint64_t(uint32_t(row)) * words;
    auto word = [&](int i) { return i < 0 ? ~0u : uint32_t(i) < words ? __ldg(w + i) : 0u; };
    return __funnelshift_r(word(rel >> 5), word((rel >> 5) + 1), uint32_t(rel) & 31u);
}
// How far behind the context a new token stands: the new tokens that it sees, itself not counted.
__device__ __forceinline__ int tree_depth(const uint32_t* tree, uint32_t words, int row, int tok)
{
    int n = 0;
    for (int i = 0; i * 32 <= tok; ++i) {
        const uint32_t x = tree_bits(tree, words, row, i * 32);
        n += __popc(tok - i * 32 >= 31 ? x : x & ((2u << (tok - i * 32)) - 1));
    }
    return max(n - 1, 0);
}

// A weight of 0 does not silence a value that is infinite or not a number, so the attention kernels look for these among the 16-bit values that some rows of a
// unit see and others do not, take them out of the product, and add them to the sums of the rows that see them.
__device__ __forceinline__ void largest_halves(uint32_t& top, uint4 x)       // the larger magnitudes of both halves, as bits: an exponent of ones is above every number
{
#pragma unroll
    for (int e = 0; e < 4; ++e) asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"((e == 0 ? x.x : e == 1 ? x.y : e == 2 ? x.z : x.w) & 0x7fff7fffu));
}
template <bool BF> __device__ __forceinline__ bool unreal(uint32_t half) { return (half & 0x7fffu) >= (BF ? 0x7f80u : 0x7c00u); }
template <bool BF> __device__ __forceinline__ bool unreal2(uint32_t both) { return unreal<BF>(both) || unreal<BF>(both >> 16); }
template <bool BF> __device__ __forceinline__ uint32_t real2(uint32_t both)  // zeros in their place
{
    return (unreal<BF>(both) ? 0u : both & 0xffffu) | (unreal<BF>(both >> 16) ? 0u : both & 0xffff0000u);
}

// Two-element vectors of the activation type, and the float conversions the kernels need.
template <bool BF> struct Act;
template <> struct Act<true> {
    static __device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b)   // a in the low half, both rounded to nearest even
    {
        uint32_t r; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a)); return r;
    }
};
template <> struct Act<false> {
    static __device__ __forceinline__ float lo(uint32_t v) { return __half2float(__ushort_as_half(uint16_t(v))); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __half2float(__ushort_as_half(uint16_t(v >> 16))); }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        uint32_t r; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a)); return r;
    }
};

// Cache codes -> two activation elements.  CACHE: wwws_cache_kind.  `pair` holds the two codes in bytes 0 and 1 ... see each.
// int8 -> f16: 0x6400 | (code ^ 0x80) is 1024 + 128 + code, exact in f16, so one subtraction of 1152 leaves the code.
// int8 -> bf16: bf16 has 7 fraction bits: 0x4300 | low 7 bits is 128 + low7; less 0x4300 | sign bit (128, or 256 when set).
// e4m3 -> f16: the hardware conversion, exact.  e4m3 -> bf16: sign and the 7 exponent/fraction bits moved to bf16's fields read as
// value * 2^-120 (exponent biases 7 and 127); the product with 2^120 is exact, subnormal codes included.
template <bool BF, int CACHE> __device__ __forceinline__ uint32_t widen(uint32_t two)   // codes in bits 0-7 and 8-15
{
    if constexpr (CACHE == WWWS_CACHE_INT8) {
        if constexpr (BF) {
            const uint32_t u = __byte_perm(two, 0x43434343u, 0x4140);
            uint32_t r; asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(u & 0xff7fff7fu), "r"(u & 0xff80ff80u)); return r;
        } else {
            const uint32_t u = __byte_perm(two ^ 0x8080u, 0x64646464u, 0x4140);
            uint32_t r; asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(u), "r"(0x64806480u)); return r;
        }
    } else {
        if constexpr (BF) {
            const uint32_t u = __byte_perm(two, 0u, 0x1404);            // codes in the high byte of each half
            const uint32_t w = (u & 0x80008000u) | ((u >> 4) & 0x07f007f0u);
            uint32_t r; asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0x7b807b80u)); return r;
        } else {
            uint32_t r; asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(uint16_t(two))); return r;
        }
    }
}
#endif

}  // namespace wwws
