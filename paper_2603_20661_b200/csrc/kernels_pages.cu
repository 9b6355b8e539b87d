// Pages of a paged cache under sequences that are forked, dropped, given room or cut back, and the copies that follow.
//
// k_fork works out the new page tables from how often each page is referred to:
//   refs -= what the old tables hold, refs += the pages that the new sequences take whole.  A page that a new sequence ends inside is to be written further:
//   it stays with the lowest sequence that ends inside it where nobody holds it otherwise (refs is 0 by then), the others get copies.
//   What a sequence needs beside these comes from the pages whose refs are 0, the lowest first, sequences in order.
// Bound by latency: the tables are a few hundred KB in L2 at most, the steps depend on one another.  One cluster of up to 8 blocks does them all, with four
// cluster barriers between them (about a microsecond each with their loads; as five launches they would cost three times that); a row of a table is
// a warp's.  Results do not depend on the order of the atomics: they are sums and minima of whole numbers.
// 48 requests of 5 beams: 13 us; one of 4: 8 us, launch included.
// k_copy_pages and k_compact move bytes and are bound by HBM: 16 bytes a lane, eight loads in flight, every layer in one launch (up to a limit).
// 45 MB copied and written for 48 requests over 6 layers: 12 us; a few tokens of each of 96 requests over 8 layers moved: 6.7 us, most of it latency.
#include <cooperative_groups.h>

#include "backend.cuh"

namespace wwws {
namespace {

constexpr int kForkThreads = 512, kForkWarps = kForkThreads / 32;
constexpr uint32_t kMaxNew = 2048;

__global__ void __launch_bounds__(kForkThreads) k_fork(ForkArgs a)
{
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t rank = cluster.block_rank(), blocks = cluster.num_blocks();
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const uint32_t thread = rank * kForkThreads + tid, threads = blocks * kForkThreads, wid = rank * kForkWarps + warp, warps = blocks * kForkWarps;
    const uint32_t page_mask = (1u << a.page_shift) - 1;
    __shared__ uint32_t prefix[kMaxNew + 1];             // fresh pages of all earlier sequences
    __shared__ uint32_t warp_sum[kForkWarps], free_of[8];
    // What each new sequence is, of the rows that are this block's throughout: its source (-1: none), whole pages, tokens in the page behind them and that page, pages.
    struct New { int source; uint32_t full, cut, held, end; };
    __shared__ New rows[kMaxNew / 8];                    // (8 blocks from 65 rows on)
    const uint32_t most = a.n_old > a.n_new ? a.n_old : a.n_new, per_block = (most + blocks - 1) / blocks, row0 = rank * per_block, row1 = min(most, row0 + per_block);
    auto page_at = [&](uint32_t i, uint32_t k) { return uint32_t(__ldg(a.table + uint64_t(i) * a.max_pages + k)); };

    // 1: refs as they are; the new sequences, a bad one empty; the words in which the first claimant of a page is found
    for (uint32_t i = row0 + tid; i < row1; i += kForkThreads) {
        New n{ -1, 0, 0, 0, 0 };
        if (i < a.n_new) {
            n.source = __ldg(a.source + i);
            const int given = __ldg(a.keep + i), keep = n.source < 0 ? 0 : given, room = __ldg(a.room + i);
            bool ok = n.source < int(a.n_old) && keep >= 0 && room >= 0;
            if (ok && n.source >= 0) {
                const int held = __ldg(a.held + n.source);
                ok = held >= 0 && uint32_t(held) <= a.max_pages && uint32_t(keep) <= uint32_t(held) << a.page_shift;
            }
            if (ok) {
                n.full = uint32_t(keep) >> a.page_shift; n.cut = uint32_t(keep) & page_mask;
                n.held = (uint32_t(max(room, keep)) + page_mask) >> a.page_shift;
                ok = n.held <= a.max_pages;
            }
            if (!ok) { report(a.err, beOffset); n = New{ -1, 0, 0, 0, 0 }; }
            a.held_out[i] = int(n.held);
            if (n.cut) { n.end = page_at(uint32_t(n.source), n.full); if (n.end < a.n_pages) a.owner[n.end] = ~0u; }
        }
        rows[i - row0] = n;
    }
    if (a.refs_out != a.refs)
        for (uint32_t p = thread; p < a.n_pages; p += threads) a.refs_out[p] = __ldg(a.refs + p);
    cluster.sync();

    // 2: old sequences let go, new ones take whole pages.  A sequence that continues itself keeps its pages without either.
    for (uint32_t i = row0 + warp; i < row1; i += kForkWarps) {
        const New n = rows[i - row0];
        int held = 0;
        if (i < a.n_old) {
            held = __ldg(a.held + i);
            if (held < 0 || uint32_t(held) > a.max_pages) { if (lane == 0) report(a.err, beOffset); held = 0; }
        }
        const bool same = n.source == int(i);
        for (uint32_t k = (same ? n.full : 0) + lane; k < uint32_t(held); k += 32) {
            const uint32_t p = page_at(i, k);
            if (p < a.n_pages) atomicAdd(a.refs_out + p, -1); else if (p != ~0u) report(a.err, bePage);       // (-1: a place that an earlier call found no page for)
        }
        if (i < a.n_new) {
            int32_t* to = a.table_out + uint64_t(i) * a.max_pages;
            for (uint32_t k = lane; k < a.max_pages; k += 32) {
                if (k < n.full) {
                    const uint32_t p = page_at(uint32_t(n.source), k);
                    if (p >= a.n_pages) report(a.err, bePage);
                    else if (!same) atomicAdd(a.refs_out + p, 1);
                    to[k] = int(p);
                } else if (k >= n.held) to[k] = 0;
            }
            if (lane == 0 && n.cut && n.end < a.n_pages) atomicMin(a.owner + n.end, i);
        }
    }
    cluster.sync();

    // 3: who keeps the page it ends inside.  Only a page's first claimant writes its refs, and only the others could see that.
    for (uint32_t i = row0 + tid; i < row1 && i < a.n_new; i += kForkThreads) {
        const New n = rows[i - row0];
        int3 move = make_int3(-1, -1, 0);
        uint32_t need = n.held - n.full;
        if (n.cut) {
            if (n.end >= a.n_pages) { report(a.err, bePage); a.table_out[uint64_t(i) * a.max_pages + n.full] = int(n.end); --need; }      // nothing to keep or to copy: it stays outside the pool
            else if (__ldcg(a.owner + n.end) == i && __ldcg(a.refs_out + n.end) == 0) {
                a.refs_out[n.end] = 1;
                a.table_out[uint64_t(i) * a.max_pages + n.full] = int(n.end); --need;
            } else move = make_int3(int(n.end), -1, int(n.cut));
        }
        a.moves[3 * i] = move.x; a.moves[3 * i + 1] = move.y; a.moves[3 * i + 2] = move.z;
        a.need[i] = need;
    }
    cluster.sync();

    // 4: running sum of the needs (every block), free pages of this block's part of the pool (its warps' parts in order)
    uint32_t carry = 0;
    for (uint32_t base = 0; base < a.n_new; base += kForkThreads) {
        const uint32_t own = base + tid < a.n_new ? __ldcg(a.need + base + tid) : 0;
        uint32_t x = own;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, m); if (lane >= uint32_t(m)) x += y; }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        uint32_t before = carry;
        for (int w = 0; w < kForkWarps; ++w) { if (w < int(warp)) before += warp_sum[w]; carry += warp_sum[w]; }
        if (base + tid < a.n_new) prefix[base + tid] = before + x - own;
        __syncthreads();
    }
    if (tid == 0) prefix[a.n_new] = carry;
    const uint32_t total = carry;
    if (total) {                                             // (the same in every block)
        const uint32_t per = ((a.n_pages + warps - 1) / warps + 31) & ~31u, from = min(wid * per, a.n_pages), end = min(from + per, a.n_pages);
        uint32_t n_free = 0;
        for (uint32_t p = from + lane; p - lane < end; p += 32) n_free += __popc(__ballot_sync(0xffffffffu, p < end && __ldcg(a.refs_out + p) == 0));
        if (lane == 0) warp_sum[warp] = n_free;
        __syncthreads();
        if (tid == 0) {
            uint32_t t = 0;
            for (int w = 0; w < kForkWarps; ++w) { const uint32_t x = warp_sum[w]; warp_sum[w] = t; t += x; }
            for (uint32_t r = 0; r < blocks; ++r) cluster.map_shared_rank(free_of, r)[rank] = t;
        }
        cluster.sync();
        uint32_t at = warp_sum[warp], all = 0;
        for (uint32_t r = 0; r < blocks; ++r) { if (r < rank) at += free_of[r]; all += free_of[r]; }

        // 5: the pages go out.  Fresh page number x is the x-th in the order of (sequence, place).
        auto give = [&](uint32_t x, int page) {
            uint32_t i = 0, hi = a.n_new;
            while (hi - i > 1) { const uint32_t mid = (i + hi) >> 1; if (prefix[mid] <= x) i = mid; else hi = mid; }
            const uint32_t need = prefix[i + 1] - prefix[i], k = uint32_t(__ldcg(a.held_out + i)) - need + (x - prefix[i]);     // the last `need` places of the row
            a.table_out[uint64_t(i) * a.max_pages + k] = page;
            if (x == prefix[i] && __ldcg(a.moves + 3 * i + 2)) a.moves[3 * i + 1] = page;
        };
        for (uint32_t p = from + lane; p - lane < end && at < total; p += 32) {
            const bool free = p < end && __ldcg(a.refs_out + p) == 0;
            const uint32_t votes = __ballot_sync(0xffffffffu, free), x = at + __popc(votes & ((1u << lane) - 1));
            if (free && x < total) { a.refs_out[p] = 1; give(x, int(p)); }
            at += __popc(votes);
        }
        if (rank == 0)                                       // the pool is short: these places have no page, and nothing is copied to them
            for (uint32_t x = all + tid; x < total; x += kForkThreads) { report(a.err, bePool); give(x, -1); }
    }
}

constexpr int kCopyThreads = 256, kAhead = 8;

// Bytes [0, 16 n) from one place to another, a block at a time, kAhead pieces of a thread in flight.
template <class F, class G> __device__ __forceinline__ void move_pieces(uint32_t n, uint32_t first, uint32_t step, F&& from, G&& to)
{
    for (uint32_t e = first; e < n; e += step * kAhead) {
        uint4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) if (e + u * step < n) x[u] = __ldcs(from(e + u * step));
#pragma unroll
        for (int u = 0; u < kAhead; ++u) if (e + u * step < n) *to(e + u * step) = x[u];
    }
}

// Block (move, part, layer): the move's tokens of every kv head, keys and values, shared out over the parts.
__global__ void __launch_bounds__(kCopyThreads) k_copy_pages(LayerArgs a, const int32_t* moves)
{
    const int32_t* m = moves + 3 * blockIdx.x;
    const int src = m[0], dst = m[1], tokens = m[2];
    if (dst < 0 || tokens <= 0 || src == dst) return;
    const Layer& l = a.layer[blockIdx.z];
    if (uint32_t(src) >= a.n_pages || uint32_t(dst) >= a.n_pages || uint32_t(tokens) > 1u << a.page_shift) {
        if (threadIdx.x == 0) report(a.err, uint32_t(tokens) > 1u << a.page_shift ? beOffset : bePage);
        return;
    }
    const uint32_t chunks = a.row_bytes / 16, run = uint32_t(tokens) * chunks;               // 16-byte pieces of a head's tokens, which lie together
    const uint64_t s0 = (uint64_t(src) * a.n_kv_heads << a.page_shift) * chunks, d0 = (uint64_t(dst) * a.n_kv_heads << a.page_shift) * chunks;
    const uint32_t step = gridDim.y * kCopyThreads, first = blockIdx.y * kCopyThreads + threadIdx.x;
    auto place = [&](uint32_t e) { const uint32_t h = e / run; return (uint64_t(h) << a.page_shift) * chunks + (e - h * run); };
    const uint32_t half = run * a.n_kv_heads;
    move_pieces(2 * half, first, step,
                [&](uint32_t e) { const bool v = e >= half; return reinterpret_cast<const uint4*>(v ? l.v : l.k) + s0 + place(v ? e - half : e); },
                [&](uint32_t e) { const bool v = e >= half; return reinterpret_cast<uint4*>(v ? l.v : l.k) + d0 + place(v ? e - half : e); });
    if (l.k_scale) {
        const uint64_t s1 = uint64_t(src) * a.n_kv_heads << a.page_shift, d1 = uint64_t(dst) * a.n_kv_heads << a.page_shift;
        const uint32_t n = uint32_t(tokens) * a.n_kv_heads;
        for (uint32_t e = first; e < 2 * n; e += step) {
            const uint32_t x = e >= n ? e - n : e, h = x / uint32_t(tokens);
            const uint64_t at = (uint64_t(h) << a.page_shift) + (x - h * uint32_t(tokens));
            float* f = e >= n ? l.v_scale : l.k_scale;
            f[d1 + at] = f[s1 + at];
        }
    }
}

// Block (sequence, layer).  A thread takes 16-byte columns: place m of the path is written only after it and everything before it is read, and what comes
// later lies behind it (path[m] >= m, ascending), so a column needs no order between threads.
__global__ void __launch_bounds__(kCopyThreads) k_compact(LayerArgs a, SeqBatch b, const int32_t* path, const int32_t* path_len, uint32_t path_stride)
{
    extern __shared__ int64_t cells[];                       // [2][path_len] cell of kv head 0: where from, where to; -1: not in the pool
    __shared__ uint32_t bad;
    const uint32_t i = blockIdx.x, tid = threadIdx.x;
    const Layer& l = a.layer[blockIdx.y];
    if (tid == 0) bad = 0;
    int q0, q_len, kv;
    const bool ok = sequence(b, i, q0, q_len, kv, a.err);
    const int n = path_len[i];
    if (!ok || n == 0) return;
    const int context = kv - q_len;
    if (n < 0 || uint32_t(n) > path_stride || n > q_len || context < 0) { if (tid == 0) report(a.err, beOffset); return; }
    __syncthreads();
    const int32_t* mine = path + uint64_t(i) * path_stride;
    for (int m = tid; m < n; m += kCopyThreads) {
        const int p = mine[m];
        if (p < 0 || p >= q_len || (m && mine[m - 1] >= p)) { bad = 1; continue; }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const uint32_t at = uint32_t(context + (side ? m : p)), page = uint32_t(__ldg(b.page_table + uint64_t(i) * b.table_stride + (at >> a.page_shift)));
            if (page >= a.n_pages) report(a.err, bePage);
            cells[side * n + m] = page >= a.n_pages ? -1 : (int64_t(page) * a.n_kv_heads << a.page_shift) + (at & ((1u << a.page_shift) - 1));
        }
    }
    __syncthreads();
    if (bad) { if (tid == 0) report(a.err, beOffset); return; }
    const uint32_t chunks = a.row_bytes / 16, columns = 2 * a.n_kv_heads * chunks, words = l.k_scale ? 2 * a.n_kv_heads : 0;
    for (uint32_t c = tid; c < columns + words; c += kCopyThreads) {
        const bool word = c >= columns;
        const uint32_t head = word ? c - columns : c / chunks;                                   // keys' heads, then values'
        const bool v = head >= a.n_kv_heads;
        const int64_t off = int64_t(v ? head - a.n_kv_heads : head) << a.page_shift;
        if (word) {
            float* f = v ? l.v_scale : l.k_scale;
            for (int m0 = 0; m0 < n; m0 += kAhead) {
                float x[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) if (m0 + u < n && cells[m0 + u] >= 0) x[u] = f[cells[m0 + u] + off];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) if (m0 + u < n && cells[m0 + u] >= 0 && cells[n + m0 + u] >= 0) f[cells[n + m0 + u] + off] = x[u];
            }
        } else {
            uint4* base = reinterpret_cast<uint4*>(v ? l.v : l.k) + c % chunks;
            for (int m0 = 0; m0 < n; m0 += kAhead) {
                uint4 x[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) if (m0 + u < n && cells[m0 + u] >= 0) x[u] = base[(cells[m0 + u] + off) * chunks];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) if (m0 + u < n && cells[m0 + u] >= 0 && cells[n + m0 + u] >= 0) base[(cells[n + m0 + u] + off) * chunks] = x[u];
            }
        }
    }
}

}  // namespace

cudaError_t launch_fork(const ForkArgs& a, cudaStream_t s)
{
    // A block per 16 rows (a warp each) or 4,096 pages of the pool, 8 at most.
    const uint32_t rows = a.n_old > a.n_new ? a.n_old : a.n_new;
    uint32_t blocks = 1;
    while (blocks < 8 && (blocks * kForkWarps < rows || blocks * 4096 < a.n_pages)) blocks *= 2;        // (8 from 65 rows on, so that a block's rows fit its shared memory)
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(blocks); c.blockDim = dim3(kForkThreads); c.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = blocks; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    c.attrs = &attr; c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_fork, a);
}

cudaError_t launch_copy_pages(const LayerArgs& a, uint32_t n_layers, const int32_t* moves, uint32_t n_moves, cudaStream_t s)
{
    // a part per 64 KB of a full page
    const uint64_t bytes = 2ull * (uint64_t(a.n_kv_heads) << a.page_shift) * a.row_bytes;
    const uint64_t parts = (bytes + 65535) / 65536;
    k_copy_pages<<<dim3(n_moves, uint32_t(parts < 64 ? parts : 64), n_layers), kCopyThreads, 0, s>>>(a, moves);
    return cudaGetLastError();
}

cudaError_t launch_compact(const LayerArgs& a, uint32_t n_layers, const SeqBatch& b, const int32_t* path, const int32_t* path_len, uint32_t path_stride, cudaStream_t s)
{
    k_compact<<<dim3(b.n_seqs, n_layers), kCopyThreads, 16 * path_stride, s>>>(a, b, path, path_len, path_stride);
    return cudaGetLastError();
}

}  // namespace wwws
