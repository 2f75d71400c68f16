// Keeping the newest keys of a sequence and those with the largest sums of weights (include/lorann_evict.h): the choice, and the move to other pages.
#pragma once
#include "codes4.hpp"

namespace lorann {

struct EvictArgs {
    Store st;
    const int32_t* tables;
    int32_t width;
    const int32_t* lengths;
    const float* sums;
    int64_t keys;              // of a table: width << shift
    int32_t budget, recent;
    const int32_t* to_tables;
    int32_t to_width;
    int32_t *kept, *kept_lengths;
    float* kept_sums;
};

// Larger sums first; -0 and +0 are alike, a NaN comes after every number.
__device__ __forceinline__ uint32_t sum_key(float x) { return x != x ? 0u : float_key_asc(x); }

constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr int kEach = 4;               // consecutive keys of a thread

__device__ __forceinline__ uint32_t wave_prefix_u32(uint32_t v) {          // sum of the lanes up to and with this one
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t w = __shfl_up(v, o, 64);
        if ((threadIdx.x & 63) >= (unsigned)o) v += w;
    }
    return v;
}
// Exclusive prefix sum over the block, and the total.  Two barriers.
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t* lds, uint32_t& total) {
    const int wave = threadIdx.x >> 6;
    const uint32_t upto = wave_prefix_u32(v);
    if ((threadIdx.x & 63) == 63) lds[wave] = upto;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kChooseWaves; ++w) {
        const uint32_t x = lds[w];
        if (w < wave) before += x;
        all += x;
    }
    __syncthreads();
    total = all;
    return before + upto - v;
}

// A block chooses for one sequence and head.  The threshold - the key of the last sum that is still kept - is found a byte at a time from histograms; keys above it are kept, and of those
// that equal it the first.
__global__ void __launch_bounds__(kChooseThreads) k_evict_choose(EvictArgs a) {
    __shared__ uint32_t hist[kChooseWaves][256];
    __shared__ uint32_t part[kChooseWaves];
    __shared__ uint32_t found[3];
    const int tid = threadIdx.x, wave = tid >> 6, s = blockIdx.x / a.st.heads, head = blockIdx.x - s * a.st.heads;
    const int n = (int)min((int64_t)max(a.lengths[s], 0), a.keys), old = max(n - a.recent, 0), P = 1 << a.st.shift;
    const int32_t* pages = a.tables + (int64_t)s * a.width;
    const float* sums = a.sums + ((int64_t)s * a.st.heads + head) * a.keys;
    int32_t* kept = a.kept + ((int64_t)s * a.st.heads + head) * a.budget;
    auto there = [&](int j) { return (uint32_t)pages[j >> a.st.shift] < (uint64_t)a.st.pages; };
    // how many keys there are, and of them old ones
    uint32_t all, olds;
    {
        uint32_t mine = 0, mine_old = 0;
        for (int p = tid; p << a.st.shift < n; p += kChooseThreads) {
            const int j = p << a.st.shift;
            if (there(j)) {
                mine += min(P, n - j);
                mine_old += min(P, max(old - j, 0));
            }
        }
        block_prefix(mine, part, all);
        block_prefix(mine_old, part, olds);
    }
    const uint32_t want = min(all, (uint32_t)a.budget), newest = all - olds;
    const uint32_t choose = want - min(newest, want);           // of the old ones (recent <= budget: newest <= want)
    uint32_t threshold = 0, equal = choose;                     // choose = all of them: every key is >= 0
    if (choose > 0 && choose < olds) {
        uint32_t rank = choose;                                 // among those that begin with `threshold`
#pragma unroll 1
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < kChooseWaves * 256; i += kChooseThreads) ((uint32_t*)hist)[i] = 0;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
            for (int j = tid; j < old; j += kChooseThreads) {
                if (!there(j)) continue;
                const uint32_t key = sum_key(sums[j]);
                if ((key & mask) == threshold) atomicAdd(&hist[wave][key >> shift & 255u], 1u);
            }
            __syncthreads();
            uint32_t mine = 0;                                  // bin 255 - tid: the largest come first
            if (tid < 256)
#pragma unroll
                for (int w = 0; w < kChooseWaves; ++w) mine += hist[w][255 - tid];
            uint32_t total;
            const uint32_t above = block_prefix(mine, part, total);
            if (tid < 256 && above < rank && rank <= above + mine) { found[0] = 255 - tid; found[1] = above; }
            __syncthreads();
            threshold |= found[0] << shift;
            rank -= found[1];
            __syncthreads();
        }
        equal = rank;
    } else if (choose == 0) {
        threshold = ~0u;                                        // (no sum has this key: it would be a NaN's)
        equal = 0;
    }
    // in order
    uint32_t kept_before = 0, equal_before = 0;
    for (int j0 = 0; j0 < n; j0 += kChooseThreads * kEach) {
        uint32_t keep = 0, same = 0;                            // bits of the thread's keys
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = j0 + tid * kEach + i;
            if (j >= n || !there(j)) continue;
            if (j >= old) keep |= 1u << i;
            else {
                const uint32_t key = sum_key(sums[j]);
                if (key > threshold) keep |= 1u << i;
                else if (key == threshold) same |= 1u << i;
            }
        }
        uint32_t total;
        const uint32_t counts = (uint32_t)__popc(keep) | (uint32_t)__popc(same) << 16;
        const uint32_t before = block_prefix(counts, part, total);
        uint32_t eq = equal_before + (before >> 16);            // equal ones before the thread's
        uint32_t at = kept_before + (before & 0xffffu) + min(eq, equal);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const bool is = same >> i & 1u;
            if (keep >> i & 1u || (is && eq < equal)) kept[at++] = j0 + tid * kEach + i;
            eq += is;
        }
        kept_before += total & 0xffffu;
        equal_before += total >> 16;
    }
    for (int i = (int)want + tid; i < a.budget; i += kChooseThreads) kept[i] = -1;
    if (head == 0 && tid == 0) a.kept_lengths[s] = (int)want;
}

// Moves the kept tokens: a block has 64 consecutive ones of a sequence and head, at the destination's keys 64 blockIdx.x on.  Bound by memory where most lines of the source's values are
// needed; a component's row of the values is gathered token by token.
template <int BITS>
__global__ void __launch_bounds__(256) k_evict_move(EvictArgs a, int dim) {
    __shared__ int64_t from[64], to[64];                        // (page * heads + head) << shift | place; -1: none
    const int tid = threadIdx.x, head = blockIdx.y, s = blockIdx.z, P = 1 << a.st.shift;
    const int r0 = blockIdx.x * 64, count = a.kept_lengths[s];
    const int64_t seat = (int64_t)s * a.st.heads + head;
    if (tid < 64) {
        const int r = r0 + tid;
        int64_t src = -1, dst = -1;
        int key = -1;
        if (r < count) {
            key = a.kept[seat * a.budget + r];
            const int page = a.tables[(int64_t)s * a.width + (key >> a.st.shift)], to_page = a.to_tables[(int64_t)s * a.to_width + (r >> a.st.shift)];
            src = a.st.row(page, head) + (key & (P - 1));
            if ((uint32_t)to_page < (uint64_t)a.st.pages) dst = a.st.row(to_page, head) + (r & (P - 1));
        }
        from[tid] = src;
        to[tid] = dst;
        if (a.kept_sums && r < (int64_t)a.to_width << a.st.shift)
            a.kept_sums[seat * ((int64_t)a.to_width << a.st.shift) + r] = key < 0 ? 0.0f : a.sums[seat * a.keys + key];
    }
    __syncthreads();
    if (r0 >= count) return;
    if (tid < 64 && to[tid] >= 0) {
        a.st.ks[to[tid]] = a.st.ks[from[tid]];
        a.st.vs[to[tid]] = a.st.vs[from[tid]];
        if constexpr (BITS == 4) {
            a.st.kf[to[tid]] = a.st.kf[from[tid]];
            a.st.vf[to[tid]] = a.st.vf[from[tid]];
        }
    }
    const int row = dim * BITS / 8, pieces = row / 16;          // bytes of a row of keys; rows of a page's values
    for (int i = tid; i < 64 * pieces; i += 256) {
        const int t = i / pieces, p = i - t * pieces;
        if (to[t] >= 0) *(i32x4*)(a.st.kc + to[t] * row + 16 * p) = *(const i32x4*)(a.st.kc + from[t] * row + 16 * p);
    }
    for (int i = tid; i < 64 * row; i += 256) {
        const int t = i & 63, c = i >> 6;
        if (to[t] < 0) continue;
        // (a page's values: row << shift bytes at (page * heads + head) << shift times row)
        const int64_t f = from[t], d = to[t];
        a.st.vc[(d >> a.st.shift << a.st.shift) * row + ((int64_t)c << a.st.shift) + (d & (P - 1))] = a.st.vc[(f >> a.st.shift << a.st.shift) * row + ((int64_t)c << a.st.shift) + (f & (P - 1))];
    }
}

}  // namespace lorann
