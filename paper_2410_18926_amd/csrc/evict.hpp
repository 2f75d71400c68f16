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

// The choice.  The threshold - the key of the last sum that is still kept - is found 11, 11 and 10 bits at a time from histograms of the old keys' sums (eleven bits spread a run of
// exponents over many bins: with eight, most lanes of a wavefront add to one bin and wait for each other); keys above it are kept, and of those that equal it the first.
constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr int kBins = 2048, kBinsEach = kBins / kChooseThreads;
constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};

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

// The sum over the block of two numbers at once.  Two barriers.
__device__ __forceinline__ uint2 block_sums(uint2 v, uint32_t* lds) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        v.x += __shfl_xor(v.x, o, 64);
        v.y += __shfl_xor(v.y, o, 64);
    }
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x >> 6] = v.x;
        lds[kChooseWaves + (threadIdx.x >> 6)] = v.y;
    }
    __syncthreads();
    uint2 all = {0, 0};
#pragma unroll
    for (int w = 0; w < kChooseWaves; ++w) {
        all.x += lds[w];
        all.y += lds[kChooseWaves + w];
    }
    __syncthreads();
    return all;
}

// A sequence and head: where its arrays are, how long it is.
struct Seat {
    int s, head, n, old;
    const int32_t* pages;
    const float* sums;
    int32_t* kept;

    __device__ __forceinline__ Seat(const EvictArgs& a, int seat) {
        s = seat / a.st.heads;
        head = seat - s * a.st.heads;
        n = (int)min((int64_t)max(a.lengths[s], 0), a.keys);
        old = max(n - a.recent, 0);
        pages = a.tables + (int64_t)s * a.width;
        sums = a.sums + (int64_t)seat * a.keys;
        kept = a.kept + (int64_t)seat * a.budget;
    }
    __device__ __forceinline__ bool there(const EvictArgs& a, int j) const { return (uint32_t)pages[j >> a.st.shift] < (uint64_t)a.st.pages; }
};

// How many keys of a sequence there are and how many are to be chosen from the old ones.
struct Wanted {
    uint32_t all, olds, want, choose;
    __device__ __forceinline__ Wanted(const EvictArgs& a, const Seat& q, uint32_t* lds) {
        uint2 mine = {0, 0};
        const int P = 1 << a.st.shift;
        for (int p = threadIdx.x; (int64_t)p << a.st.shift < q.n; p += kChooseThreads) {
            const int j = p << a.st.shift;
            if (q.there(a, j)) {
                mine.x += min(P, q.n - j);
                mine.y += min(P, max(q.old - j, 0));
            }
        }
        mine = block_sums(mine, lds);
        set(a, mine.x, mine.y);
    }
    __device__ __forceinline__ Wanted(const EvictArgs& a, uint32_t there, uint32_t old) { set(a, there, old); }
    __device__ __forceinline__ void set(const EvictArgs& a, uint32_t there, uint32_t old) {
        all = there;
        olds = old;
        want = min(all, (uint32_t)a.budget);
        choose = want - min(all - olds, want);                  // (recent <= budget: the newest are at most `want`)
    }
};

// A thread's EACH consecutive keys from j0 on: the sums' keys, and bits of those that are old or new (none: not there).
template <int EACH>
struct Mine {
    uint32_t key[EACH];
    uint32_t old, fresh;
    __device__ __forceinline__ Mine(const EvictArgs& a, const Seat& q, int64_t j0, bool wide) {
        old = fresh = 0;
        float x[EACH];
        if (wide && j0 + EACH <= a.keys) {                      // (16-byte rows: requested together)
#pragma unroll
            for (int i = 0; i < EACH; i += 4) {
                const f32x4 v = *(const f32x4*)(q.sums + j0 + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[i + k] = v[k];
            }
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) x[i] = j0 + i < a.keys ? q.sums[j0 + i] : 0.0f;
        }
        // (EACH divides a page or is 16, a page's least: the thread's keys stand on one)
        const bool there = j0 < q.n && q.there(a, (int)j0);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            key[i] = sum_key(x[i]);
            if (there && j0 + i < q.old) old |= 1u << i;
            else if (there && j0 + i < q.n) fresh |= 1u << i;
        }
    }
    // Adds the next bits of old keys that agree with the threshold so far.
    __device__ __forceinline__ void count(uint32_t* hist, int pass, uint32_t threshold) const {
        const uint32_t mask = pass == 0 ? 0u : ~0u << kShift[pass - 1];
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (old >> i & 1u && (key[i] & mask) == threshold) atomicAdd(&hist[key[i] >> kShift[pass] & ((1u << kBits[pass]) - 1)], 1u);
    }
    // Writes the kept ones: `above` kept and `same` equal ones come before the block's.
    __device__ __forceinline__ void write(const Seat& q, int64_t j0, uint32_t threshold, uint32_t equal, uint32_t above, uint32_t same, uint32_t* lds) const {
        uint32_t keep = fresh, is = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (old >> i & 1u) {
                if (key[i] > threshold) keep |= 1u << i;
                else if (key[i] == threshold) is |= 1u << i;
            }
        uint32_t total;
        const uint32_t before = block_prefix((uint32_t)__popc(keep) | (uint32_t)__popc(is) << 16, lds, total);
        uint32_t eq = same + (before >> 16), at = above + (before & 0xffffu) + min(eq, equal);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const bool e = is >> i & 1u;
            if (keep >> i & 1u || (e && eq < equal)) q.kept[at++] = (int)j0 + i;
            eq += e;
        }
    }
};

// Of the thread's bins (the largest first: thread t has bins kBins - 1 - kBinsEach t and the ones below), which one the rank falls into.  Returns that bin and how many keys are above it.
__device__ __forceinline__ void find_bin(const uint32_t (&mine)[kBinsEach], uint32_t rank, uint32_t* lds, uint32_t* found, uint32_t& bin, uint32_t& above) {
    uint32_t sum = 0, total;
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) sum += mine[i];
    uint32_t upto = block_prefix(sum, lds, total);
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) {
        if (upto < rank && rank <= upto + mine[i]) { found[0] = kBins - 1 - kBinsEach * threadIdx.x - i; found[1] = upto; }
        upto += mine[i];
    }
    __syncthreads();
    bin = found[0];
    above = found[1];
    __syncthreads();
}

// Tables of up to 1024 EACH keys: a block does it all for a sequence and head, keys in registers.  32 sequences of up to 6000 keys of 8 heads: 12 us, bound by the latency of its steps.
template <int EACH>
__global__ void __launch_bounds__(kChooseThreads) k_evict_choose(EvictArgs a, bool wide) {
    __shared__ uint32_t hist[kBins], part[2 * kChooseWaves], found[2];
    const Seat q(a, blockIdx.x);
    const int64_t j0 = (int64_t)threadIdx.x * EACH;
    const Mine<EACH> mine(a, q, j0, wide);
    const Wanted w(a, q, part);
    uint32_t threshold = 0, equal = w.choose;                   // all of the old ones: every key is >= 0
    if (w.choose == 0) threshold = ~0u;                         // (no sum has this key: it would be a NaN's)
    else if (w.choose < w.olds) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
#pragma unroll
            for (int i = 0; i < kBinsEach; ++i) hist[threadIdx.x + i * kChooseThreads] = 0;
            __syncthreads();
            mine.count(hist, pass, threshold);
            __syncthreads();
            uint32_t bins[kBinsEach], bin, above;
#pragma unroll
            for (int i = 0; i < kBinsEach; ++i) bins[i] = hist[kBins - 1 - kBinsEach * threadIdx.x - i];
            find_bin(bins, equal, part, found, bin, above);
            threshold |= bin << kShift[pass];
            equal -= above;
        }
    }
    mine.write(q, j0, threshold, equal, 0, 0, part);
    for (int i = (int)w.want + threadIdx.x; i < a.budget; i += kChooseThreads) q.kept[i] = -1;
    if (q.head == 0 && threadIdx.x == 0) a.kept_lengths[q.s] = (int)w.want;
}

// Longer tables: a block has a chunk of kChunk keys, the histograms of a sequence's chunks are joined by each of its blocks in the next of four launches (PASS 0 .. 3; the last one
// writes).  Sums over the chunks before a block's own tell where its kept keys go.  Bound by the latency of its steps, barriers among them: how many keys a chunk has is counted by the first
// launch, later ones add that up over the chunks in each wavefront for itself (one sequence of 100000 keys of 8 heads: 6 + 9 + 9.5 + 11 us; each walking the tables itself, 6 + 10 + 10.5 + 12).
constexpr int kChunkEach = 8, kChunk = kChooseThreads * kChunkEach;
struct ChunkArgs {
    EvictArgs a;
    int32_t chunks;
    uint32_t* hist[2];         // [seats][chunks][kBins], of this and of the last pass in turn
    uint32_t* place;           // [seats][chunks]: old keys above the threshold so far in the chunks before
    uint2* there;              // [seats][chunks]: keys of a chunk that are there, and the old ones among them
    uint32_t* state;           // [2][seats][2]: threshold so far, rank among the keys that begin with it, of this and of the last pass in turn
};
template <int PASS>
__global__ void __launch_bounds__(kChooseThreads) k_evict_chunks(ChunkArgs c, bool wide) {
    __shared__ uint32_t hist[kBins], part[2 * kChooseWaves], found[2];
    const EvictArgs& a = c.a;
    const int seats = gridDim.x / c.chunks, seat = blockIdx.x / c.chunks, chunk = blockIdx.x - seat * c.chunks;
    const Seat q(a, seat);
    const int64_t j0 = (int64_t)chunk * kChunk + threadIdx.x * kChunkEach;
    const int chunks = min(c.chunks, (int)((q.n + (int64_t)kChunk - 1) / kChunk));          // that hold keys
    if (chunk >= max(chunks, 1)) return;
    const Mine<kChunkEach> mine(a, q, j0, wide);
    uint2 there = {0, 0}, there_before = {0, 0};                // of all chunks, and of those before
    if constexpr (PASS == 0) {
        const uint2 own = block_sums(make_uint2(__popc(mine.old | mine.fresh), __popc(mine.old)), part);
        if (threadIdx.x == 0) c.there[(int64_t)seat * c.chunks + chunk] = own;
    } else {
        for (int k = threadIdx.x & 63; k < chunks; k += 64) {
            const uint2 t = c.there[(int64_t)seat * c.chunks + k];
            there.x += t.x;
            there.y += t.y;
            if (k < chunk) { there_before.x += t.x; there_before.y += t.y; }
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            there.x += __shfl_xor(there.x, o, 64);
            there.y += __shfl_xor(there.y, o, 64);
            there_before.x += __shfl_xor(there_before.x, o, 64);
            there_before.y += __shfl_xor(there_before.y, o, 64);
        }
    }
    const Wanted w(a, there.x, there.y);
    const bool all = PASS > 0 && w.choose == w.olds;            // (nothing is to be searched for; the first launch does not know)
    uint32_t threshold = 0, rank = w.choose, above_before = 0, equal_before = 0;
    if (PASS > 0 && !all && w.choose > 0) {
        const uint32_t* last = c.hist[(PASS + 1) & 1] + (int64_t)seat * c.chunks * kBins;
        uint32_t bins[kBinsEach], before[kBinsEach], bin, above;
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) bins[i] = before[i] = 0;
        static_assert(kBinsEach == 2, "two bins of a thread are read together");
        for (int k0 = 0; k0 < chunks; k0 += 8) {                // (eight are requested together)
            uint2 h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = *(const uint2*)(last + (int64_t)min(k0 + k, chunks - 1) * kBins + kBins - 2 - 2 * threadIdx.x);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool is = k0 + k < chunks, mine_after = k0 + k < chunk;
                bins[0] += is ? h[k].y : 0u;
                bins[1] += is ? h[k].x : 0u;
                before[0] += mine_after ? h[k].y : 0u;
                before[1] += mine_after ? h[k].x : 0u;
            }
        }
        if (PASS > 1) {
            const uint32_t* st = c.state + ((int64_t)((PASS + 1) & 1) * seats + seat) * 2;
            threshold = st[0];
            rank = st[1];
        }
        find_bin(bins, rank, part, found, bin, above);
        threshold |= bin << kShift[PASS > 0 ? PASS - 1 : 0];
        rank -= above;
        // of the chunks before: keys in the bins above, and in the bin itself
        uint32_t more = 0, same = 0;
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) {
            const uint32_t b = kBins - 1 - kBinsEach * threadIdx.x - i;
            if (b > bin) more += before[i];
            if (b == bin) same += before[i];
        }
        const uint2 before_own = block_sums(make_uint2(more, same), part);
        above_before = before_own.x;
        equal_before = before_own.y;
        uint32_t* place = c.place + (int64_t)seat * c.chunks + chunk;
        if (PASS > 1) above_before += *place;
        __syncthreads();
        if (PASS < 3 && threadIdx.x == 0) {
            *place = above_before;
            if (chunk == 0) {
                uint32_t* st = c.state + ((int64_t)(PASS & 1) * seats + seat) * 2;
                st[0] = threshold;
                st[1] = rank;
            }
        }
    }
    if constexpr (PASS < 3) {
        if (PASS > 0 && (all || w.choose == 0)) return;
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) hist[threadIdx.x + i * kChooseThreads] = 0;
        __syncthreads();
        mine.count(hist, PASS, threshold);
        __syncthreads();
        uint32_t* to = c.hist[PASS & 1] + ((int64_t)seat * c.chunks + chunk) * kBins;
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) to[threadIdx.x + i * kChooseThreads] = hist[threadIdx.x + i * kChooseThreads];
    } else {
        // keys there before the chunk: the newest count as kept, the old ones where all of them are
        const uint32_t olds = there_before.y, news = there_before.x - olds;
        if (w.choose == 0) { threshold = ~0u; rank = 0; }       // (as in k_evict_choose)
        else if (all) { rank = ~0u; above_before = olds; }      // all old keys, those that equal the threshold (0) among them
        mine.write(q, j0, threshold, rank, above_before + news, equal_before, part);
        for (int i = (int)w.want + chunk * kChooseThreads + threadIdx.x; i < a.budget; i += max(chunks, 1) * kChooseThreads) q.kept[i] = -1;
        if (q.head == 0 && chunk == 0 && threadIdx.x == 0) a.kept_lengths[q.s] = (int)w.want;
    }
}

// Moves the kept tokens: a block has 64 consecutive ones of a sequence and head, at the destination's keys 64 blockIdx.x on.  Their keys are rows of their own.  Their values lie byte by
// byte in rows of components: the 16-byte groups that hold any of the 64 are read into LDS (in order, so that lanes read neighbouring groups) and the bytes picked there - each
// byte read from memory by a lane of its own costs a cycle of the address unit, whatever the cache holds (32 sequences of up to 6000 keys cut to 2048, 4 bits, 8 heads of 128: 64 us so, 42 to 53 as built).
// Bound by memory: where few keys are kept, most lines of the source's values are read all the same.
constexpr int kMoveRoom = 1024;        // 16-byte groups in LDS
template <int BITS>
__global__ void __launch_bounds__(256) k_evict_move(EvictArgs a, int dim) {
    __shared__ int64_t from[64], to[64];                        // (page * heads + head) << shift | place; -1: none
    __shared__ int64_t group[64];                               // from of a token of each 16-token group
    __shared__ uint8_t which[64];                               // a token's group
    __shared__ int many;
    __shared__ __align__(16) i32x4 lds[kMoveRoom];
    const int tid = threadIdx.x, head = blockIdx.y, s = blockIdx.z, P = 1 << a.st.shift;
    const int r0 = blockIdx.x * 64;
    const int64_t seat = (int64_t)s * a.st.heads + head;
    float ks, vs;
    uint32_t kf = 0, vf = 0;
    if (tid < 64) {
        const int r = r0 + tid;
        const int key = r < a.budget ? a.kept[seat * a.budget + r] : -1;
        const int to_page = (r >> a.st.shift) < a.to_width ? a.to_tables[(int64_t)s * a.to_width + (r >> a.st.shift)] : -1;
        int64_t src = -1, dst = -1;
        if (key >= 0) {
            src = a.st.row(a.tables[(int64_t)s * a.width + (key >> a.st.shift)], head) + (key & (P - 1));
            if ((uint32_t)to_page < (uint64_t)a.st.pages) dst = a.st.row(to_page, head) + (r & (P - 1));
        }
        from[tid] = src;
        to[tid] = dst;
        const int64_t mine = src >> 4, last = __shfl_up(mine, 1, 64);
        const uint64_t first = __ballot(src >= 0 && (tid == 0 || mine != last));
        const int g = __popcll(first & (2ull << tid) - 1) - 1;
        which[tid] = (uint8_t)g;                                // (of a token that is not there: not used)
        if (first >> tid & 1) group[g] = src;
        if (tid == 0) many = __popcll(first);
        if (a.kept_sums && r < (int64_t)a.to_width << a.st.shift)
            a.kept_sums[seat * ((int64_t)a.to_width << a.st.shift) + r] = key < 0 ? 0.0f : a.sums[seat * a.keys + key];
        if (dst >= 0) {
            ks = a.st.ks[src];
            vs = a.st.vs[src];
            if constexpr (BITS == 4) { kf = a.st.kf[src]; vf = a.st.vf[src]; }
        }
    }
    __syncthreads();
    const int groups = many;
    if (groups == 0) return;
    const int row = dim * BITS / 8, pieces = row / 16;          // bytes of a row of keys; rows of a page's values
    const int batch = min(kMoveRoom / groups, row);             // rows of the values at a time
    // a page's values: row << shift bytes at (page * heads + head) << shift times row
    auto place = [&](int64_t at) { return a.st.vc + (at >> a.st.shift << a.st.shift) * row + (at & (P - 1)); };
    // everything of the first batch is requested before anything is stored: rounds of waiting are what a block's time is made of
    constexpr int AHEAD = kMoveRoom / 256, KEYS = BITS / 4;     // 16-byte pieces of a thread: values; keys, 64 * 128 * BITS / 8 / 16 / 256
    i32x4 v[AHEAD], k[KEYS];
    int kt[KEYS];
    auto load = [&](int c0, int rows) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int p = tid + 256 * i, c = p / groups, g = p - c * groups;
            if (c < rows) v[i] = *(const i32x4*)(place(group[g] & ~(int64_t)15) + ((int64_t)(c0 + c) << a.st.shift));
        }
    };
    load(0, batch);
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        const int p = tid + 256 * i;
        kt[i] = p / pieces;
        if (p < 64 * pieces && to[kt[i]] >= 0) k[i] = *(const i32x4*)(a.st.kc + from[kt[i]] * row + 16 * (p - kt[i] * pieces));
    }
    if (tid < 64 && to[tid] >= 0) {
        a.st.ks[to[tid]] = ks;
        a.st.vs[to[tid]] = vs;
        if constexpr (BITS == 4) { a.st.kf[to[tid]] = kf; a.st.vf[to[tid]] = vf; }
    }
    // four tokens of a row a thread, 16 threads a row: the destination's four bytes lie together
    const int t0 = (tid & 15) * 4;
    const bool any = to[t0] >= 0, four = to[t0 + 3] >= 0;       // (the four stand on one page: the first of them tells)
    int8_t* const d = place(any ? to[t0] : 0);
    int at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = from[t0 + j] >= 0 ? which[t0 + j] * 16 + (int)(from[t0 + j] & 15) : 0;
    for (int c0 = 0; c0 < row; c0 += batch) {
        const int rows = min(batch, row - c0);
        if (c0) {
            load(c0, rows);
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (tid + 256 * i < rows * groups) lds[tid + 256 * i] = v[i];
        if (!c0) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const int p = tid + 256 * i;
                if (p < 64 * pieces && to[kt[i]] >= 0) *(i32x4*)(a.st.kc + to[kt[i]] * row + 16 * (p - kt[i] * pieces)) = k[i];
            }
        }
        __syncthreads();
        if (!any) continue;
        for (int c = tid >> 4; c < rows; c += 16) {
            const uint8_t* b = (const uint8_t*)lds + c * groups * 16;
            int8_t* const to_row = d + ((int64_t)(c0 + c) << a.st.shift);
            if (four) *(uint32_t*)to_row = b[at[0]] | b[at[1]] << 8 | b[at[2]] << 16 | (uint32_t)b[at[3]] << 24;
            else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (to[t0 + j] >= 0) to_row[j] = (int8_t)b[at[j]];
            }
        }
    }
}

}  // namespace lorann
