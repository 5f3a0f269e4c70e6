// Embedding tables on replicated shares: lookup of rows by public ids, and the table's gradient.
//
// Both are linear in the shared values with public coefficients, hence local on each component of a pair
// (a, b) = (s_i, s_{i+1}), exact mod 2^64 and independent of the order of the additions:
//   lookup     z[j, :] = alpha * table[ids[j], :]
//   gradient   d[v, :] = alpha * sum of g[j, :] over the j with ids[j] = v
// An id outside [0, V) (padding) looks up a row of zeros, which in every share is a share of zero, and adds to no row.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cg.h"
#include "cg_check.h"

namespace {

using cg::aligned;
using cg::all_aligned16;
using cg::check_ptrs;
using cg::overlap;

typedef uint64_t u64;
typedef unsigned long long ull2 __attribute__((ext_vector_type(2)));

const int THREADS = 256;

// A piece of a row is what one wave moves at a time: W words (2 with 16-byte accesses, 1 without) per lane and access,
// UNROLL accesses per component.
template <int W>
struct Words;
template <>
struct Words<2> { typedef ull2 type; };
template <>
struct Words<1> { typedef u64 type; };

const int UNROLL = 4;

// 2^lg lanes (up to a wave) share a row of `units` accesses.
int row_lanes_log2(u64 units) {
    int lg = 0;
    while (lg < 6 && ((u64)1 << lg) < units) ++lg;
    return lg;
}

// Lookup.  A group of 2^lg lanes copies one piece of one row, both components: short rows share a wave, a long row is
// spread over gridDim.y pieces so that a single token's row is one round of loads, too.  Bound by memory: 8192 rows of 768
// in 24.5 us, 5.7 TB/s, with streaming stores (32 with plain ones: the table's frequent rows leave the caches).
template <class Id, int W>
__global__ __launch_bounds__(THREADS) void embed_kernel(const u64* __restrict__ ta, const u64* __restrict__ tb,
                                                        const Id* __restrict__ ids, u64 alpha, u64* __restrict__ za,
                                                        u64* __restrict__ zb, u64 n, u64 V, u64 D, int lg) {
    typedef typename Words<W>::type T;
    const int lane = threadIdx.x & ((1 << lg) - 1);
    const u64 units = D / W, c0 = ((u64)blockIdx.y * UNROLL << lg) + lane;
    for (u64 j = ((u64)blockIdx.x * THREADS + threadIdx.x) >> lg; j < n; j += (u64)gridDim.x * THREADS >> lg) {
        const u64 id = (u64)(long long)ids[j];   // a negative id is beyond every V
        const T *sa = reinterpret_cast<const T*>(ta + id * D), *sb = reinterpret_cast<const T*>(tb + id * D);
        T *oa = reinterpret_cast<T*>(za + j * D), *ob = reinterpret_cast<T*>(zb + j * D);
        const bool there = id < V;
        T a[UNROLL], b[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const u64 c = c0 + ((u64)u << lg);
            a[u] = b[u] = T(0);
            if (there && c < units) { a[u] = sa[c]; b[u] = sb[c]; }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const u64 c = c0 + ((u64)u << lg);
            if (c < units) { __builtin_nontemporal_store(a[u] * alpha, oa + c); __builtin_nontemporal_store(b[u] * alpha, ob + c); }
        }
    }
}

__global__ __launch_bounds__(THREADS) void clear_kernel(u64* a, u64* b, u64 n) {
    for (u64 i = (u64)blockIdx.x * THREADS + threadIdx.x; i < n; i += (u64)gridDim.x * THREADS) {
        a[i] = 0;
        b[i] = 0;
    }
}

__device__ __forceinline__ void add_atomically(u64* p, u64 v) {
    atomicAdd(reinterpret_cast<unsigned long long*>(p), (unsigned long long)v);
}
__device__ __forceinline__ void add_atomically(ull2* p, ull2 v) {
    add_atomically(reinterpret_cast<u64*>(p), v.x);
    add_atomically(reinterpret_cast<u64*>(p) + 1, v.y);
}

// Gradient word by word: every token's row is added to its row of the table's gradient, a wave's atomics on 64 words in a row.
// For few words that are added to a table, and where there is no scratch memory: 65536 tokens of 32000 x 1024: 833 us, 304
// with scratch memory (two words a lane: 1670).
template <class Id>
__global__ __launch_bounds__(THREADS) void embed_grad_kernel(const u64* __restrict__ ga, const u64* __restrict__ gb,
                                                             const Id* __restrict__ ids, u64 alpha, u64* da, u64* db,
                                                             u64 n, u64 V, u64 D) {
    const u64 total = n * D;
    for (u64 i = (u64)blockIdx.x * THREADS + threadIdx.x; i < total; i += (u64)gridDim.x * THREADS) {
        const u64 j = i / D, c = i - j * D, id = (u64)(long long)ids[j];
        if (id >= V) continue;
        add_atomically(da + id * D + c, ga[i] * alpha);
        add_atomically(db + id * D + c, gb[i] * alpha);
    }
}

// ---- gradient with scratch memory: tokens grouped by id ----
// The sums do not depend on the order, so grouping is all the sorting there has to be: a count per row, a place in one
// list for each row's tokens (handed out by a cursor, in whatever order), the list.  Then one group of lanes per row and
// piece adds up the row's tokens and writes the row, once.  Rows of more than `most` tokens are cut into items of that many, which
// are added to the row atomically: a frequent token must not keep one wave busy to the end.  Such a row is cleared by a
// launch before the sums' (or holds what is added to), and so is every row where the whole table is cleared first.

struct Item {
    unsigned row, first, count, whole;   // whole: all of the row's tokens
};

struct Frequent {   // a row of several items, not yet written down
    unsigned row, first, count, slot;
};

struct Grouped {   // in the scratch memory
    unsigned long long* cursor;   // tokens placed so far, and items in the upper half; starts at zero, as frequent_used and the counts do
    unsigned *frequent_used, *count, *offset, *rank, *list;
    Frequent* frequent;
    unsigned char* touched;       // of a middling call instead of all that but the list: a bit per row with tokens
    Item* items;
    u64 items_max, bytes;
    unsigned most;      // tokens of an item, at most 64
    unsigned buckets;   // of a middling call, a power of two
    bool middling;      // one launch groups
    bool clear_first;   // ... and clears the whole table by the way
};

const int GROUP_THREADS = 1024, GROUP_TOKENS = 4;   // of a block that counts tokens, and of each of its threads
const int TABLE = 2 * GROUP_THREADS * GROUP_TOKENS; // places of its hash table: at most half full
const unsigned EMPTY = ~0u;                         // no row: V < 2^31

// Middling calls: every block of `buckets` looks through all ids for those of its own rows, eight in a row and every
// buckets-th eight, and groups them in LDS.  Two launches instead of five; above 20480 tokens the looking through takes longer than
// the launches, and the sums like neighbouring rows better (18485 tokens of 27825 x 16: 29 us and 33 with three launches more;
// 32768 of 32000 x 768: 184 and 172; 65536 of 32000 x 1024: 356 and 311).
const unsigned MIDDLING = 20480, BUCKETS = 128;   // most tokens, most buckets
const u64 MIDDLING_ROWS = (u64)BUCKETS * 8 * GROUP_THREADS;

Grouped grouped_layout(char* p, u64 n, u64 V, u64 D) {
    Grouped g = {};
    // a wave takes two microseconds for eight tokens: items short enough for 8192 waves of 256 words, and in a large call
    // long enough to need few atomics (63904 tokens of 320 x 105: 53 us with 4 tokens, 36 with 8, 29 with 16, 58 with 64; items of at
    // least 8 or 16 tokens, the whole call: 2000 tokens of 30000 x 64 14.9 us and 17.1, 4096 of 32000 x 768 86.8 and 87.6, but 4096 of
    // 1000 x 768 27.8 and 26.7, of 300 x 2048 49.7 and 46.6)
    g.middling = n <= MIDDLING && V <= MIDDLING_ROWS;
    // a row with tokens is then written twice, but its clearing is hidden, and writes go faster without reads among them (4096 tokens of
    // 32000 x 768: 84 us, 87 with the rows without tokens cleared by the sums' launch; 2000 of 128000 x 255: 96 and 109; at the
    // border 12000 of 32000 x 768 113.1 and 113.4, 17000 132.4 and 131.3, 5000 of 8000 x 2048 94.2 and 92.9).  A table of positions, which
    // leaves few rows without tokens, would be better off without: 8192 of 8192 x 700 56.9 and 49.8, of 2048 x 700 36.5 and 36.0.
    g.clear_first = g.middling && n * D <= 6000000 + V * D / 5;
    g.buckets = 32;   // (16 to 64 are alike; 128 keep the clearing waiting, 5 us of 68)
    while (g.buckets < BUCKETS && (u64)g.buckets * 8 * GROUP_THREADS < V) g.buckets *= 2;
    const unsigned least = n <= 4096 ? 8 : 16;
    const double most = (double)n * (double)D / (256.0 * 8192.0);
    g.most = most < least ? least : most < 64 ? (unsigned)most : 64;
    // middling: as many places as tokens, some of them left empty; else rows with tokens, of those with c > most ceil(c / most) items each
    g.items_max = g.middling ? n : (n < V ? n : V) + 2 * n / g.most;
    u64 at = 0;
    const auto take = [&](u64 bytes) { char* q = p + at; at += (bytes + 255) / 256 * 256; return q; };
    g.cursor = reinterpret_cast<unsigned long long*>(take(12 + (g.middling ? 0 : V * 4)));
    g.frequent_used = reinterpret_cast<unsigned*>(g.cursor + 1);
    g.count = g.frequent_used + 1;
    if (g.middling) {
        g.touched = reinterpret_cast<unsigned char*>(take((V + 7) / 8));
    } else {
        g.frequent = reinterpret_cast<Frequent*>(take(n / g.most * sizeof(Frequent)));
        g.offset = reinterpret_cast<unsigned*>(take(V * 4));
        g.rank = reinterpret_cast<unsigned*>(take(n * 4));
    }
    g.list = reinterpret_cast<unsigned*>(take(n * 4));
    g.items = reinterpret_cast<Item*>(take(g.items_max * sizeof(Item)));
    g.bytes = at;
    return g;
}

__global__ __launch_bounds__(THREADS) void group_clear_kernel(unsigned* a, u64 n) {
    for (u64 i = (u64)blockIdx.x * THREADS + threadIdx.x; i < n; i += (u64)gridDim.x * THREADS) a[i] = 0;
}

// Counts a block's tokens, those of j0 + k * GROUP_THREADS, in a hash table in LDS: slot[k] is the place of token k's id
// (EMPTY for padding), rank[k] how many of the block's tokens of that id came before it.
template <class Id>
__device__ __forceinline__ void count_in_table(const Id* __restrict__ ids, u64 n, u64 V, u64 j0, unsigned* key, unsigned* count,
                                               unsigned (&slot)[GROUP_TOKENS], unsigned (&rank)[GROUP_TOKENS]) {
    u64 id[GROUP_TOKENS];
#pragma unroll
    for (int k = 0; k < GROUP_TOKENS; ++k) {
        const u64 j = j0 + (u64)k * GROUP_THREADS;
        id[k] = j < n ? (u64)(long long)ids[j] : ~(u64)0;
    }
    for (int i = threadIdx.x; i < TABLE / 4; i += GROUP_THREADS) {
        reinterpret_cast<uint4*>(key)[i] = make_uint4(EMPTY, EMPTY, EMPTY, EMPTY);
        reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < GROUP_TOKENS; ++k) {
        slot[k] = EMPTY;
        if (id[k] >= V) continue;
        unsigned at = ((unsigned)id[k] * 2654435769u) >> 19;   // 13 bits
        for (;; at = (at + 1) & (TABLE - 1)) {                 // ends: there are fewer ids in the block than places
            const unsigned was = atomicCAS(&key[at], EMPTY, (unsigned)id[k]);
            if (was == EMPTY || was == (unsigned)id[k]) break;
        }
        slot[k] = at;
        rank[k] = atomicAdd(&count[at], 1u);
    }
    __syncthreads();
}
static_assert(TABLE == 1 << 13, "the hash takes the upper 13 bits");

// Sum over the threads before this one, and over all of them.  Every thread of the block calls it.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long own, unsigned long long* wave_sum, unsigned long long* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned long long up_to = own;
    for (int h = 1; h < 64; h <<= 1) {
        const unsigned long long o = __shfl_up(up_to, h);
        if (lane >= h) up_to += o;
    }
    if (lane == 63) wave_sum[wave] = up_to;
    __syncthreads();
    unsigned long long before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < GROUP_THREADS / 64; ++w) {
        const unsigned long long s = wave_sum[w];
        if (w < wave) before += s;
        sum += s;
    }
    *all = sum;
    return before + up_to - own;
}

// Tokens in the lower half, items in the upper half of a row of c tokens.
__device__ __forceinline__ unsigned long long tokens_and_items(unsigned c, unsigned most) {
    return ((unsigned long long)((c + most - 1) / most) << 32) | c;
}

// The items of a frequent row, by thread `mine` of `threads`.
__device__ __forceinline__ void write_items(const Grouped& g, const Frequent& f, unsigned mine, unsigned threads) {
    for (unsigned k = mine; k * g.most < f.count; k += threads) {
        const unsigned left = f.count - k * g.most;
        g.items[f.slot + k] = {f.row, f.first + k * g.most, left < g.most ? left : g.most, 0};
    }
}

// Clears what `empty` says of `all` accesses to both components: this block's part of `blocks` blocks'.  A wave has `each` accesses
// in a row, up to 32 KB of either component, before it goes on (522 MB in 117 us with a stretch of either component per
// block, 99 with 8 KB in a row, 90 with 16 or 32).  `empty` is told where a row of accesses begins.
template <class T, class Empty>
__device__ __forceinline__ void clear_where(u64* da, u64* db, u64 all, unsigned each, unsigned block, unsigned blocks, const Empty& empty) {
    const u64 waves = blockDim.x / 64;
    T *pa = reinterpret_cast<T*>(da), *pb = reinterpret_cast<T*>(db);
    for (u64 i0 = (block * waves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * each; i0 < all; i0 += blocks * waves * each) {
        const auto is_empty = empty(i0);
#pragma unroll 4
        for (unsigned off = threadIdx.x & 63; off < each; off += 64) {
            if (i0 + off < all && is_empty(off)) {
                __builtin_nontemporal_store(T(0), pa + i0 + off);
                __builtin_nontemporal_store(T(0), pb + i0 + off);
            }
        }
    }
}

// ... the rows, of `units` accesses, of which `empty` holds.
template <class T, class Empty>
__device__ __forceinline__ void clear_rows(u64* da, u64* db, u64 V, unsigned units, unsigned each, unsigned block, unsigned blocks,
                                           const Empty& empty) {
    clear_where<T>(da, db, V * units, each, block, blocks, [&](u64 i0) {
        const u64 row0 = i0 / units;
        const unsigned c0 = (unsigned)(i0 - row0 * units);
        return [=, &empty](unsigned off) { return empty(row0 + (c0 + off) / units); };
    });
}

// How blocks of `threads` threads share out the clearing of so many accesses: as much in a row as leaves 4096 waves something,
// a power of two of 64 accesses (393 MB in 68 us with 16 or 32 times 64, 81 with 23).
struct Clearing {
    unsigned each, blocks;
};

Clearing clearing_of(u64 accesses, unsigned threads, u64 most_blocks) {
    Clearing c;
    c.each = 64;
    while (c.each < 32 * 64 && 2 * (u64)c.each * 4096 <= accesses) c.each *= 2;
    const u64 per_block = (u64)(threads / 64) * c.each, blocks = (accesses + per_block - 1) / per_block;
    c.blocks = (unsigned)(blocks < most_blocks ? blocks : most_blocks);
    return c;
}

// A middling call's grouping.  Nothing has to be zero before, and the blocks need nothing of each other: a block that sees all
// ids knows how many tokens the buckets before its own have, which is where its part of the list and of the items begins
// (an item has a token at least).  It also clears its frequent rows, or blocks behind the buckets' clear the whole table.
template <class Id>
__global__ __launch_bounds__(GROUP_THREADS) void group_buckets_kernel(const Id* __restrict__ ids, unsigned n, u64 V, u64 D, int accumulate,
                                                                      u64* da, u64* db, bool pairs, unsigned clear_each, Grouped g) {
    if (blockIdx.x >= g.buckets) {
        const auto every = [](u64) { return [](unsigned) { return true; }; };
        if (pairs) clear_where<ull2>(da, db, V * D / 2, clear_each, blockIdx.x - g.buckets, gridDim.x - g.buckets, every);
        else clear_where<u64>(da, db, V * D, clear_each, blockIdx.x - g.buckets, gridDim.x - g.buckets, every);
        return;
    }
    const int UNROLLED = 8;
    __shared__ __align__(16) unsigned count[8 * GROUP_THREADS];
    __shared__ unsigned long long wave_sum[GROUP_THREADS / 64];
    __shared__ uint2 frequent[MIDDLING / 16];   // rows of more than 16 tokens each, or of more than 8 of at most 4096 tokens: place and count, first item
    __shared__ unsigned frequent_used, before, valid;
    const int shift = __builtin_ctz(g.buckets);
    const unsigned b = blockIdx.x, groups = (unsigned)((V + 7) / 8), own_groups = groups > b ? (groups - b - 1) / g.buckets + 1 : 0;
    for (unsigned i = threadIdx.x; i < 2 * own_groups; i += GROUP_THREADS) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) frequent_used = before = valid = 0;
    __syncthreads();
    // calls f(token, place of its row in `count`) for the tokens of the own rows, and g(bucket) for every valid one
    const auto look_through = [&](const auto& own, const auto& any) {
        for (unsigned j0 = threadIdx.x; j0 < n; j0 += UNROLLED * GROUP_THREADS) {
            u64 id[UNROLLED];
#pragma unroll
            for (int k = 0; k < UNROLLED; ++k) {
                const unsigned j = j0 + k * GROUP_THREADS;
                id[k] = j < n ? (u64)(long long)ids[j] : ~(u64)0;
            }
#pragma unroll
            for (int k = 0; k < UNROLLED; ++k) {
                if (id[k] >= V) continue;
                const unsigned group = (unsigned)id[k] >> 3, bucket = group & (g.buckets - 1);
                any(bucket);
                if (bucket == b) own(j0 + k * GROUP_THREADS, (group >> shift) * 8 + ((unsigned)id[k] & 7));
            }
        }
    };
    unsigned smaller = 0, all_valid = 0;
    look_through([&](unsigned, unsigned place) { atomicAdd(&count[place], 1u); },
                 [&](unsigned bucket) { smaller += bucket < b; ++all_valid; });
    for (int h = 32; h > 0; h >>= 1) {
        smaller += __shfl_xor(smaller, h);
        all_valid += __shfl_xor(all_valid, h);
    }
    if ((threadIdx.x & 63) == 0) {
        atomicAdd(&before, smaller);
        atomicAdd(&valid, all_valid);
    }
    __syncthreads();
    // a thread has eight rows
    unsigned c[8];
    unsigned long long own = 0, all;
    unsigned touched = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        c[k] = threadIdx.x < own_groups ? count[8 * threadIdx.x + k] : 0;
        own += tokens_and_items(c[k], g.most);
        touched |= (c[k] > 0 ? 1u : 0u) << k;
    }
    unsigned long long at = block_scan(own, wave_sum, &all);
    Item* items = g.items + before;
    unsigned* list = g.list + before;
    if (threadIdx.x < own_groups) {
        const unsigned group = threadIdx.x * g.buckets + b;
        g.touched[group] = (unsigned char)touched;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const unsigned row = 8 * group + k, first = (unsigned)at, slot = (unsigned)(at >> 32);
            if (c[k] > g.most) frequent[atomicAdd(&frequent_used, 1u)] = make_uint2((8 * threadIdx.x + k) | c[k] << 13, slot);
            else if (c[k] > 0) items[slot] = {row, before + first, c[k], 1};
            count[8 * threadIdx.x + k] = first;
            at += tokens_and_items(c[k], g.most);
        }
    }
    for (unsigned i = (unsigned)(all >> 32) + threadIdx.x; i < (unsigned)all; i += GROUP_THREADS) items[i] = {0, 0, 0, 1};
    if (b == 0 && threadIdx.x == 0) *g.cursor = (unsigned long long)valid << 32;
    __syncthreads();
    for (unsigned i = threadIdx.x >> 6; i < frequent_used; i += GROUP_THREADS / 64) {
        const unsigned lane = threadIdx.x & 63, place = frequent[i].x & 8191, tokens = frequent[i].x >> 13;
        const unsigned row = 8 * ((place >> 3 << shift) + b) + (place & 7), first = before + count[place];
        for (unsigned k = lane; k * g.most < tokens; k += 64) {
            const unsigned left = tokens - k * g.most;
            items[frequent[i].y + k] = {row, first + k * g.most, left < g.most ? left : g.most, 0};
        }
        if (accumulate || g.clear_first) continue;
        for (u64 e = lane; e < D; e += 64) {
            da[row * D + e] = 0;
            db[row * D + e] = 0;
        }
    }
    __syncthreads();   // the counts are read above and go up below
    look_through([&](unsigned j, unsigned place) { list[atomicAdd(&count[place], 1u)] = j; }, [](unsigned) {});
}

// rank[j] = how many tokens of the same id came before.  A block adds one number per id to the row's count: atomics of
// thousands of tokens on one word of memory wait for each other (65536 tokens, 7 % of them the same: 76 us without the
// table, 10 with it).
template <class Id>
__global__ __launch_bounds__(GROUP_THREADS) void group_count_kernel(const Id* __restrict__ ids, u64 n, u64 V, Grouped g) {
    __shared__ __align__(16) unsigned key[TABLE], count[TABLE];
    const u64 j0 = (u64)blockIdx.x * (GROUP_THREADS * GROUP_TOKENS) + threadIdx.x;
    unsigned slot[GROUP_TOKENS], rank[GROUP_TOKENS];
    count_in_table(ids, n, V, j0, key, count, slot, rank);
    for (int i = threadIdx.x; i < TABLE; i += GROUP_THREADS)
        if (key[i] != EMPTY) count[i] = atomicAdd(g.count + key[i], count[i]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < GROUP_TOKENS; ++k)
        if (slot[k] != EMPTY) g.rank[j0 + (u64)k * GROUP_THREADS] = count[slot[k]] + rank[k];
}

__global__ __launch_bounds__(GROUP_THREADS) void group_offset_kernel(u64 V, Grouped g) {
    __shared__ unsigned long long wave_sum[GROUP_THREADS / 64], base;
    const u64 v = (u64)blockIdx.x * GROUP_THREADS + threadIdx.x;
    const unsigned c = v < V ? g.count[v] : 0;
    unsigned long long all, at = block_scan(tokens_and_items(c, g.most), wave_sum, &all);
    if (threadIdx.x == 0) base = all ? atomicAdd(g.cursor, all) : 0;
    __syncthreads();
    at += base;
    if (v < V) g.offset[v] = (unsigned)at;
    if (c > g.most) g.frequent[atomicAdd(g.frequent_used, 1u)] = {(unsigned)v, (unsigned)at, c, (unsigned)(at >> 32)};
    else if (c > 0) g.items[at >> 32] = {(unsigned)v, (unsigned)at, c, 1};
}

// The first token_blocks blocks fill the list; the others write down the items of frequent rows and clear the rows that those
// will be added to.
template <class Id>
__global__ __launch_bounds__(THREADS) void group_list_kernel(const Id* __restrict__ ids, u64 n, u64 V, u64 D, Grouped g,
                                                             unsigned token_blocks, int accumulate, u64* da, u64* db) {
    if (blockIdx.x < token_blocks) {
        const u64 j = (u64)blockIdx.x * THREADS + threadIdx.x;
        if (j >= n) return;
        const u64 id = (u64)(long long)ids[j];
        if (id < V) g.list[g.offset[id] + g.rank[j]] = (unsigned)j;
        return;
    }
    const unsigned used = *g.frequent_used;
    for (unsigned i = blockIdx.x - token_blocks; i < used; i += gridDim.x - token_blocks) {
        const Frequent f = g.frequent[i];
        write_items(g, f, threadIdx.x, THREADS);
        if (accumulate) continue;
        for (u64 c = threadIdx.x; c < D; c += THREADS) {
            da[f.row * D + c] = 0;
            db[f.row * D + c] = 0;
        }
    }
}

// Sum of the pieces of several rows, loads of R of them under way at a time.  Lanes behind the row's end read its last
// words and write nothing.
template <int W, int ACCESSES, int ROWS>
struct RowSum {
    typedef typename Words<W>::type T;
    static const int U = ACCESSES;   // per component and lane
    static const int R = ROWS;
    T a[U], b[U];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int u = 0; u < U; ++u) a[u] = b[u] = T(0);
    }

    // the first `valid` of N rows; all loads are under way before the first sum
    template <int N>
    __device__ __forceinline__ void add(const u64* __restrict__ ga, const u64* __restrict__ gb, const unsigned (&row)[N],
                                        unsigned valid, u64 D, const u64 (&c)[U]) {
        T x[N][U], y[N][U];
#pragma unroll
        for (int r = 0; r < N; ++r) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[r][u] = y[r][u] = T(0);
            if (r > 0 && r >= (int)valid) continue;
            const T *pa = reinterpret_cast<const T*>(ga + row[r] * D), *pb = reinterpret_cast<const T*>(gb + row[r] * D);
#pragma unroll
            for (int u = 0; u < U; ++u) { x[r][u] = __builtin_nontemporal_load(pa + c[u]); y[r][u] = __builtin_nontemporal_load(pb + c[u]); }
        }
#pragma unroll
        for (int r = 0; r < N; ++r)
#pragma unroll
            for (int u = 0; u < U; ++u) { a[u] += x[r][u]; b[u] += y[r][u]; }
    }

    // the whole wave works on one row: token i of `count`, at most 64, is in lane i, and the addresses are scalar
    __device__ __forceinline__ void add_tokens(const u64* __restrict__ ga, const u64* __restrict__ gb, unsigned mine,
                                               unsigned count, u64 D, const u64 (&c)[U]) {
        for (unsigned i = 0; i < count; i += R) {
            unsigned row[R];
#pragma unroll
            for (int r = 0; r < R; ++r) row[r] = __builtin_amdgcn_readlane(mine, i + r < count ? i + r : i);
            add(ga, gb, row, count - i, D, c);
        }
    }

    // every lane goes through its own row's tokens
    __device__ __forceinline__ void add_list(const u64* __restrict__ ga, const u64* __restrict__ gb,
                                             const unsigned* __restrict__ list, unsigned count, u64 D, const u64 (&c)[U]) {
        for (unsigned i = 0; i < count; i += R) {
            unsigned row[R];
#pragma unroll
            for (int r = 0; r < R; ++r) row[r] = list[i + r < count ? i + r : i];
            add(ga, gb, row, count - i, D, c);
        }
    }
};

// (65536 tokens of 32000 x 1024: 309 us with 4 accesses and 2 rows under way, 293 with 2 and 2, 288 with 2 and 8, 395 with 1 and 8)
template <int W>
using GroupSum = RowSum<W, 2, 8>;

// The items, by blocks below item_blocks, the pieces of a row next to each other so that its memory is read in one go; the
// other blocks clear the rows without tokens, in the order of the addresses.
template <int W, bool WAVE>
__global__ __launch_bounds__(THREADS) void group_sum_kernel(const u64* __restrict__ ga, const u64* __restrict__ gb, u64 alpha,
                                                            u64* da, u64* db, u64 V, u64 D, int accumulate, int lg,
                                                            unsigned pieces, unsigned item_blocks, unsigned clear_each, Grouped g) {
    typedef typename Words<W>::type T;
    const int U = GroupSum<W>::U;
    const unsigned units = (unsigned)(D / W);
    if (blockIdx.x >= item_blocks) {
        const unsigned block = blockIdx.x - item_blocks, blocks = gridDim.x - item_blocks;
        if (g.middling) clear_rows<T>(da, db, V, units, clear_each, block, blocks, [&](u64 row) { return !(g.touched[row >> 3] >> (row & 7) & 1); });
        else clear_rows<T>(da, db, V, units, clear_each, block, blocks, [&](u64 row) { return g.count[row] == 0; });
        return;
    }
    const unsigned used = (unsigned)(*g.cursor >> 32);
    u64 who = ((u64)blockIdx.x * THREADS + threadIdx.x) >> lg;
    if (WAVE) who = __builtin_amdgcn_readfirstlane((unsigned)who);   // below 2^32: MAX_BLOCKS blocks of 4 waves
    for (; who < (u64)used * pieces; who += (u64)item_blocks * THREADS >> lg) {
        const u64 index = who / pieces;
        const unsigned c0 = (unsigned)(who - index * pieces) * ((unsigned)U << lg) + (threadIdx.x & ((1 << lg) - 1));
        u64 c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            c[u] = c0 + ((u64)u << lg);
            if (c[u] >= units) c[u] = units - 1;
        }
        const Item it = g.items[index];
        if (it.count == 0) continue;   // a place left empty
        GroupSum<W> sum;
        sum.clear();
        if (WAVE) {
            const int lane = threadIdx.x & 63;
            sum.add_tokens(ga, gb, lane < (int)it.count ? g.list[it.first + lane] : 0, it.count, D, c);
        } else {
            sum.add_list(ga, gb, g.list + it.first, it.count, D, c);
        }
        T *pa = reinterpret_cast<T*>(da + it.row * D), *pb = reinterpret_cast<T*>(db + it.row * D);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + ((u64)u << lg) >= units) continue;
            const T x = sum.a[u] * alpha, y = sum.b[u] * alpha;
            if (!it.whole) { add_atomically(pa + c[u], x); add_atomically(pb + c[u], y); }
            else if (accumulate) { pa[c[u]] += x; pb[c[u]] += y; }
            else { __builtin_nontemporal_store(x, pa + c[u]); __builtin_nontemporal_store(y, pb + c[u]); }
        }
    }
}

const u64 MAX_COUNT = 0x7FFFFFFF;
const u64 MAX_ROW = 1 << 22;          // words of a row: its accesses are counted in 32 bits, its pieces by the lookup's grid
const u64 MAX_BLOCKS = 1 << 22;       // a grid has less than 2^32 threads; further rows are a block's next ones

cg_status check_sizes(const void* ids, int id_bytes, size_t n, size_t V, size_t D) {
    if (V < 1 || D < 1 || (id_bytes != 4 && id_bytes != 8)) return CG_ERR_SHAPE;
    u64 words;
    if (__builtin_mul_overflow((u64)n, (u64)D, &words) || words > (SIZE_MAX >> 4)) return CG_ERR_SHAPE;
    if (__builtin_mul_overflow((u64)V, (u64)D, &words) || words > (SIZE_MAX >> 4)) return CG_ERR_SHAPE;
    if (n > MAX_COUNT || V > MAX_COUNT || D > MAX_ROW) return CG_ERR_UNSUPPORTED;
    if (n > 0 && !ids) return CG_ERR_NULL;
    if (n > 0 && !aligned(ids, (size_t)id_bytes)) return CG_ERR_ALIGN;
    return CG_OK;
}

cg_status launched() { return hipGetLastError() == hipSuccess ? CG_OK : CG_ERR_DEVICE; }

template <class Id, int W>
void launch_embed(const u64* ta, const u64* tb, const void* ids, u64 alpha, u64* za, u64* zb, u64 n, u64 V, u64 D,
                  hipStream_t s) {
    const u64 units = D / W;
    const int lg = row_lanes_log2(units);
    const u64 rows = THREADS >> lg, piece = (u64)UNROLL << lg;
    const u64 blocks = (n + rows - 1) / rows;
    hipLaunchKernelGGL((embed_kernel<Id, W>), dim3((unsigned)(blocks < MAX_BLOCKS ? blocks : MAX_BLOCKS), (unsigned)((units + piece - 1) / piece)),
                       dim3(THREADS), 0, s, ta, tb, static_cast<const Id*>(ids), alpha, za, zb, n, V, D, lg);
}

// ---- gradient of few tokens, written in full: one launch, no scratch memory ----
// The first blocks hold all ids in LDS, and each of their waves has a token and a share of its row: ballots over the ids name
// the tokens of the same row, and the first of them adds them all up.  A row with more than OWN tokens waits until the
// block has come to its end: then the waves share its tokens out and meet in LDS.  The other blocks clear the rows without
// tokens, which they know from one bit per row in LDS.  (777 tokens of 1531 x 515: 12.9 us; 14 when this way was chosen, against 19
// in two launches by way of a list and 16 for clearing and then adding word by word, which is 15 instead of 12 at 16 to 256 tokens.)
const int FEW = 1024, FEW_THREADS = 512, WAVES = FEW_THREADS / 64;
const int FEW_ROWS = 1 << 18;
// Sixteen rows under way at a time and pieces of one access per lane: what counts in these calls is the time of a round trip to
// memory, and that a row of very many tokens is shared out over many compute units (1000 tokens of 768 words, all the same: 82 us with
// eight rows and two accesses, 44 us this way; all different: 11 and 15 us).
template <int W>
using FewSum = RowSum<W, 1, 16>;
const int OWN = 8;

template <class Id, int W>
__global__ __launch_bounds__(FEW_THREADS) void few_sum_kernel(const u64* __restrict__ ga, const u64* __restrict__ gb,
                                                              const Id* __restrict__ ids, u64 alpha, u64* da, u64* db, unsigned n,
                                                              u64 V, u64 D, unsigned pieces, unsigned pieces_each, unsigned shares,
                                                              unsigned sum_blocks, unsigned clear_each) {
    typedef typename Words<W>::type T;
    typedef FewSum<W> Sum;
    const int U = Sum::U, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned units = (unsigned)(D / W), steps = (n + 63) / 64;
    __shared__ unsigned key[FEW], waiting[WAVES], waiting_count;
    __shared__ union {
        unsigned touched[FEW_ROWS / 32];
        T part[WAVES - 1][2 * U][64];
    } lds;
    if (blockIdx.x >= sum_blocks) {
        for (unsigned i = threadIdx.x; i < (V + 31) / 32; i += FEW_THREADS) lds.touched[i] = 0;
        __syncthreads();
        for (unsigned j = threadIdx.x; j < n; j += FEW_THREADS) {
            const u64 id = (u64)(long long)ids[j];
            if (id < V) atomicOr(&lds.touched[id >> 5], 1u << (id & 31));
        }
        __syncthreads();
        clear_rows<T>(da, db, V, units, clear_each, blockIdx.x - sum_blocks, gridDim.x - sum_blocks,
                      [&](u64 row) { return !(lds.touched[row >> 5] >> (row & 31) & 1); });
        return;
    }
    for (unsigned j = threadIdx.x; j < steps * 64; j += FEW_THREADS) {
        const u64 id = j < n ? (u64)(long long)ids[j] : ~(u64)0;
        key[j] = id < V ? (unsigned)id : EMPTY;
    }
    if (threadIdx.x == 0) waiting_count = 0;
    __syncthreads();

    const auto write = [&](const Sum& sum, unsigned row, unsigned c0, const u64 (&c)[U]) {
        T *pa = reinterpret_cast<T*>(da + row * D), *pb = reinterpret_cast<T*>(db + row * D);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u * 64 >= units) continue;
            __builtin_nontemporal_store(sum.a[u] * alpha, pa + c[u]);
            __builtin_nontemporal_store(sum.b[u] * alpha, pb + c[u]);
        }
    };
    const auto columns = [&](unsigned c0, u64 (&c)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = c0 + u * 64 < units ? c0 + u * 64 : units - 1;
    };

    // a share is pieces_each pieces of a token's row; a block's waves take shares far apart: the same id is often that of
    // tokens close by, and its waves would wait for each other
    const unsigned own_share = sum_blocks * wave + blockIdx.x, own_token = own_share / shares;
    if (own_token < n && key[own_token] != EMPTY) {
        const unsigned row = key[own_token];
        unsigned count = 0, mine = 0;
        for (unsigned k = 0; k < steps; ++k) {
            u64 who = __ballot(key[64 * k + lane] == row);
            for (; who && count < OWN; who &= who - 1, ++count) {
                const unsigned j = 64 * k + (unsigned)__builtin_ctzll(who);
                mine = lane == (int)count ? j : mine;
            }
            count += (unsigned)__popcll(who);
        }
        if ((unsigned)__builtin_amdgcn_readfirstlane(mine) != own_token) {
            // another token is the first of this row
        } else if (count > OWN) {
            if (lane == 0) waiting[atomicAdd(&waiting_count, 1u)] = own_share;
        } else {
            const unsigned piece0 = (own_share - own_token * shares) * pieces_each;
            for (unsigned piece = piece0; piece < piece0 + pieces_each && piece < pieces; ++piece) {
                const unsigned c0 = piece * (U * 64) + lane;
                u64 c[U];
                columns(c0, c);
                Sum sum;
                sum.clear();
                sum.add_tokens(ga, gb, mine, count, D, c);
                write(sum, row, c0, c);
            }
        }
    }
    __syncthreads();
    const unsigned many = waiting_count;
    for (unsigned i = 0; i < many; ++i) {
        const unsigned share = waiting[i], token = share / shares, piece0 = (share - token * shares) * pieces_each, row = key[token];
        for (unsigned piece = piece0; piece < piece0 + pieces_each && piece < pieces; ++piece) {
            const unsigned c0 = piece * (U * 64) + lane;
            u64 c[U];
            columns(c0, c);
            Sum sum;
            sum.clear();
            unsigned mine = 0, count = 0;
            for (unsigned k = wave; k < steps; k += WAVES)   // every WAVES-th group of 64 ids is this wave's
                for (u64 who = __ballot(key[64 * k + lane] == row); who; who &= who - 1) {
                    const unsigned j = 64 * k + (unsigned)__builtin_ctzll(who);
                    mine = lane == (int)count ? j : mine;
                    if (++count == 64) {
                        sum.add_tokens(ga, gb, mine, 64, D, c);
                        count = 0;
                    }
                }
            sum.add_tokens(ga, gb, mine, count, D, c);
            if (wave > 0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    lds.part[wave - 1][u][lane] = sum.a[u];
                    lds.part[wave - 1][U + u][lane] = sum.b[u];
                }
            }
            __syncthreads();
            if (wave == 0) {
                for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        sum.a[u] += lds.part[w][u][lane];
                        sum.b[u] += lds.part[w][U + u][lane];
                    }
                write(sum, row, c0, c);
            }
            __syncthreads();
        }
    }
}

struct GradCall {
    const u64 *ga, *gb;
    const void* ids;
    u64 alpha;
    u64 *da, *db;
    u64 n, V, D;
    int accumulate;
};

// Blocks of a kernel whose threads take words in turn.
unsigned few_blocks(u64 words) { return (unsigned)((words < 4096 * THREADS ? words + THREADS - 1 : 4096 * THREADS) / THREADS); }

unsigned blocks_of(u64 threads) { return (unsigned)((threads + THREADS - 1) / THREADS); }

template <int W>
void launch_sum(const GradCall& c, const Grouped& g, hipStream_t s) {
    const int U = GroupSum<W>::U;
    const u64 units = c.D / W;
    const int lg = row_lanes_log2((units + U - 1) / U);
    const u64 piece = (u64)U << lg, pieces = (units + piece - 1) / piece;
    u64 items = ((g.items_max * pieces << lg) + THREADS - 1) / THREADS;
    if (items > MAX_BLOCKS) items = MAX_BLOCKS;
    const Clearing clear = clearing_of(c.accumulate || g.clear_first ? 0 : c.V * units, THREADS, MAX_BLOCKS);
    const dim3 grid((unsigned)items + clear.blocks);
    if (lg == 6)
        hipLaunchKernelGGL((group_sum_kernel<W, true>), grid, dim3(THREADS), 0, s, c.ga, c.gb, c.alpha, c.da, c.db, c.V, c.D, c.accumulate, lg,
                           (unsigned)pieces, (unsigned)items, clear.each, g);
    else
        hipLaunchKernelGGL((group_sum_kernel<W, false>), grid, dim3(THREADS), 0, s, c.ga, c.gb, c.alpha, c.da, c.db, c.V, c.D, c.accumulate, lg,
                           (unsigned)pieces, (unsigned)items, clear.each, g);
}

// The way of a call, by its sizes.
enum Route { FEW_TOKENS, WORD_BY_WORD, GROUPED };

// Words of gradient up to which adding to a table word by word, in one launch, is as fast as grouping (2000 tokens of 64 words 12 us
// against 19, of 515 words 20 and 22; 4000 of 768 words 45 and 34), and tokens up to which it does not suffer too much where
// all of them are the same (2000 of 64 words 53 us and 36, 4000: 104 and 61).
const u64 FEW_WORDS = 1 << 20, FEW_ADDED = 2048;

Route route_of(u64 n, u64 V, u64 D, bool accumulate) {
    if (!accumulate) return n <= (u64)FEW && V <= (u64)FEW_ROWS ? FEW_TOKENS : GROUPED;
    return n <= FEW_ADDED && n * D <= FEW_WORDS ? WORD_BY_WORD : GROUPED;
}

template <class Id, int W>
void launch_few(const GradCall& c, hipStream_t s) {
    const u64 units = c.D / W, piece = FewSum<W>::U * 64, pieces = (units + piece - 1) / piece;
    // a wave looks through the ids once for all pieces of its share of a row: as many as leave 8192 waves something to do
    u64 each = c.n * pieces / 8192;
    each = each < 1 ? 1 : each < pieces ? each : pieces;
    const u64 shares = (pieces + each - 1) / each, sums = (c.n * shares + WAVES - 1) / WAVES;
    const Clearing clear = clearing_of(c.V * units, FEW_THREADS, 2048);
    hipLaunchKernelGGL((few_sum_kernel<Id, W>), dim3((unsigned)sums + clear.blocks), dim3(FEW_THREADS), 0, s, c.ga, c.gb, static_cast<const Id*>(c.ids),
                       c.alpha, c.da, c.db, (unsigned)c.n, c.V, c.D, (unsigned)pieces, (unsigned)each, (unsigned)shares, (unsigned)sums, clear.each);
}

template <class Id>
void launch_grouped(const GradCall& c, bool vec, char* workspace, hipStream_t s) {
    const Grouped g = grouped_layout(workspace, c.n, c.V, c.D);
    const Id* ids = static_cast<const Id*>(c.ids);
    if (g.middling) {
        const u64 words = c.V * c.D;
        const bool pairs = aligned(c.da, 16) && aligned(c.db, 16) && words % 2 == 0;
        const Clearing clear = clearing_of(c.accumulate || !g.clear_first ? 0 : pairs ? words / 2 : words, GROUP_THREADS, 2048);
        hipLaunchKernelGGL(group_buckets_kernel<Id>, dim3(g.buckets + clear.blocks), dim3(GROUP_THREADS), 0, s, ids, (unsigned)c.n, c.V, c.D,
                           c.accumulate, c.da, c.db, pairs, clear.each, g);
        if (vec) launch_sum<2>(c, g, s);
        else launch_sum<1>(c, g, s);
        return;
    }
    const unsigned tokens = blocks_of(c.n), clears = blocks_of(c.V + 3);
    const unsigned per_block = GROUP_THREADS * GROUP_TOKENS;
    hipLaunchKernelGGL(group_clear_kernel, dim3(clears < 1024 ? clears : 1024), dim3(THREADS), 0, s, reinterpret_cast<unsigned*>(g.cursor), c.V + 3);
    hipLaunchKernelGGL(group_count_kernel<Id>, dim3((unsigned)((c.n + per_block - 1) / per_block)), dim3(GROUP_THREADS), 0, s, ids, c.n, c.V, g);
    hipLaunchKernelGGL(group_offset_kernel, dim3((unsigned)((c.V + GROUP_THREADS - 1) / GROUP_THREADS)), dim3(GROUP_THREADS), 0, s, c.V, g);
    hipLaunchKernelGGL(group_list_kernel<Id>, dim3(tokens + 512), dim3(THREADS), 0, s, ids, c.n, c.V, c.D, g, tokens, c.accumulate,
                       c.da, c.db);
    if (vec) launch_sum<2>(c, g, s);
    else launch_sum<1>(c, g, s);
}

}  // namespace

extern "C" {

cg_status cg_share_embedding(const uint64_t* ta, const uint64_t* tb, const void* ids, int id_bytes, uint64_t alpha,
                             uint64_t* za, uint64_t* zb, size_t n, size_t V, size_t D, void* stream) {
    if (cg_status st = check_sizes(ids, id_bytes, n, V, D)) return st;
    if (n == 0) return CG_OK;
    const void* ptrs[4] = {ta, tb, za, zb};
    if (cg_status st = check_ptrs(ptrs, 4)) return st;
    const u64 tbytes = (u64)V * D * 8, zbytes = (u64)n * D * 8, ibytes = (u64)n * id_bytes;
    for (int o = 2; o < 4; ++o)
        if (overlap(ptrs[o], zbytes, ta, tbytes) || overlap(ptrs[o], zbytes, tb, tbytes) || overlap(ptrs[o], zbytes, ids, ibytes))
            return CG_ERR_ALIAS;
    if (overlap(za, zbytes, zb, zbytes)) return CG_ERR_ALIAS;
    const bool vec = D % 2 == 0 && all_aligned16(ptrs, 4);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (id_bytes == 8) {
        if (vec) launch_embed<long long, 2>(ta, tb, ids, alpha, za, zb, n, V, D, s);
        else launch_embed<long long, 1>(ta, tb, ids, alpha, za, zb, n, V, D, s);
    } else {
        if (vec) launch_embed<int, 2>(ta, tb, ids, alpha, za, zb, n, V, D, s);
        else launch_embed<int, 1>(ta, tb, ids, alpha, za, zb, n, V, D, s);
    }
    return launched();
}

size_t cg_share_embedding_grad_workspace_bytes(size_t n, size_t V, size_t D, int accumulate) {
    int id = 0;
    if (n == 0 || check_sizes(&id, 4, n, V, D) || route_of(n, V, D, accumulate != 0) != GROUPED) return 0;
    return (size_t)grouped_layout(reinterpret_cast<char*>(256), n, V, D).bytes;
}

cg_status cg_share_embedding_grad(const uint64_t* ga, const uint64_t* gb, const void* ids, int id_bytes, uint64_t alpha,
                                  uint64_t* da, uint64_t* db, size_t n, size_t V, size_t D, int accumulate,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if (cg_status st = check_sizes(ids, id_bytes, n, V, D)) return st;
    if (accumulate != 0 && accumulate != 1) return CG_ERR_SHAPE;
    const void* out[2] = {da, db};
    if (cg_status st = check_ptrs(out, 2)) return st;
    const u64 dbytes = (u64)V * D * 8, gbytes = (u64)n * D * 8, ibytes = (u64)n * id_bytes;
    if (overlap(da, dbytes, db, dbytes)) return CG_ERR_ALIAS;
    bool vec = D % 2 == 0 && all_aligned16(out, 2);
    if (n > 0) {
        const void* in[2] = {ga, gb};
        if (cg_status st = check_ptrs(in, 2)) return st;
        for (int o = 0; o < 2; ++o)
            if (overlap(out[o], dbytes, ga, gbytes) || overlap(out[o], dbytes, gb, gbytes) || overlap(out[o], dbytes, ids, ibytes))
                return CG_ERR_ALIAS;
        vec = vec && all_aligned16(in, 2);
    }
    const u64 need = cg_share_embedding_grad_workspace_bytes(n, V, D, accumulate);
    const bool scratch = need > 0 && workspace && workspace_bytes >= need && aligned(workspace, 16);
    if (scratch) {
        const void* operands[5] = {ga, gb, ids, da, db};
        const u64 bytes[5] = {gbytes, gbytes, ibytes, dbytes, dbytes};
        for (int k = 0; k < 5; ++k)
            if (overlap(workspace, need, operands[k], bytes[k])) return CG_ERR_ALIAS;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const GradCall c = {ga, gb, ids, alpha, da, db, n, V, D, accumulate};
    if (n > 0 && route_of(n, V, D, accumulate) == FEW_TOKENS) {
        if (id_bytes == 8) {
            if (vec) launch_few<long long, 2>(c, s);
            else launch_few<long long, 1>(c, s);
        } else {
            if (vec) launch_few<int, 2>(c, s);
            else launch_few<int, 1>(c, s);
        }
        return launched();
    }
    if (scratch) {
        if (id_bytes == 8) launch_grouped<long long>(c, vec, static_cast<char*>(workspace), s);
        else launch_grouped<int>(c, vec, static_cast<char*>(workspace), s);
        return launched();
    }
    if (!accumulate) hipLaunchKernelGGL(clear_kernel, dim3(few_blocks((u64)V * D)), dim3(THREADS), 0, s, da, db, (u64)V * D);
    if (n > 0) {
        const dim3 grid(few_blocks((u64)n * D));
        if (id_bytes == 8)
            hipLaunchKernelGGL(embed_grad_kernel<long long>, grid, dim3(THREADS), 0, s, ga, gb, static_cast<const long long*>(ids), alpha, da,
                               db, n, V, D);
        else
            hipLaunchKernelGGL(embed_grad_kernel<int>, grid, dim3(THREADS), 0, s, ga, gb, static_cast<const int*>(ids), alpha, da, db, n, V, D);
    }
    return launched();
}

}  // extern "C"
