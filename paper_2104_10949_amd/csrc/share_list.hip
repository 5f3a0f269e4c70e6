// Gradient clipping on replicated shares: the squared norm over many tensors, the public clip factor, the scaling.
//
// Sum of squares: with x = s_0 + s_1 + s_2 one party's three-term product of x with itself is
// x_i x_i + x_{i+1} x_i + x_i x_{i+1} = x_i (x_i + 2 x_{i+1}), one ring product per element; its sum over all elements
// of all tensors is one additive share of the squared norm.  Everything is exact mod 2^64 whatever the order.
// 16 bytes are read per element and one word is written: bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include <algorithm>

#include "cg.h"
#include "cg_check.h"

namespace {

using cg::aligned;
using cg::check_ptrs;

typedef uint64_t u64;

const int THREADS = 256;

// Tensors of one launch, by value in the kernel's arguments (4 KB): no copy to the device, nothing to keep alive.  A tensor
// longer than MAX_PART is several entries.
const int NORM_MAX = 160, CLIP_MAX = 96;
const u64 MAX_PART = (u64)1 << 31;

struct NormArgs {
    const u64 *a[NORM_MAX], *b[NORM_MAX];
    unsigned n[NORM_MAX];
    unsigned first[NORM_MAX];   // block with the entry's first chunk
    unsigned keep_from;         // first block whose loads may stay in the caches
    int count;
};

struct ClipArgs {
    const u64 *a[CLIP_MAX], *b[CLIP_MAX];
    u64 *za[CLIP_MAX], *zb[CLIP_MAX];
    unsigned n[CLIP_MAX];
    unsigned first[CLIP_MAX];
    int count;
};
static_assert(sizeof(NormArgs) + 32 <= 4096 && sizeof(ClipArgs) + 16 <= 4096, "kernel arguments");

// tensor that a block works on
template <class Args>
__device__ __forceinline__ int tensor_of(const Args& t, unsigned block) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= block) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void set_word_kernel(u64* z, u64 v) { *z = v; }

const int NORM_UNROLL = 8;   // loads of each component under way per lane

// Clipping reads what the norm has read, as soon as the factor is there.  The norm's last KEEP_WORDS elements (both
// components, 64 MB of the 256 MB that the memory-side cache holds) are therefore read as what is wanted again, and
// clipping begins at the end; what lies before them streams past the caches, which is faster for the norm.  Norm of 25.5
// million elements alone, norm and clipping of 19.3 million: 64, 52 and 103 us this way, 68, 52 and 102 with 128 MB kept, 71, 53 and
// 96 with 192 MB; with plain accesses and clipping from the beginning 82, 87 and 101.  (What the norm alone gains from
// 192 to 64 MB, 7 us, norm and clipping lose, 6: a norm that is only watched has no call after it to win them back.)
const u64 KEEP_WORDS = (u64)4 << 20;

template <bool KEEP>
__device__ __forceinline__ u64 load(const u64* p) {
    return KEEP ? *p : __builtin_nontemporal_load(p);
}

// Blocks of 1024 threads, so that few of them fill the chip: their sums meet in one word, at about 10 ns each (1.2 million
// elements in 1200 blocks: 20 us, in 150: 8).
const int NORM_THREADS = 1024;

template <bool KEEP>
__device__ __forceinline__ u64 sum_of_squares(const u64* __restrict__ a, const u64* __restrict__ b, u64 i, u64 end) {
    u64 sum = 0;
    for (; i + (NORM_UNROLL - 1) * NORM_THREADS < end; i += NORM_UNROLL * NORM_THREADS) {
        u64 x[NORM_UNROLL], y[NORM_UNROLL];
#pragma unroll
        for (int u = 0; u < NORM_UNROLL; ++u) { x[u] = load<KEEP>(a + i + u * NORM_THREADS); y[u] = load<KEEP>(b + i + u * NORM_THREADS); }
#pragma unroll
        for (int u = 0; u < NORM_UNROLL; ++u) sum += x[u] * (x[u] + 2 * y[u]);
    }
    u64 x[NORM_UNROLL], y[NORM_UNROLL];   // the rest in one round trip, too
#pragma unroll
    for (int u = 0; u < NORM_UNROLL; ++u) {
        x[u] = y[u] = 0;
        if (i + u * NORM_THREADS < end) { x[u] = a[i + u * NORM_THREADS]; y[u] = b[i + u * NORM_THREADS]; }
    }
#pragma unroll
    for (int u = 0; u < NORM_UNROLL; ++u) sum += x[u] * (x[u] + 2 * y[u]);
    return sum;
}

// Chunk by chunk; `alone`: one block has all of them and its sum is the result.
__global__ __launch_bounds__(NORM_THREADS) void sq_norm_kernel(NormArgs t, unsigned chunks, u64 chunk, bool alone, u64* z) {
    u64 sum = 0;
    for (unsigned b = blockIdx.x; b < chunks; b += gridDim.x) {
        const int k = tensor_of(t, b);
        const u64 begin = (u64)(b - t.first[k]) * chunk, end = begin + chunk < t.n[k] ? begin + chunk : t.n[k];
        sum += b >= t.keep_from ? sum_of_squares<true>(t.a[k], t.b[k], begin + threadIdx.x, end)
                                : sum_of_squares<false>(t.a[k], t.b[k], begin + threadIdx.x, end);
    }
    for (int h = 32; h > 0; h >>= 1) sum += __shfl_xor((unsigned long long)sum, h);
    __shared__ u64 part[NORM_THREADS / 64];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NORM_THREADS / 64; ++w) sum += part[w];
        if (alone) *z = sum;
        else atomicAdd(reinterpret_cast<unsigned long long*>(z), (unsigned long long)sum);
    }
}

const int CLIP_UNROLL = 4;

// The list and every tensor's chunks from the end to the beginning (see KEEP_WORDS).
__global__ __launch_bounds__(THREADS) void clip_kernel(ClipArgs t, u64 chunk, const u64* __restrict__ factor) {
    const int k = tensor_of(t, blockIdx.x);
    const u64 n = t.n[k], last = (n - 1) / chunk;
    const u64 begin = (last - (blockIdx.x - t.first[k])) * chunk, end = begin + chunk < n ? begin + chunk : n;
    const u64 c = *factor;
    const u64 *a = t.a[k], *b = t.b[k];
    u64 *za = t.za[k], *zb = t.zb[k];
    u64 i = begin + threadIdx.x;
    for (; i + (CLIP_UNROLL - 1) * THREADS < end; i += CLIP_UNROLL * THREADS) {
        u64 x[CLIP_UNROLL], y[CLIP_UNROLL];
#pragma unroll
        for (int u = 0; u < CLIP_UNROLL; ++u) { x[u] = a[i + u * THREADS]; y[u] = b[i + u * THREADS]; }
#pragma unroll
        for (int u = 0; u < CLIP_UNROLL; ++u) {
            __builtin_nontemporal_store(x[u] * c, za + i + u * THREADS);
            __builtin_nontemporal_store(y[u] * c, zb + i + u * THREADS);
        }
    }
    u64 x[CLIP_UNROLL], y[CLIP_UNROLL];   // the rest in one round trip, too
#pragma unroll
    for (int u = 0; u < CLIP_UNROLL; ++u)
        if (i + u * THREADS < end) { x[u] = a[i + u * THREADS]; y[u] = b[i + u * THREADS]; }
#pragma unroll
    for (int u = 0; u < CLIP_UNROLL; ++u)
        if (i + u * THREADS < end) {
            za[i + u * THREADS] = x[u] * c;
            zb[i + u * THREADS] = y[u] * c;
        }
}

// Largest r with r * r <= v: bit by bit, in integers, so that the three parties' factors are the same word.
__device__ u64 floor_sqrt(u64 v) {
    u64 r = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const u64 t = r | ((u64)1 << bit);
        if (t * t <= v) r = t;
    }
    return r;
}

__global__ void clip_factor_kernel(const u64* s0, const u64* s1, const u64* s2, u64 max_norm, int frac_bits, u64* factor) {
    const u64 norm = floor_sqrt(*s0 + *s1 + *s2);
    *factor = norm <= max_norm ? (u64)1 << frac_bits : (max_norm << frac_bits) / norm;
}

// ---- host ----
struct Range {
    uintptr_t begin, end;
    bool written;
    bool operator<(const Range& o) const { return begin < o.begin; }
};

// Do lists that lie one behind the other, as views of one buffer per component do, meet?  True if none of them can: every
// list of outputs ascends without overlap, and its hull meets no other list's (an input that is its own output aside).
bool lists_apart(const u64* const* const* lists, const size_t* n, size_t count) {
    uintptr_t lo[4], hi[4];
    for (int p = 0; p < 4; ++p) {
        lo[p] = UINTPTR_MAX;
        hi[p] = 0;
        for (size_t k = 0; k < count; ++k) {
            if (n[k] == 0 || (p < 2 && lists[p][k] == lists[p + 2][k])) continue;
            const uintptr_t b = reinterpret_cast<uintptr_t>(lists[p][k]), e = b + n[k] * 8;
            if (p >= 2 && b < hi[p]) return false;
            if (b < lo[p]) lo[p] = b;
            if (e > hi[p]) hi[p] = e;
        }
    }
    for (int p = 2; p < 4; ++p)
        for (int q = 0; q < p; ++q)
            if (lo[p] < hi[q] && lo[q] < hi[p]) return false;
    return true;
}

// Every word that is written is written once and read by nobody else: outputs meet neither each other nor an input,
// except an output equal to the input of its own position.
cg_status check_written(const u64* const* const* lists, const size_t* n, size_t count) {
    if (lists_apart(lists, n, count)) return CG_OK;
    Range* r = static_cast<Range*>(malloc(4 * count * sizeof(Range)));
    if (!r) return CG_ERR_DEVICE;
    size_t m = 0;
    for (size_t k = 0; k < count; ++k) {
        if (n[k] == 0) continue;
        for (int part = 0; part < 4; ++part) {
            if (part < 2 && lists[part][k] == lists[part + 2][k]) continue;   // in place
            const uintptr_t b = reinterpret_cast<uintptr_t>(lists[part][k]);
            r[m++] = {b, b + n[k] * 8, part >= 2};
        }
    }
    std::sort(r, r + m);
    uintptr_t read_end = 0, written_end = 0;
    bool bad = false;
    for (size_t i = 0; i < m && !bad; ++i) {
        bad = r[i].begin < written_end || (r[i].written && r[i].begin < read_end);
        uintptr_t& end = r[i].written ? written_end : read_end;
        if (r[i].end > end) end = r[i].end;
    }
    free(r);
    return bad ? CG_ERR_ALIAS : CG_OK;
}

cg_status check_list(const u64* const* const* lists, int parts, const size_t* n, size_t count, u64* total) {
    *total = 0;
    if (count == 0) return CG_OK;
    if (!n) return CG_ERR_NULL;
    for (int p = 0; p < parts; ++p)
        if (!lists[p]) return CG_ERR_NULL;
    for (size_t k = 0; k < count; ++k) {
        if (n[k] == 0) continue;
        for (int p = 0; p < parts; ++p)
            if (!lists[p][k]) return CG_ERR_NULL;
        for (int p = 0; p < parts; ++p)
            if (!aligned(lists[p][k], 8)) return CG_ERR_ALIGN;
        if (n[k] > (SIZE_MAX >> 4) || __builtin_add_overflow(*total, (u64)n[k], total) || *total > (SIZE_MAX >> 4)) return CG_ERR_SHAPE;
    }
    return CG_OK;
}

// Words of a block's chunk: a power of two, at least `least` and as many as leave at most `blocks` blocks (and one per tensor).
u64 chunk_words(u64 total, u64 blocks, u64 least) {
    u64 c = least;
    while (c * blocks < total) c *= 2;
    return c;
}

}  // namespace

extern "C" {

cg_status cg_share_sq_norm(const uint64_t* const* x_i, const uint64_t* const* x_ip1, const size_t* n, size_t count,
                           uint64_t* z_i, void* stream) {
    if (!z_i) return CG_ERR_NULL;
    if (!aligned(z_i, 8)) return CG_ERR_ALIGN;
    const u64* const* lists[2] = {x_i, x_ip1};
    u64 total;
    if (cg_status st = check_list(lists, 2, n, count, &total)) return st;
    for (size_t k = 0; k < count; ++k)
        if (n[k] > 0 && (cg::overlap(z_i, 8, x_i[k], n[k] * 8) || cg::overlap(z_i, 8, x_ip1[k], n[k] * 8))) return CG_ERR_ALIAS;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const u64 chunk = chunk_words(total, 2048, NORM_UNROLL * NORM_THREADS);
    // up to four chunks, a round trip to memory each, are less than a launch that clears the word
    u64 chunks = 0;
    for (size_t k = 0; k < count && chunks <= 4; ++k) chunks += (n[k] + chunk - 1) / chunk;
    const bool alone = chunks >= 1 && chunks <= 4;   // of at most four tensors, hence one launch
    if (!alone) hipLaunchKernelGGL(set_word_kernel, dim3(1), dim3(1), 0, s, z_i, (u64)0);
    u64 left = total, done = 0;   // words of the list from here on, words of tensor k before here
    for (size_t k = 0; k < count;) {
        NormArgs t;
        t.count = 0;
        t.keep_from = ~0u;
        u64 blocks = 0;
        while (k < count && t.count < NORM_MAX) {
            const u64 part = n[k] - done < MAX_PART ? n[k] - done : MAX_PART;
            if (part > 0) {
                t.a[t.count] = x_i[k] + done;
                t.b[t.count] = x_ip1[k] + done;
                t.n[t.count] = (unsigned)part;
                t.first[t.count++] = (unsigned)blocks;
                if (t.keep_from == ~0u && left <= KEEP_WORDS + part)   // the entry that holds the border, or the first one behind it
                    t.keep_from = (unsigned)(blocks + (left > KEEP_WORDS ? (left - KEEP_WORDS) / chunk : 0));
                blocks += (part + chunk - 1) / chunk;
                left -= part;
                done += part;
            }
            if (done == n[k]) { ++k; done = 0; }
        }
        if (t.count > 0)
            hipLaunchKernelGGL(sq_norm_kernel, dim3(alone ? 1 : (unsigned)blocks), dim3(NORM_THREADS), 0, s, t, (unsigned)blocks, chunk, alone, z_i);
    }
    return hipGetLastError() == hipSuccess ? CG_OK : CG_ERR_DEVICE;
}

cg_status cg_clip_factor(const uint64_t* s0, const uint64_t* s1, const uint64_t* s2, uint64_t max_norm, int frac_bits,
                         uint64_t* factor, void* stream) {
    const void* ptrs[4] = {s0, s1, s2, factor};
    if (cg_status st = check_ptrs(ptrs, 4)) return st;
    if (frac_bits < 0 || frac_bits > 62 || max_norm > (~(u64)0 >> frac_bits)) return CG_ERR_SHAPE;
    hipLaunchKernelGGL(clip_factor_kernel, dim3(1), dim3(1), 0, static_cast<hipStream_t>(stream), s0, s1, s2, max_norm,
                       frac_bits, factor);
    return hipGetLastError() == hipSuccess ? CG_OK : CG_ERR_DEVICE;
}

cg_status cg_share_clip(const uint64_t* const* xa, const uint64_t* const* xb, const uint64_t* factor,
                        uint64_t* const* za, uint64_t* const* zb, const size_t* n, size_t count, void* stream) {
    if (!factor) return CG_ERR_NULL;
    if (!aligned(factor, 8)) return CG_ERR_ALIGN;
    const u64* const* lists[4] = {xa, xb, const_cast<const u64* const*>(za), const_cast<const u64* const*>(zb)};
    u64 total;
    if (cg_status st = check_list(lists, 4, n, count, &total)) return st;
    for (size_t k = 0; k < count; ++k)
        if (n[k] > 0 && (cg::overlap(factor, 8, za[k], n[k] * 8) || cg::overlap(factor, 8, zb[k], n[k] * 8))) return CG_ERR_ALIAS;
    if (total == 0) return CG_OK;
    if (cg_status st = check_written(lists, n, count)) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const u64 chunk = chunk_words(total, 1 << 22, 1024);
    u64 done = 0;   // words of tensor k behind here
    for (size_t next = count; next > 0;) {
        ClipArgs t;
        t.count = 0;
        u64 blocks = 0;
        while (next > 0 && t.count < CLIP_MAX) {
            const size_t k = next - 1;
            const u64 part = n[k] - done < MAX_PART ? n[k] - done : MAX_PART, at = n[k] - done - part;
            if (part > 0) {
                t.a[t.count] = xa[k] + at;
                t.b[t.count] = xb[k] + at;
                t.za[t.count] = za[k] + at;
                t.zb[t.count] = zb[k] + at;
                t.n[t.count] = (unsigned)part;
                t.first[t.count++] = (unsigned)blocks;
                blocks += (part + chunk - 1) / chunk;
                done += part;
            }
            if (done == n[k]) { --next; done = 0; }
        }
        if (t.count > 0) hipLaunchKernelGGL(clip_kernel, dim3((unsigned)blocks), dim3(THREADS), 0, s, t, chunk, factor);
    }
    return hipGetLastError() == hipSuccess ? CG_OK : CG_ERR_DEVICE;
}

}  // extern "C"
