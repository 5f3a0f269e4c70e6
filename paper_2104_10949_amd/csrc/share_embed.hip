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

// 2^*lg lanes (up to a wave) share a row of `units` accesses.
int row_lanes_log2(u64 units) {
    int lg = 0;
    while (lg < 6 && ((u64)1 << lg) < units) ++lg;
    return lg;
}

// Lookup.  A group of 2^lg lanes copies one piece of one row, both components: short rows share a wave, a long row is
// spread over gridDim.y pieces so that a single token's row is one round of loads, too.
template <class Id, int W>
__global__ __launch_bounds__(THREADS) void embed_kernel(const u64* __restrict__ ta, const u64* __restrict__ tb,
                                                        const Id* __restrict__ ids, u64 alpha, u64* __restrict__ za,
                                                        u64* __restrict__ zb, u64 n, u64 V, u64 D, int lg) {
    typedef typename Words<W>::type T;
    const int lane = threadIdx.x & ((1 << lg) - 1);
    const u64 j = ((u64)blockIdx.x * THREADS + threadIdx.x) >> lg;
    if (j >= n) return;
    const u64 units = D / W, id = (u64)(long long)ids[j];   // a negative id is beyond every V
    const u64 c0 = ((u64)blockIdx.y * UNROLL << lg) + lane;
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
        if (c < units) { oa[c] = a[u] * alpha; ob[c] = b[u] * alpha; }
    }
}

__global__ __launch_bounds__(THREADS) void clear_kernel(u64* a, u64* b, u64 n) {
    for (u64 i = (u64)blockIdx.x * THREADS + threadIdx.x; i < n; i += (u64)gridDim.x * THREADS) {
        a[i] = 0;
        b[i] = 0;
    }
}

// Gradient: every token's row is added to its row of the table's gradient, word by word.
template <class Id>
__global__ __launch_bounds__(THREADS) void embed_grad_kernel(const u64* __restrict__ ga, const u64* __restrict__ gb,
                                                             const Id* __restrict__ ids, u64 alpha, u64* da, u64* db,
                                                             u64 n, u64 V, u64 D) {
    const u64 total = n * D;
    for (u64 i = (u64)blockIdx.x * THREADS + threadIdx.x; i < total; i += (u64)gridDim.x * THREADS) {
        const u64 j = i / D, c = i - j * D, id = (u64)(long long)ids[j];
        if (id >= V) continue;
        atomicAdd(reinterpret_cast<unsigned long long*>(da + id * D + c), (unsigned long long)(ga[i] * alpha));
        atomicAdd(reinterpret_cast<unsigned long long*>(db + id * D + c), (unsigned long long)(gb[i] * alpha));
    }
}

const u64 MAX_COUNT = 0x7FFFFFFF;

cg_status check_sizes(const void* ids, int id_bytes, size_t n, size_t V, size_t D) {
    if (V < 1 || D < 1 || (id_bytes != 4 && id_bytes != 8)) return CG_ERR_SHAPE;
    u64 words;
    if (__builtin_mul_overflow((u64)n, (u64)D, &words) || words > (SIZE_MAX >> 4)) return CG_ERR_SHAPE;
    if (__builtin_mul_overflow((u64)V, (u64)D, &words) || words > (SIZE_MAX >> 4)) return CG_ERR_SHAPE;
    if (n > MAX_COUNT || V > MAX_COUNT || D > MAX_COUNT) return CG_ERR_UNSUPPORTED;
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
    hipLaunchKernelGGL((embed_kernel<Id, W>), dim3((unsigned)((n + rows - 1) / rows), (unsigned)((units + piece - 1) / piece)),
                       dim3(THREADS), 0, s, ta, tb, static_cast<const Id*>(ids), alpha, za, zb, n, V, D, lg);
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
    if ((D / (vec ? 2 : 1) + 64 * UNROLL - 1) / (64 * UNROLL) > 65535) return CG_ERR_UNSUPPORTED;
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

cg_status cg_share_embedding_grad(const uint64_t* ga, const uint64_t* gb, const void* ids, int id_bytes, uint64_t alpha,
                                  uint64_t* da, uint64_t* db, size_t n, size_t V, size_t D, int accumulate,
                                  void* stream) {
    if (cg_status st = check_sizes(ids, id_bytes, n, V, D)) return st;
    if (accumulate != 0 && accumulate != 1) return CG_ERR_SHAPE;
    const void* out[2] = {da, db};
    if (cg_status st = check_ptrs(out, 2)) return st;
    const u64 dbytes = (u64)V * D * 8, gbytes = (u64)n * D * 8, ibytes = (u64)n * id_bytes;
    if (overlap(da, dbytes, db, dbytes)) return CG_ERR_ALIAS;
    if (n > 0) {
        const void* in[2] = {ga, gb};
        if (cg_status st = check_ptrs(in, 2)) return st;
        for (int o = 0; o < 2; ++o)
            if (overlap(out[o], dbytes, ga, gbytes) || overlap(out[o], dbytes, gb, gbytes) || overlap(out[o], dbytes, ids, ibytes))
                return CG_ERR_ALIAS;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!accumulate) hipLaunchKernelGGL(clear_kernel, dim3(2048), dim3(THREADS), 0, s, da, db, (u64)V * D);
    if (n > 0) {
        if (id_bytes == 8)
            hipLaunchKernelGGL(embed_grad_kernel<long long>, dim3(4096), dim3(THREADS), 0, s, ga, gb,
                               static_cast<const long long*>(ids), alpha, da, db, n, V, D);
        else
            hipLaunchKernelGGL(embed_grad_kernel<int>, dim3(4096), dim3(THREADS), 0, s, ga, gb,
                               static_cast<const int*>(ids), alpha, da, db, n, V, D);
    }
    return launched();
}

}  // extern "C"
