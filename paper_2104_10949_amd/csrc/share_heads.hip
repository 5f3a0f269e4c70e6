// Norms of the query and key heads on replicated shares, with the position rotation.
//
// A head's norm takes an inverse root, which is a protocol of its own (as the truncation after a product is); what a
// party computes locally around it is
//   sums of squares   q[t,h] = sum_d x_i (x_i + 2 x_{i+1})                      (the three-term product of x with itself)
//   product + turn    u = x_i (r_i + r_{i+1}) + x_{i+1} r_i,  z = R_pos u       (r: the shared inverse norm of the head)
//   gradients         v = R_pos^T g on both components (R is public, so this is local),
//                     dx = v_i (r_i + r_{i+1}) + v_{i+1} r_i,   dr[t,h] = sum_d x_i (v_i + v_{i+1}) + x_{i+1} v_i
// R_pos turns the pairs of the first `rot` elements by the position's angles, in public fixed-point words c and s with f
// fractional bits: (u1, u2) -> (u1 c - u2 s, u1 s + u2 c); the other elements are multiplied by 2^f, so that a head has
// one scale.  A position outside the table turns its row to zero, a share of zero.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cg.h"
#include "cg_check.h"

namespace {

using cg::aligned;
using cg::check_ptrs;
using cg::overlap;

typedef uint64_t u64;

const int THREADS = 256;

struct HeadParams {
    const u64 *ga, *gb, *xa, *xb, *ra, *rb, *cos, *sin;
    const void* pos;
    u64 *out, *dr;
    u64 rows, ld_x, ld_g, ld_out, positions;
    int heads, dim, rot, frac, interleaved, pos64;
};

typedef unsigned long long ull2 __attribute__((ext_vector_type(2)));
template <int W>
struct Words { typedef ull2 type; };
template <>
struct Words<1> { typedef u64 type; };
__device__ __forceinline__ u64 sum_of(u64 v) { return v; }
__device__ __forceinline__ u64 sum_of(ull2 v) { return v.x + v.y; }

// A group of 2^lg lanes per head, SQ_UNROLL accesses of W words per lane and component under way: 16 lanes for 128 elements,
// so that a wave has four heads to load before the first sum.  Bound by memory: 4096 x 25 heads of 128 in 36 us, 5.9 TB/s.
// Plain loads, because the rotation reads the same words next (streaming ones: 33 us here and 55 instead of 48 there).
const int SQ_UNROLL = 4;

template <int W>
__global__ __launch_bounds__(THREADS) void sq_sum_kernel(HeadParams p, int lg) {
    typedef typename Words<W>::type T;
    const unsigned lane = threadIdx.x & ((1 << lg) - 1), units = (unsigned)p.dim / W;
    for (u64 w = ((u64)blockIdx.x * THREADS + threadIdx.x) >> lg; w < p.rows * p.heads; w += (u64)gridDim.x * THREADS >> lg) {
        const unsigned t = (unsigned)w / (unsigned)p.heads, h = (unsigned)w - t * (unsigned)p.heads;
        const T *a = reinterpret_cast<const T*>(p.xa + t * p.ld_x + (u64)h * p.dim), *b = reinterpret_cast<const T*>(p.xb + t * p.ld_x + (u64)h * p.dim);
        T sum = T(0);
        for (unsigned i = lane; i < units; i += SQ_UNROLL << lg) {
            T x[SQ_UNROLL], y[SQ_UNROLL];
#pragma unroll
            for (int u = 0; u < SQ_UNROLL; ++u) {
                const unsigned c = i + (u << lg);
                x[u] = y[u] = T(0);
                if (c < units) { x[u] = a[c]; y[u] = b[c]; }
            }
#pragma unroll
            for (int u = 0; u < SQ_UNROLL; ++u) sum += x[u] * (x[u] + 2 * y[u]);
        }
        u64 all = sum_of(sum);
        for (int h2 = 1 << lg >> 1; h2 > 0; h2 >>= 1) all += __shfl_xor((unsigned long long)all, h2);
        if (lane == 0) p.out[w] = all;
    }
}

// The pair of a turn that lies at unit i of a head: W words each (two neighbouring pairs at a time where they lie half a
// turn apart), or both words of one pair in one access where they lie next to each other.
template <int W, bool INTER>
struct Pairs {
    typedef typename Words<INTER ? 1 : W>::type T;
    static __device__ __forceinline__ void load(const u64* __restrict__ p, unsigned i, unsigned half, T* first, T* second) {
        if (INTER && W == 2) {
            const ull2 v = reinterpret_cast<const ull2*>(p)[i];
            *first = v.x;
            *second = v.y;
        } else if (INTER) {
            *first = p[2 * i];
            *second = p[2 * i + 1];
        } else {
            *first = reinterpret_cast<const T*>(p)[i];
            *second = reinterpret_cast<const T*>(p + half)[i];
        }
    }
    static __device__ __forceinline__ void store(u64* p, unsigned i, unsigned half, T first, T second) {
        if (INTER && W == 2) {
            ull2 v = {(unsigned long long)sum_of(first), (unsigned long long)sum_of(second)};
            __builtin_nontemporal_store(v, reinterpret_cast<ull2*>(p) + i);
        } else if (INTER) {
            p[2 * i] = sum_of(first);
            p[2 * i + 1] = sum_of(second);
        } else {
            __builtin_nontemporal_store(first, reinterpret_cast<T*>(p) + i);
            __builtin_nontemporal_store(second, reinterpret_cast<T*>(p + half) + i);
        }
    }
};

// A group of 2^lg lanes per head: first the pairs that are turned, UNROLL units per lane under way, then the elements that
// are only scaled.  Lanes behind the end read the last unit again and write nothing.  A position outside the table has
// zeros for its angles and for the scale.  Bound by memory (four to eight products of 64 bits per element are a quarter of
// the vector units' time): 4096 x 25 heads of 128 in 48 us right after the sums, 6.6 TB/s with what those left in the caches; the gradient of
// 2048 x 25 in 47 us, 5.6.
template <bool GRAD, int W, bool INTER>
__global__ __launch_bounds__(THREADS) void rotate_kernel(HeadParams p, int lg) {
    typedef Pairs<W, INTER> P;
    typedef typename P::T T;
    typedef typename Words<W>::type S;
    const int UNROLL = GRAD ? 1 : 2;
    const unsigned lane = threadIdx.x & ((1 << lg) - 1), half = (unsigned)p.rot / 2;
    const unsigned pairs = INTER ? half : half / W, singles = (unsigned)(p.dim - p.rot) / W;
    for (u64 w = ((u64)blockIdx.x * THREADS + threadIdx.x) >> lg; w < p.rows * p.heads; w += (u64)gridDim.x * THREADS >> lg) {
        const unsigned t = (unsigned)w / (unsigned)p.heads, h = (unsigned)w - t * (unsigned)p.heads;
        const u64 *xa = p.xa + t * p.ld_x + (u64)h * p.dim, *xb = p.xb + t * p.ld_x + (u64)h * p.dim;
        const u64 *ga = GRAD ? p.ga + t * p.ld_g + (u64)h * p.dim : nullptr, *gb = GRAD ? p.gb + t * p.ld_g + (u64)h * p.dim : nullptr;
        u64* out = p.out + t * p.ld_out + (u64)h * p.dim;
        u64 at = 0;
        bool there = true;
        if (half) {
            at = p.pos64 ? (u64) static_cast<const long long*>(p.pos)[t] : (u64)(long long) static_cast<const int*>(p.pos)[t];
            there = at < p.positions;
            if (!there) at = 0;
        }
        const T *cos = reinterpret_cast<const T*>(p.cos + at * half), *sin = reinterpret_cast<const T*>(p.sin + at * half);
        const u64 ra = p.ra[w], r2 = ra + p.rb[w];
        u64 dr = 0;
        for (unsigned i0 = lane; i0 < pairs; i0 += UNROLL << lg) {
            T a1[UNROLL], a2[UNROLL], b1[UNROLL], b2[UNROLL], c[UNROLL], s[UNROLL];
            T xa1[UNROLL], xa2[UNROLL], xb1[UNROLL], xb2[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const unsigned i = i0 + (u << lg) < pairs ? i0 + (u << lg) : pairs - 1;
                P::load(GRAD ? ga : xa, i, half, &a1[u], &a2[u]);
                P::load(GRAD ? gb : xb, i, half, &b1[u], &b2[u]);
                if (GRAD) {
                    P::load(xa, i, half, &xa1[u], &xa2[u]);
                    P::load(xb, i, half, &xb1[u], &xb2[u]);
                }
                c[u] = cos[i];
                s[u] = sin[i];
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const unsigned i = i0 + (u << lg);
                if (i >= pairs) continue;
                if (!there) c[u] = s[u] = T(0);
                if (!GRAD) {
                    const T u1 = a1[u] * r2 + b1[u] * ra, u2 = a2[u] * r2 + b2[u] * ra;
                    P::store(out, i, half, u1 * c[u] - u2 * s[u], u1 * s[u] + u2 * c[u]);
                } else {
                    const T va1 = a1[u] * c[u] + a2[u] * s[u], va2 = a2[u] * c[u] - a1[u] * s[u];
                    const T vb1 = b1[u] * c[u] + b2[u] * s[u], vb2 = b2[u] * c[u] - b1[u] * s[u];
                    P::store(out, i, half, va1 * r2 + vb1 * ra, va2 * r2 + vb2 * ra);
                    dr += sum_of(xa1[u] * (va1 + vb1) + xb1[u] * va1 + xa2[u] * (va2 + vb2) + xb2[u] * va2);
                }
            }
        }
        for (unsigned i = lane; i < singles; i += 1 << lg) {
            const S va = reinterpret_cast<const S*>((GRAD ? ga : xa) + p.rot)[i] * ((u64)there << p.frac);
            const S vb = reinterpret_cast<const S*>((GRAD ? gb : xb) + p.rot)[i] * ((u64)there << p.frac);
            __builtin_nontemporal_store(va * r2 + vb * ra, reinterpret_cast<S*>(out + p.rot) + i);
            if (GRAD) {
                const S x = reinterpret_cast<const S*>(xa + p.rot)[i], y = reinterpret_cast<const S*>(xb + p.rot)[i];
                dr += sum_of(x * (va + vb) + y * va);
            }
        }
        if (GRAD) {
            for (int o = 1 << lg >> 1; o > 0; o >>= 1) dr += __shfl_xor((unsigned long long)dr, o);
            if (lane == 0) p.dr[w] = dr;
        }
    }
}

// ---- host ----
const int64_t MAX_DIM = 0x7FFFFFFF;

// Extent in bytes of [rows, heads, dim] words with `ld` words from a row to the next; 0 if that overflows or ld is too small.
u64 extent(int64_t rows, int64_t heads, int64_t dim, int64_t ld) {
    int64_t row, all;
    if (__builtin_mul_overflow(heads, dim, &row) || ld < row || __builtin_mul_overflow(rows - 1, ld, &all) ||
        __builtin_add_overflow(all, row, &all) || all > (INT64_MAX >> 4))
        return 0;
    return (u64)all * 8;
}

cg_status check_dims(int64_t rows, int64_t heads, int64_t dim) {
    if (rows < 0 || heads < 1 || dim < 1) return CG_ERR_SHAPE;
    int64_t all;
    if (__builtin_mul_overflow(rows, heads, &all) || __builtin_mul_overflow(all, dim, &all) || all > (INT64_MAX >> 4)) return CG_ERR_SHAPE;
    if (heads > MAX_DIM || dim > MAX_DIM || rows * heads > MAX_DIM) return CG_ERR_UNSUPPORTED;
    return CG_OK;
}

cg_status check_rotate(const cg_head_desc* d, const u64* cos, const u64* sin, const void* pos) {
    if (!d) return CG_ERR_NULL;
    if (cg_status st = check_dims(d->rows, d->heads, d->dim)) return st;
    if (d->rot < 0 || d->rot > d->dim || d->rot % 2 != 0 || d->frac_bits < 0 || d->frac_bits > 63 ||
        (d->interleaved != 0 && d->interleaved != 1))
        return CG_ERR_SHAPE;
    if (d->rot > 0) {
        int64_t words;
        if (d->positions < 1 || (d->pos_bytes != 4 && d->pos_bytes != 8) ||
            __builtin_mul_overflow(d->positions, d->rot / 2, &words) || words > (INT64_MAX >> 4))
            return CG_ERR_SHAPE;
        const void* tables[2] = {cos, sin};
        if (d->rows > 0) {
            if (!pos) return CG_ERR_NULL;
            if (cg_status st = check_ptrs(tables, 2)) return st;
            if (!aligned(pos, (size_t)d->pos_bytes)) return CG_ERR_ALIGN;
        }
    }
    return CG_OK;
}

HeadParams head_params(const u64* xa, const u64* xb, const u64* ra, const u64* rb, const u64* cos, const u64* sin,
                       const void* pos, u64* out, const cg_head_desc* d) {
    HeadParams p = {};
    p.xa = xa; p.xb = xb; p.ra = ra; p.rb = rb; p.cos = cos; p.sin = sin; p.pos = pos; p.out = out;
    p.rows = (u64)d->rows; p.ld_x = (u64)d->ld_x; p.ld_g = (u64)d->ld_g; p.ld_out = (u64)d->ld_out;
    p.positions = (u64)d->positions;
    p.heads = (int)d->heads; p.dim = (int)d->dim; p.rot = (int)d->rot;
    p.frac = (int)d->frac_bits; p.interleaved = (int)d->interleaved; p.pos64 = d->pos_bytes == 8;
    return p;
}

// no output meets an input: `in` and their sizes, the tables and the positions
bool meets_inputs(const void* out, u64 bytes, const void* const* in, const u64* in_bytes, int count) {
    for (int i = 0; i < count; ++i)
        if (in_bytes[i] && overlap(out, bytes, in[i], in_bytes[i])) return true;
    return false;
}

// 2^lg lanes, up to a wave, for `units` accesses, `each` per lane
int lanes_log2(int64_t units, int each) {
    int lg = 0;
    while (lg < 6 && ((int64_t)each << lg) < units) ++lg;
    return lg;
}

// Blocks for `groups` groups of 2^lg lanes: a grid has less than 2^32 threads, further groups are a block's next ones.
dim3 group_blocks(u64 groups, int lg) {
    const u64 blocks = ((groups << lg) + THREADS - 1) / THREADS, most = 1 << 22;
    return dim3((unsigned)(blocks < most ? blocks : most));
}

template <bool GRAD, int W>
void launch_rotate(const HeadParams& p, hipStream_t s) {
    const int64_t pairs = p.interleaved ? p.rot / 2 : p.rot / 2 / W, singles = (p.dim - p.rot) / W;
    const int lg = pairs > singles ? lanes_log2(pairs, GRAD ? 1 : 2) : lanes_log2(singles, 1);
    const dim3 grid = group_blocks(p.rows * p.heads, lg);
    if (p.interleaved) hipLaunchKernelGGL((rotate_kernel<GRAD, W, true>), grid, dim3(THREADS), 0, s, p, lg);
    else hipLaunchKernelGGL((rotate_kernel<GRAD, W, false>), grid, dim3(THREADS), 0, s, p, lg);
}

// 16-byte accesses where everything that is read or written that way begins and goes on in whole pairs of words.
template <bool GRAD>
void launch_rotate(const HeadParams& p, void* stream) {
    const void* ptrs[7] = {p.xa, p.xb, p.out, p.ga, p.gb, p.cos, p.sin};
    bool vec = (p.dim | p.rot | (int)((p.ld_x | p.ld_g | p.ld_out) & 1)) % 2 == 0 && (p.interleaved || p.rot % 4 == 0);
    for (int i = 0; i < (p.rot > 0 && !p.interleaved ? 7 : 5); ++i) vec = vec && aligned(ptrs[i], 16);
    if (vec) launch_rotate<GRAD, 2>(p, static_cast<hipStream_t>(stream));
    else launch_rotate<GRAD, 1>(p, static_cast<hipStream_t>(stream));
}

cg_status launched() { return hipGetLastError() == hipSuccess ? CG_OK : CG_ERR_DEVICE; }

}  // namespace

extern "C" {

cg_status cg_share_head_sq_sum(const uint64_t* x_i, const uint64_t* x_ip1, uint64_t* z_i, int64_t rows, int64_t heads,
                               int64_t dim, int64_t ld_x, void* stream) {
    if (cg_status st = check_dims(rows, heads, dim)) return st;
    if (rows == 0) return CG_OK;
    const u64 xbytes = extent(rows, heads, dim, ld_x), zbytes = (u64)rows * heads * 8;
    if (!xbytes) return CG_ERR_SHAPE;
    const void* ptrs[3] = {x_i, x_ip1, z_i};
    if (cg_status st = check_ptrs(ptrs, 3)) return st;
    if (overlap(z_i, zbytes, x_i, xbytes) || overlap(z_i, zbytes, x_ip1, xbytes)) return CG_ERR_ALIAS;
    HeadParams p = {};
    p.xa = x_i; p.xb = x_ip1; p.out = z_i;
    p.rows = (u64)rows; p.ld_x = (u64)ld_x; p.heads = (int)heads; p.dim = (int)dim;
    const bool vec = dim % 2 == 0 && ld_x % 2 == 0 && aligned(x_i, 16) && aligned(x_ip1, 16);
    const int lg = lanes_log2(dim / (vec ? 2 : 1), SQ_UNROLL);
    const dim3 grid = group_blocks(p.rows * p.heads, lg);
    if (vec) hipLaunchKernelGGL(sq_sum_kernel<2>, grid, dim3(THREADS), 0, static_cast<hipStream_t>(stream), p, lg);
    else hipLaunchKernelGGL(sq_sum_kernel<1>, grid, dim3(THREADS), 0, static_cast<hipStream_t>(stream), p, lg);
    return launched();
}

cg_status cg_share_head_norm_rotate(const uint64_t* x_i, const uint64_t* x_ip1, const uint64_t* r_i, const uint64_t* r_ip1,
                                    const uint64_t* cos, const uint64_t* sin, const void* pos, uint64_t* z_i,
                                    const cg_head_desc* d, void* stream) {
    if (cg_status st = check_rotate(d, cos, sin, pos)) return st;
    if (d->rows == 0) return CG_OK;
    const u64 xbytes = extent(d->rows, d->heads, d->dim, d->ld_x), zbytes = extent(d->rows, d->heads, d->dim, d->ld_out);
    if (!xbytes || !zbytes) return CG_ERR_SHAPE;
    const void* ptrs[5] = {x_i, x_ip1, r_i, r_ip1, z_i};
    if (cg_status st = check_ptrs(ptrs, 5)) return st;
    const u64 rbytes = (u64)d->rows * d->heads * 8, tbytes = (u64)d->positions * (d->rot / 2) * 8;
    const void* in[7] = {x_i, x_ip1, r_i, r_ip1, cos, sin, pos};
    const u64 in_bytes[7] = {xbytes, xbytes, rbytes, rbytes, d->rot ? tbytes : 0, d->rot ? tbytes : 0,
                             d->rot ? (u64)d->rows * d->pos_bytes : 0};
    if (meets_inputs(z_i, zbytes, in, in_bytes, 7)) return CG_ERR_ALIAS;
    HeadParams p = head_params(x_i, x_ip1, r_i, r_ip1, cos, sin, pos, z_i, d);
    p.ld_g = 0;   // there is no g
    launch_rotate<false>(p, stream);
    return launched();
}

cg_status cg_share_head_norm_rotate_grad(const uint64_t* g_i, const uint64_t* g_ip1, const uint64_t* x_i,
                                         const uint64_t* x_ip1, const uint64_t* r_i, const uint64_t* r_ip1,
                                         const uint64_t* cos, const uint64_t* sin, const void* pos, uint64_t* dx_i,
                                         uint64_t* dr_i, const cg_head_desc* d, void* stream) {
    if (cg_status st = check_rotate(d, cos, sin, pos)) return st;
    if (d->rows == 0) return CG_OK;
    const u64 xbytes = extent(d->rows, d->heads, d->dim, d->ld_x), gbytes = extent(d->rows, d->heads, d->dim, d->ld_g),
              dxbytes = extent(d->rows, d->heads, d->dim, d->ld_out);
    if (!xbytes || !gbytes || !dxbytes) return CG_ERR_SHAPE;
    const void* ptrs[8] = {g_i, g_ip1, x_i, x_ip1, r_i, r_ip1, dx_i, dr_i};
    if (cg_status st = check_ptrs(ptrs, 8)) return st;
    const u64 rbytes = (u64)d->rows * d->heads * 8, tbytes = (u64)d->positions * (d->rot / 2) * 8;
    const void* in[9] = {g_i, g_ip1, x_i, x_ip1, r_i, r_ip1, cos, sin, pos};
    const u64 in_bytes[9] = {gbytes, gbytes, xbytes, xbytes, rbytes, rbytes, d->rot ? tbytes : 0, d->rot ? tbytes : 0,
                             d->rot ? (u64)d->rows * d->pos_bytes : 0};
    if (meets_inputs(dx_i, dxbytes, in, in_bytes, 9) || meets_inputs(dr_i, rbytes, in, in_bytes, 9) ||
        overlap(dx_i, dxbytes, dr_i, rbytes))
        return CG_ERR_ALIAS;
    HeadParams p = head_params(x_i, x_ip1, r_i, r_ip1, cos, sin, pos, dx_i, d);
    p.ga = g_i; p.gb = g_ip1; p.dr = dr_i;
    launch_rotate<true>(p, stream);
    return launched();
}

}  // extern "C"
