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

__device__ __forceinline__ u64 wave_sum(u64 v) {
    for (int h = 32; h > 0; h >>= 1) v += __shfl_xor((unsigned long long)v, h);
    return v;
}

struct HeadParams {
    const u64 *ga, *gb, *xa, *xb, *ra, *rb, *cos, *sin;
    const void* pos;
    u64 *out, *dr;
    u64 rows, ld_x, ld_g, ld_out, positions;
    int heads, dim, rot, frac, interleaved, pos64;
};

// One wave per head of a row, one pair of elements per lane and step.
__global__ __launch_bounds__(THREADS) void sq_sum_kernel(HeadParams p) {
    const u64 w = ((u64)blockIdx.x * THREADS + threadIdx.x) >> 6, lane = threadIdx.x & 63;
    const u64 t = w / p.heads, h = w - t * p.heads;
    if (t >= p.rows) return;
    const u64 *a = p.xa + t * p.ld_x + h * p.dim, *b = p.xb + t * p.ld_x + h * p.dim;
    u64 sum = 0;
    for (u64 d = lane; d < (u64)p.dim; d += 64) sum += a[d] * (a[d] + 2 * b[d]);
    sum = wave_sum(sum);
    if (lane == 0) p.out[w] = sum;
}

template <bool GRAD>
__global__ __launch_bounds__(THREADS) void rotate_kernel(HeadParams p) {
    const u64 w = ((u64)blockIdx.x * THREADS + threadIdx.x) >> 6, lane = threadIdx.x & 63;
    const u64 t = w / p.heads, h = w - t * p.heads;
    if (t >= p.rows) return;
    const int half = p.rot / 2;
    const u64 at = p.rot == 0 ? 0 : p.pos64 ? (u64) static_cast<const long long*>(p.pos)[t]
                                            : (u64)(long long) static_cast<const int*>(p.pos)[t];
    const bool there = p.rot == 0 || at < p.positions;
    const u64 *xa = p.xa + t * p.ld_x + h * p.dim, *xb = p.xb + t * p.ld_x + h * p.dim;
    const u64 *ga = GRAD ? p.ga + t * p.ld_g + h * p.dim : nullptr, *gb = GRAD ? p.gb + t * p.ld_g + h * p.dim : nullptr;
    u64* out = p.out + t * p.ld_out + h * p.dim;
    const u64 ra = p.ra[w], r2 = ra + p.rb[w], one = (u64)1 << p.frac;
    u64 dr = 0;
    const int items = half + (p.dim - p.rot);   // pairs to turn, then single elements
    for (int i = (int)lane; i < items; i += 64) {
        const bool pair = i < half;
        const int d1 = !pair ? p.rot + (i - half) : p.interleaved ? 2 * i : i;
        const int d2 = !pair ? d1 : p.interleaved ? 2 * i + 1 : i + half;
        if (!there) {
            out[d1] = 0;
            out[d2] = 0;
            continue;
        }
        const u64 c = pair ? p.cos[at * half + i] : one, s = pair ? p.sin[at * half + i] : 0;
        if (!GRAD) {
            const u64 u1 = xa[d1] * r2 + xb[d1] * ra, u2 = xa[d2] * r2 + xb[d2] * ra;
            out[d1] = u1 * c - u2 * s;
            if (pair) out[d2] = u1 * s + u2 * c;
        } else {
            const u64 a1 = ga[d1], a2 = ga[d2], b1 = gb[d1], b2 = gb[d2];
            const u64 va1 = a1 * c + a2 * s, vb1 = b1 * c + b2 * s;
            out[d1] = va1 * r2 + vb1 * ra;
            dr += xa[d1] * (va1 + vb1) + xb[d1] * va1;
            if (pair) {
                const u64 va2 = a2 * c - a1 * s, vb2 = b2 * c - b1 * s;
                out[d2] = va2 * r2 + vb2 * ra;
                dr += xa[d2] * (va2 + vb2) + xb[d2] * va2;
            }
        }
    }
    if (GRAD) {
        dr = wave_sum(dr);
        if (lane == 0) p.dr[w] = dr;
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

unsigned wave_blocks(u64 waves) { return (unsigned)((waves + THREADS / 64 - 1) / (THREADS / 64)); }

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
    hipLaunchKernelGGL(sq_sum_kernel, dim3(wave_blocks(p.rows * p.heads)), dim3(THREADS), 0, static_cast<hipStream_t>(stream), p);
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
    const HeadParams p = head_params(x_i, x_ip1, r_i, r_ip1, cos, sin, pos, z_i, d);
    hipLaunchKernelGGL(rotate_kernel<false>, dim3(wave_blocks(p.rows * p.heads)), dim3(THREADS), 0, static_cast<hipStream_t>(stream), p);
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
    hipLaunchKernelGGL(rotate_kernel<true>, dim3(wave_blocks(p.rows * p.heads)), dim3(THREADS), 0, static_cast<hipStream_t>(stream), p);
    return launched();
}

}  // extern "C"
