// Layer normalisation over the features of a row, forward and backward (point-wise work and reductions in
// FP32 on FP16 data: paper section 3.3), and the reduction of the scale and shift vectors' gradients.
//
//   forward   mean = sum x / n ;  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps) ;  h = (x - mean) * rstd
//             y = rn16(h * gamma + beta)
//   backward  g = dy * gamma ;  c1 = sum g / n ;  c2 = sum g*h / n ;  dx = rn16(rstd * (g - c1 - h * c2))
//             dgamma = rn16(sum over rows of dy * h) ;  dbeta = rn16(sum over rows of dy)
//
// Bound: HBM.  Forward reads x and writes y (4 bytes an element), backward reads dy and x and writes dx (6).
// A row lives in the registers of one warp (up to 1024 features) or of one CTA, so everything is read once;
// the variance is a second pass over those registers (sum of squared deviations), not a difference of sums.
// The backward pass adds dy*h and dy into per-thread FP32 column sums while the rows stream by, leaves one
// partial row of them per CTA in the workspace and adds those in a second kernel in a fixed order: results are
// run-to-run identical, nothing is added atomically.  The partial sums are at most 296 rows whatever the batch.
#include <math.h>

#include "mpt_common.cuh"

namespace mpt {
namespace {

__device__ __forceinline__ void unpack8(const uint4 v, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const float2 t = __half22float2(*(const __half2 *)&w[q]);
        f[2 * q] = t.x;
        f[2 * q + 1] = t.y;
    }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const __half2 h = __floats2half2_rn(f[2 * q], f[2 * q + 1]);
        w[q] = *(const uint32_t *)&h;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight neighbouring FP16 values of a row, zeros from `cols` on.  VEC: the row starts on a 16-byte boundary.
// STREAM: data that is used once (evict first); the scale and shift vectors are read by every row instead and
// stay in L1.
template <bool VEC, bool STREAM>
__device__ __forceinline__ uint4 load8(const uint16_t *row, int col, int cols)
{
    if (VEC && col + 8 <= cols) return STREAM ? __ldcs((const uint4 *)(row + col)) : __ldg((const uint4 *)(row + col));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (col + e < cols) w[e >> 1] |= (uint32_t)row[col + e] << (16 * (e & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool VEC>
__device__ __forceinline__ void store8(uint16_t *row, int col, int cols, const uint4 v)
{
    if (VEC && col + 8 <= cols) {
        __stcs((uint4 *)(row + col), v);
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (col + e < cols) row[col + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// Sum over the CTA, the same bits in every thread (xor butterflies over the lanes, then over the warps'
// results).  One barrier; the caller alternates between two `red` arrays, so that a slow warp's reads and the
// next use of an array are always a barrier apart.
__device__ __forceinline__ float cta_sum(float v, float *red)
{
    const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
    v = warp_sum(v);
    if (lane == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(lane < nw ? red[lane] : 0.0f);
}
__device__ __forceinline__ void cta_sum2(float &a, float &b, float2 *red)
{
    const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
    a = warp_sum(a);
    b = warp_sum(b);
    if (lane == 0) red[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    const float2 r = lane < nw ? red[lane] : make_float2(0.0f, 0.0f);
    a = warp_sum(r.x);
    b = warp_sum(r.y);
}

struct LnFwd {
    int rows, cols;
    const uint16_t *x;
    size_t ldx;
    const uint16_t *gamma, *beta;      // beta may be null
    float eps;
    uint16_t *y;
    size_t ldy;
    float *mean, *rstd;                // may be null
};

// One row per warp (WARP) or per CTA; thread t of the group holds the vectors t, t + T, ... (at most VPT).
// MAXT threads at most; rows of one CTA are kept to 384 threads where they fit (12288 features), so that four
// CTAs share an SM and one row's loads run under another's reductions.
template <int VPT, bool VEC, bool WARP, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 384 ? 4 : 1) k_ln_fwd(const LnFwd p)
{
    pdl_trigger();
    pdl_wait();
    __shared__ float red[2][32];
    const int T = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int per_cta = WARP ? blockDim.x >> 5 : 1;
    const float n = (float)p.cols;
    for (int row = blockIdx.x * per_cta + (WARP ? threadIdx.x >> 5 : 0); row < p.rows; row += gridDim.x * per_cta) {
        const uint16_t *xr = p.x + (size_t)row * p.ldx;
        uint4 v[VPT];
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            const int col = (t + u * T) * 8;
            v[u] = col < p.cols ? load8<VEC, true>(xr, col, p.cols) : make_uint4(0u, 0u, 0u, 0u);
        }
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            float f[8];
            unpack8(v[u], f);
            s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
        }
        const float mean = __fdiv_rn(WARP ? warp_sum(s) : cta_sum(s, red[0]), n);
        float d2 = 0.0f;
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            const int col = (t + u * T) * 8;
            float f[8];
            unpack8(v[u], f);
            if (col + 8 <= p.cols) {
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float d = f[e] - mean;
                    d2 = fmaf(d, d, d2);
                }
            } else if (col < p.cols) {
#pragma unroll
                for (int e = 0; e < 7; e++) {
                    const float d = f[e] - mean;
                    if (col + e < p.cols) d2 = fmaf(d, d, d2);
                }
            }
        }
        const float var = __fdiv_rn(WARP ? warp_sum(d2) : cta_sum(d2, red[1]), n);
        const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(var + p.eps));
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        uint16_t *yr = p.y + (size_t)row * p.ldy;
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            const int col = (t + u * T) * 8;
            if (col < p.cols) {
                float f[8], g[8], b[8] = {};
                unpack8(v[u], f);
                unpack8(load8<VEC, false>(p.gamma, col, p.cols), g);
                if (p.beta) unpack8(load8<VEC, false>(p.beta, col, p.cols), b);
#pragma unroll
                for (int e = 0; e < 8; e++) f[e] = fmaf((f[e] - mean) * rstd, g[e], b[e]);
                store8<VEC>(yr, col, p.cols, pack8(f));
            }
        }
    }
}

// Rows too long for one CTA's registers: three passes over the row (the second and third hit L2).
template <bool VEC>
__global__ void __launch_bounds__(1024) k_ln_fwd_long(const LnFwd p)
{
    pdl_trigger();
    pdl_wait();
    __shared__ float red[2][32];
    const float n = (float)p.cols;
    const int step = blockDim.x * 8;
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const uint16_t *xr = p.x + (size_t)row * p.ldx;
        float s = 0.0f;
        for (int col = threadIdx.x * 8; col < p.cols; col += step) {
            float f[8];
            unpack8(load8<VEC, false>(xr, col, p.cols), f);
            s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
        }
        const float mean = __fdiv_rn(cta_sum(s, red[0]), n);
        float d2 = 0.0f;
        for (int col = threadIdx.x * 8; col < p.cols; col += step) {
            float f[8];
            unpack8(load8<VEC, false>(xr, col, p.cols), f);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = f[e] - mean;
                if (col + e < p.cols) d2 = fmaf(d, d, d2);
            }
        }
        const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(cta_sum(d2, red[1]), n) + p.eps));
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        uint16_t *yr = p.y + (size_t)row * p.ldy;
        for (int col = threadIdx.x * 8; col < p.cols; col += step) {
            float f[8], g[8], b[8] = {};
            unpack8(load8<VEC, true>(xr, col, p.cols), f);
            unpack8(load8<VEC, false>(p.gamma, col, p.cols), g);
            if (p.beta) unpack8(load8<VEC, false>(p.beta, col, p.cols), b);
#pragma unroll
            for (int e = 0; e < 8; e++) f[e] = fmaf((f[e] - mean) * rstd, g[e], b[e]);
            store8<VEC>(yr, col, p.cols, pack8(f));
        }
    }
}

struct LnBwd {
    int rows, cols;
    const uint16_t *dy;
    size_t lddy;
    const uint16_t *x;
    size_t ldx;
    const uint16_t *gamma;
    const float *mean, *rstd;
    uint16_t *dx;
    size_t lddx;
    float *parts;                      // [2][gridDim.x][colp]: partial dgamma, then partial dbeta
    int colp;
};

// One row per warp (WARP, 8 warps) or per CTA.  The next row's loads are issued before the reduction of the
// present one.
template <int VPT, bool VEC, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 768) k_ln_bwd(const LnBwd p)
{
    pdl_trigger();
    pdl_wait();
    extern __shared__ float cols_smem[];            // WARP: [8 warps][VPT * 256]
    __shared__ float2 red[2][32];
    const int T = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int per_cta = WARP ? 8 : 1, warp = threadIdx.x >> 5;
    const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
    float ag[VPT][8], ab[VPT][8];
    uint4 gm[VPT];
#pragma unroll
    for (int u = 0; u < VPT; u++) {
        const int col = (t + u * T) * 8;
        gm[u] = col < p.cols ? load8<VEC, false>(p.gamma, col, p.cols) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int e = 0; e < 8; e++) ag[u][e] = ab[u][e] = 0.0f;
    }
    const int first = blockIdx.x * per_cta + (WARP ? warp : 0), stride = gridDim.x * per_cta;
    uint4 nx[VPT], nd[VPT];
    float nmean = 0.0f, nrstd = 0.0f;
    auto fetch = [&](int row) {
        const uint16_t *xr = p.x + (size_t)row * p.ldx, *dr = p.dy + (size_t)row * p.lddy;
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            const int col = (t + u * T) * 8;
            nx[u] = nd[u] = make_uint4(0u, 0u, 0u, 0u);
            if (col < p.cols) {
                nx[u] = load8<VEC, true>(xr, col, p.cols);
                nd[u] = load8<VEC, true>(dr, col, p.cols);
            }
        }
        nmean = p.mean[row];
        nrstd = p.rstd[row];
    };
    if (first < p.rows) fetch(first);
    int flip = 0;
    for (int row = first; row < p.rows; row += stride, flip ^= 1) {
        uint4 vx[VPT], vd[VPT];
#pragma unroll
        for (int u = 0; u < VPT; u++) { vx[u] = nx[u]; vd[u] = nd[u]; }
        const float mean = nmean, rstd = nrstd;
        if (row + stride < p.rows) fetch(row + stride);
        float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            float x[8], d[8], g[8];
            unpack8(vx[u], x);
            unpack8(vd[u], d);
            unpack8(gm[u], g);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float h = (x[e] - mean) * rstd, gy = d[e] * g[e];
                c1 += gy;
                c2 = fmaf(gy, h, c2);
                ag[u][e] = fmaf(d[e], h, ag[u][e]);
                ab[u][e] += d[e];
            }
        }
        if (WARP) {
            c1 = warp_sum(c1);
            c2 = warp_sum(c2);
        } else {
            cta_sum2(c1, c2, red[flip]);
        }
        c1 *= inv_n;
        c2 *= inv_n;
        uint16_t *o = p.dx + (size_t)row * p.lddx;
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            const int col = (t + u * T) * 8;
            if (col < p.cols) {
                float x[8], d[8], g[8];
                unpack8(vx[u], x);
                unpack8(vd[u], d);
                unpack8(gm[u], g);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float h = (x[e] - mean) * rstd;
                    d[e] = rstd * (fmaf(d[e], g[e], -c1) - h * c2);
                }
                store8<VEC>(o, col, p.cols, pack8(d));
            }
        }
    }
    // the CTA's column sums: for rows held by warps, the eight warps' sums are added in warp order
    float *pg = p.parts + (size_t)blockIdx.x * p.colp, *pb = pg + (size_t)gridDim.x * p.colp;
    if (WARP) {
#pragma unroll
        for (int which = 0; which < 2; which++) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < VPT; u++) {
                float4 *s = (float4 *)(cols_smem + warp * (VPT * 256) + (t + u * 32) * 8);
                float (&a)[8] = which ? ab[u] : ag[u];
                s[0] = make_float4(a[0], a[1], a[2], a[3]);
                s[1] = make_float4(a[4], a[5], a[6], a[7]);
            }
            __syncthreads();
            for (int c = threadIdx.x; c < p.cols; c += 256) {
                float s = cols_smem[c];
#pragma unroll
                for (int w = 1; w < 8; w++) s += cols_smem[w * (VPT * 256) + c];
                (which ? pb : pg)[c] = s;
            }
        }
    } else {
#pragma unroll
        for (int u = 0; u < VPT; u++) {
            const int col = (t + u * T) * 8;
            if (col < p.cols) {                    // colp is a multiple of 8: a started vector is whole
                float4 *s = (float4 *)(pg + col), *b = (float4 *)(pb + col);
                s[0] = make_float4(ag[u][0], ag[u][1], ag[u][2], ag[u][3]);
                s[1] = make_float4(ag[u][4], ag[u][5], ag[u][6], ag[u][7]);
                b[0] = make_float4(ab[u][0], ab[u][1], ab[u][2], ab[u][3]);
                b[1] = make_float4(ab[u][4], ab[u][5], ab[u][6], ab[u][7]);
            }
        }
    }
}

// Rows too long for the registers: dx row by row (the second pass over a row hits L2) ...
template <bool VEC>
__global__ void __launch_bounds__(1024) k_ln_bwd_long(const LnBwd p)
{
    pdl_trigger();
    pdl_wait();
    __shared__ float2 red[2][32];
    const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
    const int step = blockDim.x * 8;
    int flip = 0;
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x, flip ^= 1) {
        const uint16_t *xr = p.x + (size_t)row * p.ldx, *dr = p.dy + (size_t)row * p.lddy;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float c1 = 0.0f, c2 = 0.0f;
        for (int col = threadIdx.x * 8; col < p.cols; col += step) {
            float x[8], d[8], g[8];
            unpack8(load8<VEC, false>(xr, col, p.cols), x);
            unpack8(load8<VEC, false>(dr, col, p.cols), d);
            unpack8(load8<VEC, false>(p.gamma, col, p.cols), g);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float gy = d[e] * g[e];
                c1 += gy;
                c2 = fmaf(gy, (x[e] - mean) * rstd, c2);
            }
        }
        cta_sum2(c1, c2, red[flip]);
        c1 *= inv_n;
        c2 *= inv_n;
        uint16_t *o = p.dx + (size_t)row * p.lddx;
        for (int col = threadIdx.x * 8; col < p.cols; col += step) {
            float x[8], d[8], g[8];
            unpack8(load8<VEC, false>(xr, col, p.cols), x);
            unpack8(load8<VEC, false>(dr, col, p.cols), d);
            unpack8(load8<VEC, false>(p.gamma, col, p.cols), g);
#pragma unroll
            for (int e = 0; e < 8; e++) d[e] = rstd * (fmaf(d[e], g[e], -c1) - (x[e] - mean) * rstd * c2);
            store8<VEC>(o, col, p.cols, pack8(d));
        }
    }
}
// ... and the column sums of dy*h and dy by a kernel of their own: CTA (i, j) adds the rows j, j + gridDim.y, ...
// of 2048 columns into partial row j.
template <bool VEC>
__global__ void __launch_bounds__(256) k_ln_cols_long(const LnBwd p)
{
    pdl_trigger();
    pdl_wait();
    const int col = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= p.cols) return;
    float ag[8] = {}, ab[8] = {};
    for (int row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const float mean = p.mean[row], rstd = p.rstd[row];
        float x[8], d[8];
        unpack8(load8<VEC, true>(p.x + (size_t)row * p.ldx, col, p.cols), x);
        unpack8(load8<VEC, true>(p.dy + (size_t)row * p.lddy, col, p.cols), d);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            ag[e] = fmaf(d[e], (x[e] - mean) * rstd, ag[e]);
            ab[e] += d[e];
        }
    }
    float *pg = p.parts + (size_t)blockIdx.y * p.colp, *pb = pg + (size_t)gridDim.y * p.colp;
#pragma unroll
    for (int e = 0; e < 8; e++) { pg[col + e] = ag[e]; pb[col + e] = ab[e]; }
}

// dgamma / dbeta: the partial rows added in a fixed order (eight warps take every eighth row, their sums are
// then added in warp order), rounded to FP16 and inspected for inf/NaN.  blockIdx.y: 0 dgamma, 1 dbeta.
__global__ void __launch_bounds__(256) k_ln_param_grad(const float *__restrict__ parts, int nparts, int cols, int colp,
                                                       uint16_t *__restrict__ dgamma, uint16_t *__restrict__ dbeta,
                                                       uint32_t *nonfinite_flag)
{
    pdl_trigger();
    pdl_wait();
    __shared__ float sh[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const float *src = parts + (size_t)blockIdx.y * nparts * colp;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 4
        for (int r = warp; r < nparts; r += 8) s += src[(size_t)r * colp + col];
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0) {
        bool bad = false;
        if (col < cols) {
            s = sh[0][lane];
#pragma unroll
            for (int w = 1; w < 8; w++) s += sh[w][lane];
            const uint32_t h = (uint32_t)__half_as_ushort(__float2half_rn(s));
            bad = half_bits_nonfinite(h);
            (blockIdx.y ? dbeta : dgamma)[col] = (uint16_t)h;
        }
        if (nonfinite_flag && __any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(nonfinite_flag, 1u);
    }
}

constexpr int kLnMaxParts = 296;      // partial rows of the column sums: at most two CTAs on each of the 148 SMs

constexpr int kLnMaxCols = 1 << 30;   // column indexes stay far inside 32 bits

int ln_colp(int cols) { return (cols + 7) / 8 * 8; }
int ln_parts(int rows) { return rows < kLnMaxParts ? rows : kLnMaxParts; }

template <int VPT, bool WARP, int MAXT>
cudaError_t run_fwd(const LnFwd &p, bool vec, int grid, int threads, cudaStream_t st)
{
    if (vec) MPT_LAUNCH((k_ln_fwd<VPT, true, WARP, MAXT>), dim3((unsigned)grid), dim3((unsigned)threads), 0, st, p);
    else MPT_LAUNCH((k_ln_fwd<VPT, false, WARP, MAXT>), dim3((unsigned)grid), dim3((unsigned)threads), 0, st, p);
    return cudaSuccess;
}

template <int VPT, bool WARP>
cudaError_t run_bwd(const LnBwd &p, bool vec, int grid, int threads, cudaStream_t st)
{
    const size_t smem = WARP ? (size_t)8 * VPT * 256 * sizeof(float) : 0;
    if (vec) MPT_LAUNCH((k_ln_bwd<VPT, true, WARP>), dim3((unsigned)grid), dim3((unsigned)threads), smem, st, p);
    else MPT_LAUNCH((k_ln_bwd<VPT, false, WARP>), dim3((unsigned)grid), dim3((unsigned)threads), smem, st, p);
    return cudaSuccess;
}

cudaError_t launch_ln_fwd(const LnFwd &p, cudaStream_t st)
{
    const uintptr_t bits = (uintptr_t)p.x | (uintptr_t)p.y | (uintptr_t)p.gamma | (uintptr_t)p.beta;
    const bool vec = (bits & 15) == 0 && ((p.ldx | p.ldy) & 7) == 0;
    const int c8 = (p.cols + 7) / 8;
    if (c8 <= 128) {
        // a warp per row; few rows are spread over the SMs, one warp to a CTA
        int warps = (p.rows + 147) / 148;
        warps = warps < 1 ? 1 : (warps > 8 ? 8 : warps);
        const long ctas = ((long)p.rows + warps - 1) / warps;
        const int grid = (int)(ctas < 148 * 8 ? ctas : 148 * 8);
        if (c8 <= 32) return run_fwd<1, true, 256>(p, vec, grid, warps * 32, st);
        if (c8 <= 64) return run_fwd<2, true, 256>(p, vec, grid, warps * 32, st);
        return run_fwd<4, true, 256>(p, vec, grid, warps * 32, st);
    }
    if (c8 <= 4 * 1024) {
        const int threads = ((c8 + 3) / 4 + 31) / 32 * 32;
        const int per_sm = threads <= 384 ? (1536 / threads < 16 ? 1536 / threads : 16) : 1;
        const int grid = p.rows < 148 * per_sm ? p.rows : 148 * per_sm;
        return threads <= 384 ? run_fwd<4, false, 384>(p, vec, grid, threads, st) : run_fwd<4, false, 1024>(p, vec, grid, threads, st);
    }
    const int grid = p.rows < 296 ? p.rows : 296;
    if (vec) MPT_LAUNCH(k_ln_fwd_long<true>, dim3((unsigned)grid), dim3(1024), 0, st, p);
    else MPT_LAUNCH(k_ln_fwd_long<false>, dim3((unsigned)grid), dim3(1024), 0, st, p);
    return cudaSuccess;
}

cudaError_t launch_ln_bwd(const LnBwd &p, uint16_t *dgamma, uint16_t *dbeta, uint32_t *nonfinite_flag, cudaStream_t st)
{
    const uintptr_t bits = (uintptr_t)p.x | (uintptr_t)p.dy | (uintptr_t)p.dx | (uintptr_t)p.gamma;
    const bool vec = (bits & 15) == 0 && ((p.ldx | p.lddy | p.lddx) & 7) == 0;
    const int c8 = (p.cols + 7) / 8;
    int nparts = 0;
    cudaError_t e = cudaSuccess;
    if (p.rows > 0 && c8 <= 128) {
        const int ctas = (p.rows + 7) / 8;
        nparts = ctas < kLnMaxParts ? ctas : kLnMaxParts;
        if (c8 <= 32) e = run_bwd<1, true>(p, vec, nparts, 256, st);
        else if (c8 <= 64) e = run_bwd<2, true>(p, vec, nparts, 256, st);
        else e = run_bwd<4, true>(p, vec, nparts, 256, st);
    } else if (p.rows > 0 && c8 <= 2 * 768) {
        const int threads = ((c8 + 1) / 2 + 31) / 32 * 32;
        const int most = threads <= 384 ? 296 : 148;
        nparts = p.rows < most ? p.rows : most;
        e = run_bwd<2, false>(p, vec, nparts, threads, st);
    } else if (p.rows > 0) {
        const int grid = p.rows < 296 ? p.rows : 296;
        if (vec) MPT_LAUNCH(k_ln_bwd_long<true>, dim3((unsigned)grid), dim3(1024), 0, st, p);
        else MPT_LAUNCH(k_ln_bwd_long<false>, dim3((unsigned)grid), dim3(1024), 0, st, p);
        nparts = p.rows < 128 ? p.rows : 128;
        const dim3 cgrid((unsigned)((c8 + 255) / 256), (unsigned)nparts);
        if (vec) MPT_LAUNCH(k_ln_cols_long<true>, cgrid, dim3(256), 0, st, p);
        else MPT_LAUNCH(k_ln_cols_long<false>, cgrid, dim3(256), 0, st, p);
    }
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((p.cols + 31) / 32), dbeta ? 2u : 1u);
    MPT_LAUNCH(k_ln_param_grad, grid, dim3(256), 0, st, (const float *)p.parts, nparts, p.cols, p.colp, dgamma, dbeta, nonfinite_flag);
    return cudaSuccess;
}

}  // namespace
}  // namespace mpt

using namespace mpt;

extern "C" {

int mpt_layernorm_forward(int rows, int cols, const uint16_t *x_dev, int ldx, const uint16_t *gamma16_dev,
                          const uint16_t *beta16_dev, float eps, uint16_t *y_dev, int ldy, float *mean_dev, float *rstd_dev,
                          void *cuda_stream)
{
    if (!x_dev || !gamma16_dev || !y_dev || x_dev == y_dev) return MPT_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || !isfinite(eps)) return MPT_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || cols > kLnMaxCols || ldx < cols || ldy < cols) return MPT_ERR_SHAPE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) return MPT_OK;
    const LnFwd p = {rows, cols, x_dev, (size_t)ldx, gamma16_dev, beta16_dev, eps, y_dev, (size_t)ldy, mean_dev, rstd_dev};
    return launch_ln_fwd(p, st) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

int mpt_layernorm_workspace_bytes(int rows, int cols, size_t *bytes_out)
{
    if (!bytes_out) return MPT_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || cols > kLnMaxCols) return MPT_ERR_SHAPE;
    *bytes_out = (size_t)2 * (size_t)(ln_parts(rows) > 0 ? ln_parts(rows) : 1) * (size_t)ln_colp(cols) * sizeof(float);
    return MPT_OK;
}

int mpt_layernorm_backward(int rows, int cols, const uint16_t *dy_dev, int lddy, const uint16_t *x_dev, int ldx,
                           const uint16_t *gamma16_dev, const float *mean_dev, const float *rstd_dev, uint16_t *dx_dev, int lddx,
                           uint16_t *dgamma16_dev, uint16_t *dbeta16_dev, uint32_t *nonfinite_flag_dev, void *workspace_dev,
                           size_t workspace_bytes, void *cuda_stream)
{
    if (!dy_dev || !x_dev || !gamma16_dev || !mean_dev || !rstd_dev || !dx_dev || !dgamma16_dev || !workspace_dev)
        return MPT_ERR_INVALID_ARG;
    if (dx_dev == dy_dev || dx_dev == x_dev) return MPT_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || cols > kLnMaxCols || lddy < cols || ldx < cols || lddx < cols) return MPT_ERR_SHAPE;
    size_t need = 0;
    mpt_layernorm_workspace_bytes(rows, cols, &need);
    if (workspace_bytes < need || ((uintptr_t)workspace_dev & 15) != 0) return MPT_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const LnBwd p = {rows, cols, dy_dev, (size_t)lddy, x_dev, (size_t)ldx, gamma16_dev, mean_dev, rstd_dev, dx_dev, (size_t)lddx,
                     (float *)workspace_dev, ln_colp(cols)};
    return launch_ln_bwd(p, dgamma16_dev, dbeta16_dev, nonfinite_flag_dev, st) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

}  // extern "C"
