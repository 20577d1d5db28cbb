// Linear layer over a large vocabulary fused with the softmax cross-entropy of its outputs (paper sections 3.2,
// 3.3: FP16 operands, FP32 sums and softmax arithmetic, gradient multiplied by S / N before it is rounded).  The logits are
// neither rounded nor stored; for the gradients a block of rows keeps FP16 exponentials of them:
//
//   z = x . W^T in FP32 ;  loss_i = log sum_v exp(z_iv) - z_i,y(i)
//   dx = rn16(S / N * sum_v (p_iv - [v = y(i)]) W_v) ;  dW_v = rn16(S / N * sum_i (p_iv - [v = y(i)]) x_i)
//
// Work: 2 N V H for the losses, 6 N V H with both gradients; bound: the tensor pipe (for few rows: reading W and
// writing dW).  The rows go through in blocks of R; per block
//   1  the logits product with a softmax epilogue: the accumulators of 128 classes of a row become FP16
//      exponentials relative to their own maximum (CeEpi), with their FP32 sum, and the label's FP32 logit
//   2  k_ce_combine: the row's whole sum, and the row's loss (and x without the ignored rows, for step 5)
//   3  k_ce_rescale: exponentials -> 2^14 (p - [v = y]) in place (2 and 3 in one, k_ce_finish, for a few short rows)
//   4  dx = product of those with W, 5 dW = product of their transpose with x, both with the factor S / N * 2^-14
//      in the epilogue (up to 128 rows: dW by k_ce_dw)
// Keeping the exponentials costs 2 bytes a logit of a block and step 3 (4 bytes a logit through HBM: 143/H of the
// products' time), computing them a second time would cost a fourth product (1/3).  FP16 keeps them, and p, to
// 2^-11 of the value each (together 2.8e-4 on average, which is what dx and dW are off) whatever S and N: the scale 2^14 leaves 2^-38 of a group's largest term (resp. of 1) above
// zero, where p * S / N in FP16 would lose p below 2^-24 N / S.  Over several row blocks dW is summed in FP32.
// Measured: 4096 x 32000 x 12288 7.4-8.5 ms (1.13-1.3 PFLOP/s, under the power cap), 1024 x 793471 x 1024 5.4-6.3 ms,
// losses alone 2500 x 50001 x 2048 0.41 ms (1.25 PFLOP/s), 64 x 1000 x 512 20 us.
#include <math.h>

#include "mpt_common.cuh"

namespace mpt {
namespace {

constexpr int kGroup = 128;           // classes of one softmax group (CeEpi)
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kDefaultRows = 4096;    // rows of a block when the caller does not choose
constexpr int kMaxSize = 1 << 30;     // N and H: what is added to their indexes stays inside 32 bits
constexpr int kMaxRows = 65536;       // largest block: CTAs of a pass over it stay inside 31 bits

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// (m, s) pairs, s e^m each, added.  m = -inf: no terms (s = 0), or only NaN, which stays.
__device__ __forceinline__ void join(float &m1, float &s1, float m2, float s2)
{
    const float mn = fmaxf(m1, m2);
    s1 = (m1 == mn ? s1 : s1 * ex2((m1 - mn) * kLog2e)) + (m2 == mn ? s2 : s2 * ex2((m2 - mn) * kLog2e));
    m1 = mn;
}
// The loss of a row with the sum 2^-14 s e^m and the label's logit z: the logits' difference first, whatever their size.
__device__ __forceinline__ float row_loss_of(float m, float s, float z)
{
    return (float)((log2((double)s) - 14.0) * 0.69314718055994530942 + ((double)m - (double)z));
}
// Eight exponentials of a row, the first of class col, to 2^14 (p - [v = y]).
__device__ __forceinline__ uint4 rescale8(const uint4 v, float f, int y, int col, float z, float2 sum)
{
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const float2 t = __half22float2(*(const __half2 *)&x[q]);
        const __half2 h = __floats2half2_rn(t.x * f, t.y * f);
        w[q] = *(const uint32_t *)&h;
    }
    if (y - col >= 0 && y - col < 8) {           // the label's element from its FP32 logit
        const float p = ex2(fmaf(z - sum.x, kLog2e, 14.0f)) * __fdiv_rn(1.0f, sum.y);
        const uint32_t h = (uint32_t)__half_as_ushort(__float2half_rn((p - 1.0f) * 16384.0f));
#pragma unroll
        for (int q = 0; q < 4; q++) {
            if (((y - col) >> 1) == q) w[q] = ((y - col) & 1) ? ((w[q] & 0x0000FFFFu) | (h << 16)) : ((w[q] & 0xFFFF0000u) | h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Row sums from the group sums: sum_g s_g e^(m_g) = y e^x as the pair (x, y), x the largest m_g, and the row's
// loss.  The pair stays apart: the logarithm of large logits' sum as one FP32 number would not resolve p.  Four rows per CTA (a
// 32-byte sector of `stats` holds one group of four rows), THREADS / 4 threads a row (few rows of many groups: 256, else
// the chain of loads is long: 3 x 136611 10 us); fixed order.
// xs (null: not wanted) receives x with the rows of ignored labels as zeros: what a padding row holds, NaN
// perhaps, must not meet its zero gradient in dW's product.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_ce_combine(const float2 *__restrict__ stats, int R, int V, int groups,
                                                    const int32_t *__restrict__ labels, const float *__restrict__ zlabel,
                                                    float2 *__restrict__ rowsum, float *__restrict__ row_loss, uint32_t *bad_labels,
                                                    const uint16_t *__restrict__ x, int ldx, int H, uint16_t *__restrict__ xs,
                                                    float *__restrict__ factor)
{
    pdl_trigger();
    pdl_wait();
    constexpr int PER_ROW = THREADS / 4;
    __shared__ float2 red[THREADS / 32][4];
    if (xs) {
        const int xrow = blockIdx.x * 4 + threadIdx.x / PER_ROW;
        if (xrow < R) {
            const bool live = (unsigned)labels[xrow] < (unsigned)V;
            const uint4 *src = (const uint4 *)(x + (size_t)xrow * ldx);
            uint4 *dst = (uint4 *)(xs + (size_t)xrow * H);
            for (int i = threadIdx.x % PER_ROW; i < H / 8; i += PER_ROW) dst[i] = live ? src[i] : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    const int r = threadIdx.x & 3, row = blockIdx.x * 4 + r;
    float m = -INFINITY, s = 0.0f;
    if (row < R) {
        for (int g = threadIdx.x >> 2; g < groups; g += PER_ROW) {
            const float2 t = stats[(size_t)g * R + row];
            join(m, s, t.y, t.x);
        }
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
        const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, s, o);
        join(m, s, m2, s2);
    }
    if ((threadIdx.x & 31) < 4) red[threadIdx.x >> 5][r] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x < 4 && row < R) {
        m = red[0][r].x;
        s = red[0][r].y;
#pragma unroll
        for (int w = 1; w < THREADS / 32; w++) join(m, s, red[w][r].x, red[w][r].y);
        const int y = labels[row];
        const bool good = y >= 0 && y < V;
        rowsum[row] = make_float2(m, s);
        if (good) row_loss[row] = row_loss_of(m, s, zlabel[row]);
        else row_loss[row] = 0.0f;                      // contributes neither loss nor gradient
        if (!good && bad_labels) atomicAdd(bad_labels, 1u);
        red[0][r] = make_float2(m, good ? s : INFINITY);     // an ignored row's factors are zeros
    }
    if (!factor) return;
    // what turns a group's exponentials into 2^14 p, a row's groups next to each other (the statistics come from L2 now)
    __syncthreads();
    m = red[0][r].x;
    s = red[0][r].y;
    if (row < R) {
        const float inv = __fdiv_rn(1.0f, s);
        float *f = factor + (size_t)row * groups;
        for (int g = threadIdx.x >> 2; g < groups; g += PER_ROW) f[g] = s == INFINITY ? 0.0f : ex2(fmaf(stats[(size_t)g * R + row].y - m, kLog2e, 14.0f)) * inv;
    }
}

// e -> 2^14 (p - [v = y]) in place, and the mean loss.  A CTA takes 16384 neighbouring columns of one row (32 KB), 16 bytes a lane and
// load, all loads ahead of the first use.
__global__ void __launch_bounds__(256) k_ce_rescale(uint16_t *__restrict__ e16, int ld, const float *__restrict__ factor, int groups,
                                                    int V, const int32_t *__restrict__ labels, const float *__restrict__ zlabel,
                                                    const float2 *__restrict__ rowsum, const float *__restrict__ row_loss, int N,
                                                    float *__restrict__ loss, int chunks)
{
    pdl_trigger();
    pdl_wait();
    // one CTA more than there is work for, after the last block of rows: the mean loss
    if (loss && blockIdx.x == gridDim.x - 1) {
        __shared__ double red[256];
        mean_of_rows(row_loss, N, loss, red);
        return;
    }
    const int row = (int)(blockIdx.x / (unsigned)chunks), col0 = (int)(blockIdx.x % (unsigned)chunks) * 16384 + threadIdx.x * 8;
    uint16_t *er = e16 + (size_t)row * ld;
    const float *fr = factor + (size_t)row * groups;
    uint4 v[8];
    float f[8];
#pragma unroll
    for (int u = 0; u < 8; u++) {
        const int col = col0 + u * 2048;
        if (col < ld) {
            v[u] = __ldcs((const uint4 *)(er + col));
            f[u] = __ldg(fr + col / kGroup);
        }
    }
    const int y = labels[row];           // asked for last: nothing waits for it before the row's loads are out
    const bool good = y >= 0 && y < V;
#pragma unroll
    for (int u = 0; u < 8; u++) {
        const int col = col0 + u * 2048;
        if (col >= ld) continue;
        const bool label = good && y - col >= 0 && y - col < 8;
        *(uint4 *)(er + col) = good ? rescale8(v[u], f[u], y, col, label ? zlabel[row] : 0.0f, label ? rowsum[row] : make_float2(0.0f, 1.0f))
                                    : make_uint4(0u, 0u, 0u, 0u);
    }
}

// Both passes in one for a few rows of at most 128 groups: a CTA takes a whole row (64 x 1000 x 512: 22.7 us with five launches,
// 20.1 with four).
constexpr int kSmallGroups = 128;
__global__ void __launch_bounds__(256) k_ce_finish(uint16_t *__restrict__ e16, int ld, const float2 *__restrict__ stats, int R, int V, int groups,
                                                   const int32_t *__restrict__ labels, const float *__restrict__ zlabel,
                                                   float *__restrict__ row_loss, uint32_t *bad_labels, const uint16_t *__restrict__ x, int ldx,
                                                   int H, uint16_t *__restrict__ xs)
{
    pdl_trigger();
    pdl_wait();
    __shared__ float2 red[4];
    __shared__ float factor[kSmallGroups];
    const int row = blockIdx.x, t = threadIdx.x, y = labels[row];
    const bool good = y >= 0 && y < V;
    uint16_t *er = e16 + (size_t)row * ld;
    uint4 v[8];
#pragma unroll
    for (int u = 0; u < 8; u++)
        if (t * 8 + u * 2048 < ld) v[u] = __ldcs((const uint4 *)(er + t * 8 + u * 2048));
    const uint4 *src = (const uint4 *)(x + (size_t)row * ldx);
    uint4 *dst = (uint4 *)(xs + (size_t)row * H);
    for (int i = t; i < H / 8; i += 256) dst[i] = good ? src[i] : make_uint4(0u, 0u, 0u, 0u);
    float m = -INFINITY, s = 0.0f;
    if (t < groups) {
        const float2 st = stats[(size_t)t * R + row];
        s = st.x;
        m = st.y;
    }
    const float group_m = m;
    if (t < kSmallGroups) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, s, o);
            join(m, s, m2, s2);
        }
        if ((t & 31) == 0) red[t >> 5] = make_float2(m, s);
    }
    __syncthreads();
    m = red[0].x;
    s = red[0].y;
#pragma unroll
    for (int w = 1; w < kSmallGroups / 32; w++) join(m, s, red[w].x, red[w].y);
    if (t < groups) factor[t] = ex2(fmaf(group_m - m, kLog2e, 14.0f)) * __fdiv_rn(1.0f, s);
    if (t == 0) {
        row_loss[row] = good ? row_loss_of(m, s, zlabel[row]) : 0.0f;
        if (!good && bad_labels) atomicAdd(bad_labels, 1u);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 8; u++) {
        const int col = t * 8 + u * 2048;
        if (col >= ld) continue;
        *(uint4 *)(er + col) = good ? rescale8(v[u], factor[col / kGroup], y, col, zlabel[row], make_float2(m, s)) : make_uint4(0u, 0u, 0u, 0u);
    }
}

// dW of few rows, d^T x with a contraction over at most 128 rows: writing dW is what takes time, and the tcgen05 kernels, whose
// epilogues reach 1.5 to 2.2 TB/s, are bound by that.  Here the sums are in registers as they are made (warp-wide mma with FP32
// sums), pass through shared memory and leave in 16-byte stores: 4.9 TB/s for 3 rows of 136611 x 2304, where the stores are the
// bound, 1.8 TB/s for 96 rows, where mma.sync and the waits for d are (tensor pipe 46 %, one buffer of d).
// Whole calls in us, the product kernel and this one: 3 rows, 136611 x 2304 643 and 390; 64 rows, 50000 x 2048 229 and 187; 82 rows,
// 8491 x 9776 225 and 200; 128 rows, 32000 x 4096 294 and 276, 136611 x 2304 661 and 604, 50000 x 1024 156 and 156.  For few features
// and 65 to 128 rows the product kernel would be the faster: 20000 x 512 63 and 65, 793471 x 1024 1435 and 1605.
// A CTA keeps x for 128 features and goes through the words 128 at a time, up to 64 rows the next 128 words' d on the way
// meanwhile.
constexpr int kDwRows = 128, kDwTile = 128, kDwPitch = kDwTile + 8;      // pitch: 8 rows of a matrix load lie in different banks
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
constexpr __host__ __device__ int dw_buffers(int steps) { return steps < 8 ? 2 : 1; }      // of d: two CTAs fit on an SM
constexpr uint32_t dw_smem(int steps) { return (uint32_t)((1 + dw_buffers(steps)) * steps * 16 + 8 * 16) * kDwPitch * 2u; }
template <int STEPS>
__global__ void __launch_bounds__(256) k_ce_dw(const uint16_t *__restrict__ d, int ldd, const uint16_t *__restrict__ x, int H, int R, int V,
                                               float alpha, uint16_t *__restrict__ dW, int lddw, uint32_t *nonfinite_flag, int chunks, int step,
                                               const float *__restrict__ row_loss, float *__restrict__ loss)
{
    extern __shared__ __align__(128) uint8_t smem[];
    constexpr int K = STEPS * 16, BUFFERS = dw_buffers(STEPS);
    uint16_t *xt = (uint16_t *)smem, *dt = xt + K * kDwPitch;                   // x | d | a warp's results
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint16_t *out = dt + BUFFERS * K * kDwPitch + warp * 16 * kDwPitch;
    pdl_trigger();
    pdl_wait();
    if (loss && blockIdx.x == gridDim.x - 1) {       // one CTA more than there is work for: the mean loss
        mean_of_rows(row_loss, R, loss, (double *)smem);
        return;
    }
    // rows of a matrix [R, width] from column c0 on, zeros outside
    auto load = [&](uint16_t *to, const uint16_t *from, int ld, int c0, int width) {
        for (int i = threadIdx.x; i < K * (kDwTile / 8); i += 256) {
            const int row = i / (kDwTile / 8), col = i % (kDwTile / 8) * 8;
            const bool in = row < R && c0 + col < width;
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to + row * kDwPitch + col);
            const uint16_t *src = in ? from + (size_t)row * ld + c0 + col : from;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const int h0 = (int)(blockIdx.x % (unsigned)chunks) * kDwTile, tiles = (V + kDwTile - 1) / kDwTile;
    int tile = (int)(blockIdx.x / (unsigned)chunks), at = 0;
    load(xt, x, H, h0, H);
    if (tile < tiles) load(dt, d, ldd, tile * kDwTile, ldd);
    bool bad = false;
    for (; tile < tiles; tile += step, at ^= BUFFERS - 1) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();                         // this tile is there for all, and all are done with the one before
        if (BUFFERS == 2 && tile + step < tiles) load(dt + (at ^ 1) * K * kDwPitch, d, ldd, (tile + step) * kDwTile, ldd);
        const uint16_t *dd = dt + at * K * kDwPitch;
        const int r = lane & 7, m = lane >> 3;
        float c[kDwTile / 8][4] = {};
#pragma unroll
        for (int k = 0; k < STEPS; k++) {
            uint32_t a[4];
            ldmatrix_x4_trans(a, (uint32_t)__cvta_generic_to_shared(dd + (k * 16 + (m >> 1) * 8 + r) * kDwPitch + warp * 16 + (m & 1) * 8));
#pragma unroll
            for (int n = 0; n < kDwTile / 16; n++) {
                uint32_t b[4];
                ldmatrix_x4_trans(b, (uint32_t)__cvta_generic_to_shared(xt + (k * 16 + (m & 1) * 8 + r) * kDwPitch + n * 16 + (m >> 1) * 8));
                mma_16816(c[2 * n], a, b[0], b[1]);
                mma_16816(c[2 * n + 1], a, b[2], b[3]);
            }
        }
        if (BUFFERS == 1) {
            __syncthreads();                     // all have used d
            if (tile + step < tiles) load(dt, d, ldd, (tile + step) * kDwTile, ldd);
        }
        __syncwarp();                            // the last tile's results have left `out`
#pragma unroll
        for (int n = 0; n < kDwTile / 8; n++) {
            const int col = n * 8 + (lane & 3) * 2, row = lane >> 2;
            *(__half2 *)(out + row * kDwPitch + col) = __floats2half2_rn(c[n][0] * alpha, c[n][1] * alpha);
            *(__half2 *)(out + (row + 8) * kDwPitch + col) = __floats2half2_rn(c[n][2] * alpha, c[n][3] * alpha);
        }
        __syncwarp();
        const int col = (lane & 15) * 8;
        if (h0 + col < H) {
#pragma unroll
            for (int q = 0; q < 8; q++) {
                const int row = q * 2 + (lane >> 4), v = tile * kDwTile + warp * 16 + row;
                const uint4 y = *(const uint4 *)(out + row * kDwPitch + col);
                if (v < V) {
                    bad |= half_bits_nonfinite(y.x) || half_bits_nonfinite(y.x >> 16) || half_bits_nonfinite(y.y) || half_bits_nonfinite(y.y >> 16) ||
                           half_bits_nonfinite(y.z) || half_bits_nonfinite(y.z >> 16) || half_bits_nonfinite(y.w) || half_bits_nonfinite(y.w >> 16);
                    __stcs((uint4 *)(dW + (size_t)v * lddw + h0 + col), y);
                }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (nonfinite_flag && __any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(nonfinite_flag, 1u);
}
template <int STEPS>
cudaError_t run_dw(int R, int V, int H, const uint16_t *d, int ldd, const uint16_t *x, float alpha, uint16_t *dW, int lddw,
                   uint32_t *nonfinite_flag, const float *row_loss, float *loss, cudaStream_t st)
{
    static bool configured[kMaxDevices] = {};
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(k_ce_dw<STEPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dw_smem(STEPS));
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const int chunks = (H + kDwTile - 1) / kDwTile, tiles = (V + kDwTile - 1) / kDwTile;
    // CTAs of neighbouring features work on the same words; about as many CTAs as fit, in whole sets of them, or, where whole
    // sets leave SMs idle, CTAs of eight tiles each
    const int fit = 148 * (int)(227u * 1024u / (dw_smem(STEPS) + 1024u));
    int sets = fit / chunks;
    if (sets * chunks < fit - fit / 8) sets = (tiles + 7) / 8;
    if (sets > tiles) sets = tiles;
    return launch_pdl(k_ce_dw<STEPS>, dim3((unsigned)chunks * (unsigned)sets + (loss ? 1u : 0u)), dim3(256), dw_smem(STEPS), st, d, ldd, x, H, R,
                      V, alpha, dW, lddw, nonfinite_flag, chunks, sets, row_loss, loss);
}
cudaError_t launch_dw(int R, int V, int H, const uint16_t *d, int ldd, const uint16_t *x, float alpha, uint16_t *dW, int lddw,
                      uint32_t *nonfinite_flag, const float *row_loss, float *loss, cudaStream_t st)
{
    if (R <= 16) return run_dw<1>(R, V, H, d, ldd, x, alpha, dW, lddw, nonfinite_flag, row_loss, loss, st);
    if (R <= 32) return run_dw<2>(R, V, H, d, ldd, x, alpha, dW, lddw, nonfinite_flag, row_loss, loss, st);
    if (R <= 64) return run_dw<4>(R, V, H, d, ldd, x, alpha, dW, lddw, nonfinite_flag, row_loss, loss, st);
    return run_dw<8>(R, V, H, d, ldd, x, alpha, dW, lddw, nonfinite_flag, row_loss, loss, st);
}

bool bad_sizes(int N, int V, int H, int row_block)
{
    return N < 0 || N > kMaxSize || V < 1 || V > MPT_LINEAR_CE_MAX_V || H < 8 || H > kMaxSize || H % 8 || row_block < 0 ||
           row_block > kMaxRows || row_block % 256;
}

// Where things are in the workspace (256-byte aligned offsets).
struct Plan {
    int R, blocks;        // rows of a block, number of blocks
    int lde;              // pitch of the exponentials
    int groups;
    int ldacc;
    size_t e16, stats, factor, rowsum, zlabel, xs, splitk, splitk_bytes, dx32, acc32, total;
};

// The split of dx's contraction over the vocabulary: for few rows the product has few tiles and reading W is what
// takes time, so as many SMs as possible have to take part.
constexpr int kDxSplit = 64;

// dx of a few hundred to a few thousand rows: 256x256 tiles that do not fill the 74 CTA pairs, and a contraction of tens
// of thousands.  As many parts of it as fit into one round of units, part by part, so that the tiles of a part walk
// through the same operand panels side by side: 1024 x 1024 with K = 793471 (16 tiles) in 4 parts reads its operands
// once from DRAM; in 9 parts, two rounds and 97 % of the pairs busy, the second round's units start apart and nothing is
// shared any more (7.8 instead of 3.4 GB read, 1.53 ms); two pairs per tile in one cluster leave 57 % of the SMs idle
// (1.82 ms).  A part keeps at least 64 k-blocks, under which the FP32 parts' way through L2 disappears.
// Whatever the kernel, no accumulator sums more than kDxPart terms: the tensor core's FP32 sums lose up to half a step
// at each of their K / 16 additions, always towards zero, which over 793471 terms is 4e-4 of the sum - more than all
// FP16 roundings together.  The parts are added with correct rounding.
constexpr int kDxPart = 32768;

int dx_parts(int V) { return (V + kDxPart - 1) / kDxPart; }

int dx_pair_split(int M, int N, int K)
{
    if (M < 256 || N < 256) return 0;
    const int tiles = ((M + 255) / 256) * ((N + 255) / 256), nkb = (K + 63) / 64;
    int s = tiles <= 37 ? 74 / tiles : 0;
    if (s > 16) s = 16;
    while (s > 1 && nkb / s < 64) s--;
    return s > 1 ? s : 0;
}
// Parts that one pair works off one after the other beside s - 1 others.
int dx_pair_seq(int s, int K) { return (dx_parts(K) + s - 1) / s; }
// dx on the CTA-pair kernel with more tiles than that: one launch per part of the contraction, FP32 sums in between.
bool dx_in_launches(int M, int N, int K) { return dx_parts(K) > 1 && !dx_pair_split(M, N, K) && tc2_gemm_preferred(M, N, K); }

// Scratch of dx's and dW's products besides the FP32 sums.
size_t product_scratch(int op, int M, int N, int K)
{
    if (op == MPT_OP_DGRAD) {
        if (const int s = dx_pair_split(M, N, K)) return (size_t)s * dx_pair_seq(s, K) * M * ((N + 31) / 32 * 32) * sizeof(float);
        if (dx_in_launches(M, N, K)) return 0;
    }
    if (tc4_split_for(M, N, K)) return 0;
    size_t need = 0;
    if (tc2_gemm_preferred(M, N, K)) return tc2_tail_ws_bytes(M, N, K);
    const int least = op == MPT_OP_DGRAD ? dx_parts(K) : 1, most = op == MPT_OP_DGRAD ? (least > kDxSplit ? least : kDxSplit) : 8;
    int bn, split;
    tc_gemm_plan(M, N, K, (size_t)1 << 40, &bn, &split, &need, nullptr, most, least);
    return need;
}

Plan make_plan(int N, int V, int H, bool want_dx, bool want_dW, int row_block)
{
    Plan p = {};
    p.R = row_block > 0 ? row_block : kDefaultRows;
    if (p.R > N) p.R = N > 0 ? N : 1;
    p.blocks = (N + p.R - 1) / p.R;
    p.lde = (V + 7) / 8 * 8;
    p.groups = (V + kGroup - 1) / kGroup;
    p.ldacc = (H + 31) / 32 * 32;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const bool grads = want_dx || want_dW;
    p.e16 = take(grads ? (size_t)p.R * p.lde * 2 : 0);
    p.stats = take((size_t)p.groups * p.R * sizeof(float2));
    p.factor = take(grads ? (size_t)p.groups * p.R * sizeof(float) : 0);
    p.rowsum = take((size_t)p.R * sizeof(float2));
    p.zlabel = take((size_t)p.R * sizeof(float));
    p.xs = take(want_dW ? (size_t)p.R * H * 2 : 0);
    size_t sk = 0, acc = 0;
    if (want_dx) {
        sk = product_scratch(MPT_OP_DGRAD, p.R, H, V);
        if (dx_in_launches(p.R, H, V)) acc = (size_t)p.R * p.ldacc * sizeof(float);
        const int rest = N - (p.blocks - 1) * p.R;          // the last block may be shorter
        if (p.blocks > 1 && rest != p.R) {
            const size_t s2 = product_scratch(MPT_OP_DGRAD, rest, H, V);
            sk = s2 > sk ? s2 : sk;
            if (dx_in_launches(rest, H, V) && acc == 0) acc = (size_t)rest * p.ldacc * sizeof(float);
        }
    }
    if (want_dW && p.blocks == 1 && p.R > kDwRows) {
        const size_t s2 = product_scratch(MPT_OP_WGRAD, V, H, p.R);
        sk = s2 > sk ? s2 : sk;
    }
    p.splitk_bytes = sk;
    p.splitk = take(sk);
    p.dx32 = take(acc);
    p.acc32 = take(want_dW && p.blocks > 1 ? (size_t)V * p.ldacc * sizeof(float) : 0);
    p.total = at;
    return p;
}

// One of the products, on the kernel the plain entry point would choose.
cudaError_t product(int op, int M, int N, int K, const uint16_t *A, int lda, const uint16_t *B, int ldb, uint16_t *C, int ldc,
                    const ProductExtra &x, uint32_t *nonfinite, uint32_t *status, void *ws, size_t ws_bytes, cudaStream_t st)
{
    if (x.ce) {
        // 256-row tiles only where there are more than 128 rows and enough tiles for the CTA pairs
        const long tiles = (long)((M + 255) / 256) * ((N + 255) / 256);
        if (M > 128 && N >= 256 && tiles > 74)
            return launch_gemm_tc2(op, M, N, K, A, lda, B, ldb, C, ldc, false, nullptr, 0, nonfinite, status, st, nullptr, nullptr, 0, &x);
        return launch_gemm_tc(op, M, N, K, A, lda, B, ldb, C, ldc, false, nullptr, 0, nonfinite, status, st, nullptr, 0, nullptr, &x);
    }
    if (op == MPT_OP_DGRAD) {
        if (const int s = dx_pair_split(M, N, K)) {
            ProductExtra y = x;
            y.split = s;
            y.split_seq = dx_pair_seq(s, K);
            return launch_gemm_tc2(op, M, N, K, A, lda, B, ldb, C, ldc, false, nullptr, 0, nonfinite, status, st, nullptr, ws, ws_bytes, &y);
        }
    }
    if (!x.acc32) {
        if (const int split = tc4_split_for(M, N, K))
            return launch_gemm_tc4(op, M, N, K, A, lda, B, ldb, C, ldc, false, nullptr, 0, nonfinite, status, st, split, x.alpha);
    }
    if (tc2_gemm_preferred(M, N, K))
        return launch_gemm_tc2(op, M, N, K, A, lda, B, ldb, C, ldc, false, nullptr, 0, nonfinite, status, st, nullptr, ws, ws_bytes, &x);
    return launch_gemm_tc(op, M, N, K, A, lda, B, ldb, C, ldc, false, nullptr, 0, nonfinite, status, st, (float *)ws, ws_bytes, nullptr, &x);
}

}  // namespace
}  // namespace mpt

using namespace mpt;

extern "C" {

int mpt_linear_ce_workspace_bytes(int N, int V, int H, int want_dx, int want_dW, int row_block, size_t *bytes_out)
{
    if (!bytes_out) return MPT_ERR_INVALID_ARG;
    if (bad_sizes(N, V, H, row_block)) return MPT_ERR_SHAPE;
    *bytes_out = make_plan(N, V, H, want_dx != 0, want_dW != 0, row_block).total;
    return MPT_OK;
}

int mpt_linear_ce(int N, int V, int H, const uint16_t *x_dev, int ldx, const uint16_t *W_dev, int ldw, const int32_t *labels_dev,
                  float S, int row_block, uint16_t *dx_dev, int lddx, uint16_t *dW_dev, int lddw, float *row_loss_dev,
                  float *loss_dev, uint32_t *bad_labels_dev, uint32_t *nonfinite_flag_dev, uint32_t *status_dev,
                  void *workspace_dev, size_t workspace_bytes, void *cuda_stream)
{
    // an empty batch has no addresses: what holds rows may be null then
    if (!W_dev || !loss_dev || !workspace_dev || (N != 0 && (!x_dev || !labels_dev || !row_loss_dev || dx_dev == x_dev))) return MPT_ERR_INVALID_ARG;
    if (((dx_dev || dW_dev) && !isfinite(S)) || dW_dev == W_dev) return MPT_ERR_INVALID_ARG;
    if (bad_sizes(N, V, H, row_block)) return MPT_ERR_SHAPE;
    if (ldx < H || ldw < H || (dx_dev && lddx < H) || (dW_dev && lddw < H)) return MPT_ERR_SHAPE;
    const uintptr_t bits = (uintptr_t)x_dev | (uintptr_t)W_dev | (uintptr_t)dx_dev | (uintptr_t)dW_dev;
    if ((bits & 15) || ldx % 8 || ldw % 8 || (dx_dev && lddx % 8) || (dW_dev && lddw % 8)) return MPT_ERR_SHAPE;
    const Plan p = make_plan(N, V, H, dx_dev != nullptr, dW_dev != nullptr, row_block);
    if (workspace_bytes < p.total || ((uintptr_t)workspace_dev & 255)) return MPT_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    uint8_t *ws = (uint8_t *)workspace_dev;
    uint16_t *e16 = (uint16_t *)(ws + p.e16);
    float2 *stats = (float2 *)(ws + p.stats);
    float2 *rowsum = (float2 *)(ws + p.rowsum);
    float *zlabel = (float *)(ws + p.zlabel);
    uint16_t *xs = dW_dev ? (uint16_t *)(ws + p.xs) : nullptr;
    const bool grads = dx_dev || dW_dev;
    float *factor = grads ? (float *)(ws + p.factor) : nullptr;
    cudaError_t e = cudaSuccess;
    if (bad_labels_dev) e = cudaMemsetAsync(bad_labels_dev, 0, sizeof(uint32_t), st);
    if (e == cudaSuccess && N == 0 && dW_dev) e = cudaMemset2DAsync(dW_dev, (size_t)lddw * 2, 0, (size_t)H * 2, (size_t)V, st);
    const float alpha = S / (float)N * (1.0f / 16384.0f);
    for (int b = 0; b < p.blocks && e == cudaSuccess; b++) {
        const int r0 = b * p.R, R = N - r0 < p.R ? N - r0 : p.R;
        const uint16_t *x = x_dev + (size_t)r0 * ldx;
        const int32_t *labels = labels_dev + r0;
        const CeEpi ce = {labels, stats, zlabel, grads ? 1 : 0};
        ProductExtra xl, xd, xw;
        xl.ce = &ce;
        e = product(MPT_OP_FWD, R, V, H, x, ldx, W_dev, ldw, grads ? e16 : nullptr, p.lde, xl, nullptr, status_dev, nullptr, 0, st);
        if (e != cudaSuccess) break;
        // the mean loss comes with the rescale pass or, for few rows of few groups, with dW
        const bool small = dW_dev && p.blocks == 1 && R <= kDwRows && p.groups <= kSmallGroups;
        if (small) {
            e = launch_pdl(k_ce_finish, dim3((unsigned)R), dim3(256), 0, st, e16, p.lde, (const float2 *)stats, R, V, p.groups, labels,
                           (const float *)zlabel, row_loss_dev, bad_labels_dev, x, ldx, H, xs);
        } else {
            const bool wide = p.groups >= 256 && R <= 4 * 148;
            e = launch_pdl(wide ? k_ce_combine<1024> : k_ce_combine<256>, dim3((unsigned)((R + 3) / 4)), dim3(wide ? 1024 : 256), 0, st,
                           (const float2 *)stats, R, V, p.groups, labels, (const float *)zlabel, rowsum, row_loss_dev + r0, bad_labels_dev, x, ldx, H, xs, factor);
            if (e != cudaSuccess || !grads) continue;
            const bool last = b + 1 == p.blocks;
            const int chunks = (p.lde + 16383) / 16384;
            e = launch_pdl(k_ce_rescale, dim3((unsigned)chunks * (unsigned)R + (unsigned)last), dim3(256), 0, st, e16, p.lde,
                           (const float *)factor, p.groups, V, labels, (const float *)zlabel, (const float2 *)rowsum,
                           (const float *)row_loss_dev, N, last ? loss_dev : (float *)nullptr, chunks);
        }
        if (e == cudaSuccess && dx_dev) {
            xd.alpha = alpha;
            uint16_t *dx = dx_dev + (size_t)r0 * lddx;
            const int parts = dx_parts(V);
            if (dx_in_launches(R, H, V)) {
                xd.acc32 = (float *)(ws + p.dx32);
                xd.ldacc = p.ldacc;
                const int step = ((V + parts - 1) / parts + 7) / 8 * 8;        // operands stay 16-byte aligned
                for (int v = 0; v < V && e == cudaSuccess; v += step) {
                    xd.acc_add = v > 0;
                    xd.acc_store = v + step < V;
                    e = launch_gemm_tc2(MPT_OP_DGRAD, R, H, V - v < step ? V - v : step, e16 + v, p.lde, W_dev + (size_t)v * ldw, ldw, dx,
                                        lddx, false, nullptr, 0, nullptr, status_dev, st, nullptr, nullptr, 0, &xd);
                }
            } else {
                xd.min_split = parts;
                xd.max_split = parts > kDxSplit ? parts : kDxSplit;
                e = product(MPT_OP_DGRAD, R, H, V, e16, p.lde, W_dev, ldw, dx, lddx, xd, nullptr, status_dev, ws + p.splitk,
                            p.splitk_bytes, st);
            }
        }
        if (e == cudaSuccess && dW_dev) {
            xw.alpha = alpha;
            if (p.blocks > 1) {
                xw.acc32 = (float *)(ws + p.acc32);
                xw.ldacc = p.ldacc;
                xw.acc_add = b > 0;
                xw.acc_store = b + 1 < p.blocks;
            }
            if (p.blocks == 1 && R <= kDwRows) 
                e = launch_dw(R, V, H, e16, p.lde, xs, alpha, dW_dev, lddw, nonfinite_flag_dev, row_loss_dev, small ? loss_dev : nullptr, st);
            else e = product(MPT_OP_WGRAD, V, H, R, e16, p.lde, xs, H, dW_dev, lddw, xw, xw.acc_store ? nullptr : nonfinite_flag_dev,
                        status_dev, ws + p.splitk, p.splitk_bytes, st);
        }
    }
    if (e == cudaSuccess && (!grads || N == 0)) e = launch_loss_mean(row_loss_dev, N, loss_dev, st);
    return e == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

}  // extern "C"
