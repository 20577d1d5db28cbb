// Layer normalisation over the features of a row, forward and backward (point-wise work and reductions in
// FP32 on FP16 data: paper section 3.3), and the reduction of the scale and shift vectors' gradients.
//
//   forward   mean = sum x / n ;  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps) ;  h = (x - mean) * rstd
//             y = rn16(h * gamma + beta)
//   backward  g = dy * gamma ;  c1 = sum g / n ;  c2 = sum g*h / n ;  dx = rn16(rstd * (g - c1 - h * c2))
//             dgamma = rn16(sum over rows of dy * h) ;  dbeta = rn16(sum over rows of dy)
//
// Bound: HBM.  Forward reads x and writes y (4 bytes an element), backward reads dy and x and writes dx (6).
// Up to 1024 features belong to one warp, longer rows (up to 16384 features, backward 12288) to as many warps of a CTA as
// that takes; a warp keeps its features for all rows it works on, so the column sums of the parameter gradients stay in its
// registers.  Every warp is a pipeline of its own: its part of the next rows arrives in shared memory by bulk copies while
// the present row is in registers (with all SMs' copies queued at the memory a load takes a few microseconds, longer than a
// row), results leave by 16-byte stores.  Scale and shift are in shared memory.  The warps of a long row exchange their sums
// through shared memory and a named barrier.  The variance is a second pass over the registers (sum of squared deviations),
// not a difference of sums.
// The backward pass adds dy*h and dy into per-lane FP32 column sums, leaves one partial row of them per CTA in the
// workspace and adds those in a second kernel in a fixed order: results are run-to-run identical, nothing is added
// atomically.  The partial sums are at most 148 rows whatever the batch.
// Rows that lie across 16-byte boundaries are copied in the vectors that they lie in, shifted as a lane takes them, and
// shifted back between lanes on the way out.
// Measured: 4096 x 12288 forward 44 us (4.6 TB/s), 40960 x 1024 forward 33 (5.1 TB/s), backward 52 us (4.8 TB/s), 2047 x 8191
// backward 32 us; 4096 x 12287 without a pitch 69 and 148 us.
#include <math.h>

#include "mpt_common.cuh"
#include "tc_ptx.cuh"

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

// Two FP32 values in one 64-bit register: add, mul and fma of both (each rounded as the scalar operation) in one
// instruction, which halves the issue slots that these kernels would otherwise run out of before HBM does.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float a, float b)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 halves(f2 v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float sum2(f2 v)
{
    const float2 t = halves(v);
    return t.x + t.y;
}
__device__ __forceinline__ void widen8(const uint4 v, f2 (&f)[4])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const float2 t = __half22float2(*(const __half2 *)&w[q]);
        f[q] = pair(t.x, t.y);
    }
}
__device__ __forceinline__ uint4 round8(const f2 (&f)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const float2 t = halves(f[q]);
        const __half2 h = __floats2half2_rn(t.x, t.y);
        w[q] = *(const uint32_t *)&h;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
struct Whole { static constexpr bool value = true; };      // a warp's part is 32 R whole vectors: no element needs a check
struct Ragged { static constexpr bool value = false; };

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

// The work of one warp: features [8 v0, 8 (v0 + nv)) of the rows first, first + stride, ... (n of them), and the ring of
// buffers through which NIN input matrices arrive.
constexpr int kLnMaxRowWarps = 16;    // warps a row may take
constexpr int kLnFwdWarps = 24;       // warps of a CTA of the forward kernel
// Warps of a CTA of the backward kernel: as many as its column sums, 16 registers a vector, leave room for.
constexpr __host__ __device__ int ln_bwd_warps(int R) { return R <= 2 ? 16 : 12; }
// Buffers of a warp: as many as shared memory has room for beside the scale and shift vectors.
constexpr __host__ __device__ int ln_buffers(int inputs) { return inputs == 1 ? 3 : 4; }
// Shared memory of a CTA: buffers [warps][ln_buffers][inputs][32 R + 1] of 16 bytes | the scale vector (forward: and the
// shift vector) [row_warps][32 R] | mbarriers [warps][ln_buffers].
constexpr __host__ __device__ uint32_t ln_params_at(int warps, int R, int inputs) 
{
    return (uint32_t)(warps * ln_buffers(inputs) * inputs * (R * 512 + 16));
}
constexpr __host__ __device__ uint32_t ln_bars_at(int warps, int row_warps, int R, int inputs)
{
    return ln_params_at(warps, R, inputs) + (uint32_t)((inputs == 1 ? 2 : 1) * row_warps * R * 512);
}
constexpr __host__ __device__ uint32_t ln_smem(int warps, int row_warps, int R, int inputs)
{
    return ln_bars_at(warps, row_warps, R, inputs) + (uint32_t)(warps * ln_buffers(inputs) * 8);
}

template <int R, int NIN, bool BULK>
struct LnWarp {
    int warp, lane, w, g, nw, v0, nv, c8, rows, cols, first, stride, n;
    const uint16_t *src[NIN];
    size_t ld[NIN];
    uint4 *buf;
    uint32_t bar;
    int s_ask = 0, s_use = 0;
    uint32_t parity = 0;
    volatile uint32_t *abort_flag;
    uint32_t *status;
    bool dead = false;

    static constexpr int kPart = R * 32 + 1;        // vectors of an input in a buffer: a part across 16-byte boundaries touches one more
    static constexpr int kSlot = NIN * kPart;
    static constexpr int kBuffers = ln_buffers(NIN);

    __device__ __forceinline__ LnWarp(uint8_t *smem, int row_warps, int rows_, int cols_, volatile uint32_t *abort, uint32_t *status_)
    {
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        nw = row_warps;
        const int warps = (int)blockDim.x >> 5, groups = warps / nw;
        g = warp / nw;
        w = warp - g * nw;
        rows = rows_;
        cols = cols_;
        c8 = (cols + 7) / 8;
        v0 = w * 32 * R;
        nv = min(c8 - v0, 32 * R);
        first = (int)blockIdx.x * groups + g;
        stride = (int)gridDim.x * groups;
        n = first < rows ? (rows - 1 - first) / stride + 1 : 0;
        buf = (uint4 *)smem + (size_t)warp * kBuffers * kSlot;
        bar = smem_u32(smem + ln_bars_at(warps, nw, R, NIN)) + 8u * (uint32_t)(warp * kBuffers);
        abort_flag = abort;
        status = status_;
        if (lane == 0)
            for (int s = 0; s < kBuffers; s++) mbar_init(bar + 8u * (uint32_t)s, 1);
        if (threadIdx.x == 0) *abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    __device__ __forceinline__ int row_of(int i) const { return first + i * stride; }
    // Elements between the 16-byte boundary before row i of a matrix and its start (BULK: none).
    __device__ __forceinline__ int shift(const uint16_t *base, size_t pitch, int i) const
    {
        return BULK ? 0 : (int)((((uintptr_t)base >> 1) + (size_t)row_of(i) * pitch) & 7);
    }
    // Row i into the next buffer (which is free), in the vectors that it lies in.  Vectors that it shares come whole (take()
    // clears what lies behind the row), but for one that reaches out of the matrix's memory: by elements.
    __device__ __forceinline__ void request(int i)
    {
        if (i >= n) return;
        uint4 *dst = buf + s_ask * kSlot;
        const int row = row_of(i), length = min(nv * 8, cols - v0 * 8);       // elements of this warp's part
        const uint32_t b = bar + 8u * (uint32_t)s_ask;
        const uint16_t *from[NIN];
        int lo[NIN], hi[NIN], bytes = 0;
#pragma unroll
        for (int k = 0; k < NIN; k++) {
            const int sh = shift(src[k], ld[k], i);
            const size_t at = (size_t)row * ld[k] + (size_t)v0 * 8;
            from[k] = src[k] + ((ptrdiff_t)at - sh);
            lo[k] = !BULK && at < (size_t)sh ? 1 : 0;
            const int touched = (sh + length + 7) / 8;
            hi[k] = touched - (at - sh + (size_t)touched * 8 > (size_t)(rows - 1) * ld[k] + (size_t)cols ? 1 : 0);
            if (hi[k] < lo[k]) hi[k] = lo[k];
            bytes += (hi[k] - lo[k]) * 16;
            if (lane < 8 && (lo[k] > 0 || hi[k] < touched)) {
                uint16_t *to = (uint16_t *)(dst + k * kPart);
                auto elements = [&](int v) {
                    const int e = v * 8 + lane;
                    to[e] = e >= sh && e < sh + length ? from[k][e] : (uint16_t)0;
                };
                if (lo[k] > 0) elements(0);
                if (hi[k] < touched) elements(touched - 1);
                // the copy that refills this place some rows later comes after these ordinary stores
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
        }
        __syncwarp();
        if (lane == 0) {
            if (bytes > 0) mbar_arrive_expect_tx(b, (uint32_t)bytes);
            else mbar_arrive(b);
#pragma unroll
            for (int k = 0; k < NIN; k++)
                if (hi[k] > lo[k])
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                 ::"r"(smem_u32(dst + k * kPart + lo[k])), "l"(from[k] + lo[k] * 8), "r"((uint32_t)(hi[k] - lo[k]) * 16u), "r"(b)
                                 : "memory");
        }
        __syncwarp();
        s_ask = s_ask + 1 == kBuffers ? 0 : s_ask + 1;
    }
    // Eight neighbouring elements from the `from`-th of the sixteen of two vectors on.
    __device__ __forceinline__ static uint4 across(const uint4 a, const uint4 b, int from)
    {
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (from & 4) {
#pragma unroll
            for (int i = 0; i < 6; i++) w[i] = w[i + 2];
        }
        if (from & 2) {
#pragma unroll
            for (int i = 0; i < 5; i++) w[i] = w[i + 1];
        }
        const uint32_t s = (uint32_t)(from & 1) * 16u;
        return make_uint4(__funnelshift_r(w[0], w[1], s), __funnelshift_r(w[1], w[2], s), __funnelshift_r(w[2], w[3], s),
                          __funnelshift_r(w[3], w[4], s));
    }
    // Keeps the first `left` of eight values, zeros behind them.
    __device__ __forceinline__ static void clear_behind(uint4 &v, int left)
    {
        v.x = left >= 2 ? v.x : (left == 1 ? v.x & 0xFFFFu : 0u);
        v.y = left >= 4 ? v.y : (left == 3 ? v.y & 0xFFFFu : 0u);
        v.z = left >= 6 ? v.z : (left == 5 ? v.z & 0xFFFFu : 0u);
        v.w = left >= 8 ? v.w : (left == 7 ? v.w & 0xFFFFu : 0u);
    }
    // Row i, the next one, into registers (zeros from the last feature on).
    template <bool WHOLE>
    __device__ __forceinline__ void take(int i, uint4 (&x)[NIN][R])
    {
        if (!mbar_try_wait(bar + 8u * (uint32_t)s_use, parity) && !mbar_wait(bar + 8u * (uint32_t)s_use, parity, abort_flag)) {
            // all later waits of the CTA end at once; what is computed from here on is not valid
            if (status && !*abort_flag) atomicCAS(status, 0u, (uint32_t)KERR_WAIT_FULL | 0x40u | ((uint32_t)blockIdx.x << 8));
            *abort_flag = 1u;
            dead = true;
        }
        const uint4 *from = buf + s_use * kSlot;
#pragma unroll
        for (int k = 0; k < NIN; k++) {
            const int sh = shift(src[k], ld[k], i);
#pragma unroll
            for (int u = 0; u < R; u++) {
                const int j = lane + 32 * u;
                x[k][u] = WHOLE || j < nv ? from[k * kPart + j] : make_uint4(0u, 0u, 0u, 0u);
                if (!BULK && sh > 0) x[k][u] = across(x[k][u], WHOLE || j < nv ? from[k * kPart + j + 1] : x[k][u], sh);
                if (!WHOLE && !whole(u)) clear_behind(x[k][u], cols - (v0 + j) * 8);
            }
        }
        __syncwarp();
        if (++s_use == kBuffers) {
            s_use = 0;
            parity ^= 1u;
        }
    }
    // Sum over the row's warps, in warp order; `red`: 16 words of this group, zero from nw on.
    __device__ __forceinline__ float row_sum(float v, float *red) const
    {
        v = warp_sum(v);
        if (nw == 1) return v;
        if (lane == 0) red[w] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + g), "r"(nw * 32) : "memory");
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < kLnMaxRowWarps / 4; q++) {
            const float4 t = ((const float4 *)red)[q];
            s += (t.x + t.y) + (t.z + t.w);
        }
        return s;
    }
    // After a wait that ran out: copies still on their way get a bounded time to land before the CTA's memory is used otherwise.
    __device__ __forceinline__ void settle() const
    {
        if (dead) {
            const unsigned long long t0 = global_ns();
            while (global_ns() - t0 < 1000000ull) {}
        }
        __syncthreads();
    }
    // whether the warp's vectors 32 u ... 32 u + 31 are all whole (the same for all lanes)
    __device__ __forceinline__ bool whole(int u) const { return (v0 + 32 * (u + 1)) * 8 <= cols; }
    // The warp's part of row i of a result, by 16-byte stores: the vectors between 16-byte boundaries of the output are put
    // together from a lane's own and its neighbour's elements; at the ends of the part, element by element.
    __device__ __forceinline__ void put(uint16_t *base, size_t pitch, int i, const uint4 (&y)[R]) const
    {
        uint16_t *o = base + (size_t)row_of(i) * pitch;
        const int sh = shift(base, pitch, i);
        uint4 before = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int u = 0; u < R; u++) {
            const int j = lane + 32 * u, at = (v0 + j) * 8;
            if (BULK || sh == 0) {
                if (j < nv) store8<true>(o, at, cols, y[u]);
                continue;
            }
            const int left = (lane + 31) & 31;
            const uint4 turned = make_uint4(__shfl_sync(0xFFFFFFFFu, y[u].x, left), __shfl_sync(0xFFFFFFFFu, y[u].y, left),
                                            __shfl_sync(0xFFFFFFFFu, y[u].z, left), __shfl_sync(0xFFFFFFFFu, y[u].w, left));
            const uint4 v = across(lane == 0 ? before : turned, y[u], 8 - sh);
            before = turned;
            if (j >= nv) continue;
            if (j > 0 && at - sh + 8 <= cols) __stcs((uint4 *)(o + (at - sh)), v);
            else elements(o, at - sh, v, j > 0 ? at - sh : at, cols);
            if (j == nv - 1) elements(o, at, y[u], at - sh + 8, cols);
        }
    }
    // Those of eight elements from `at` on that lie in [lo, hi).
    __device__ __forceinline__ static void elements(uint16_t *o, int at, const uint4 v, int lo, int hi)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (at + e >= lo && at + e < hi) o[at + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
};

// A scale or shift vector (null: zeros) to shared memory, zeros from the last feature on; all loads are asked for before the
// first is there.  Not inlined: its registers would be taken from the row loop's (4096 x 12288 forward 45 us, inlined 47.5).
template <int R, bool BULK>
__device__ __noinline__ void ln_params(uint4 *to, const uint16_t *from, int vectors, int cols)
{
    uint4 v[R];
#pragma unroll
    for (int u = 0; u < R; u++) {
        const int col = ((int)threadIdx.x + u * (int)blockDim.x) * 8;
        v[u] = from && col < cols ? load8<BULK, false>(from, col, cols) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < R; u++) {
        const int j = (int)threadIdx.x + u * (int)blockDim.x;
        if (j < vectors) to[j] = v[u];
    }
}

struct LnFwd {
    int rows, cols, row_warps;
    const uint16_t *x;
    size_t ldx;
    const uint16_t *gamma, *beta;      // beta may be null
    float eps;
    uint16_t *y;
    size_t ldy;
    float *mean, *rstd;                // may be null
    uint32_t *status;                  // may be null
};

template <int R, bool BULK>
__global__ void __launch_bounds__(kLnFwdWarps * 32, 1) k_ln_fwd(const LnFwd p)
{
    pdl_trigger();
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float red[kLnFwdWarps / 2][2][16];      // a row of one warp has no use for it
    __shared__ uint32_t abort_word;
    for (int i = threadIdx.x; i < kLnFwdWarps * 16; i += blockDim.x) (&red[0][0][0])[i] = 0.0f;
    LnWarp<R, 1, BULK> c(smem, p.row_warps, p.rows, p.cols, &abort_word, p.status);
    pdl_wait();                       // up to here nothing was read or written that another kernel knows of
    c.src[0] = p.x;
    c.ld[0] = p.ldx;
    for (int i = 0; i < c.kBuffers; i++) c.request(i);
    const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
    const int col0 = (c.v0 + c.lane) * 8;
    // scale and shift in shared memory, zeros from the last feature on (48 KB of them for 12288 features do not stay in the L1
    // that the buffers leave: read through it, every row waited for L2; 40960 x 1024 37 us, now 33)
    const int vectors = c.nw * 32 * R;
    uint4 *gamma = (uint4 *)(smem + ln_params_at((int)(blockDim.x >> 5), R, 1)), *beta = gamma + vectors;
    ln_params<R, BULK>(gamma, p.gamma, vectors, p.cols);
    ln_params<R, BULK>(beta, p.beta, vectors, p.cols);
    __syncthreads();
    gamma += c.v0 + c.lane;
    beta += c.v0 + c.lane;
    auto rows = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        for (int i = 0; i < c.n; i++) {
            uint4 x[1][R];
            c.template take<W>(i, x);
            c.request(i + c.kBuffers);
            f2 f[R][4];
            f2 s = pair(0.0f, 0.0f);
#pragma unroll
            for (int u = 0; u < R; u++) {
                widen8(x[0][u], f[u]);
                s = add2(s, add2(add2(f[u][0], f[u][1]), add2(f[u][2], f[u][3])));
            }
            const float mean = c.row_sum(sum2(s), red[c.g][0]) * inv_n;
            const f2 minus = pair(-mean, -mean);
            f2 q0 = pair(0.0f, 0.0f), q1 = q0;
#pragma unroll
            for (int u = 0; u < R; u++) {
#pragma unroll
                for (int e = 0; e < 4; e++) f[u][e] = add2(f[u][e], minus);
                if (!W && !c.whole(u)) {           // what lies behind the last feature must not count: deviation zero
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int col = col0 + 256 * u + 2 * e;
                        const float2 d = halves(f[u][e]);
                        f[u][e] = pair(col < p.cols ? d.x : 0.0f, col + 1 < p.cols ? d.y : 0.0f);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    q0 = fma2(f[u][e], f[u][e], q0);
                    q1 = fma2(f[u][e + 1], f[u][e + 1], q1);
                }
            }
            const float var = c.row_sum(sum2(add2(q0, q1)), red[c.g][1]) * inv_n;
            const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(var + p.eps));
            const int row = c.row_of(i);
            if (c.w == 0 && c.lane == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
            const f2 r2 = pair(rstd, rstd);
            uint4 y[R];
#pragma unroll
            for (int u = 0; u < R; u++) {
                f2 g[4], b[4];
                widen8(gamma[32 * u], g);
                widen8(beta[32 * u], b);
#pragma unroll
                for (int e = 0; e < 4; e++) f[u][e] = fma2(mul2(f[u][e], r2), g[e], b[e]);
                y[u] = round8(f[u]);
                if (BULK && W) __stcs((uint4 *)(p.y + (size_t)row * p.ldy + col0 + 256 * u), y[u]);
            }
            if (!(BULK && W)) c.put(p.y, p.ldy, i, y);
        }
    };
    if (c.whole(R - 1)) rows(Whole{});
    else rows(Ragged{});
    c.settle();
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
    int rows, cols, row_warps;
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
    uint32_t *status;                  // may be null
};

template <int R, bool BULK>
__global__ void __launch_bounds__(ln_bwd_warps(R) * 32, 1) k_ln_bwd(const LnBwd p)
{
    pdl_trigger();
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float red[8][2][2][16];       // a row of one warp has no use for it
    __shared__ uint32_t abort_word;
    for (int i = threadIdx.x; i < 8 * 64; i += blockDim.x) (&red[0][0][0][0])[i] = 0.0f;
    LnWarp<R, 2, BULK> c(smem, p.row_warps, p.rows, p.cols, &abort_word, p.status);
    pdl_wait();                       // up to here nothing was read or written that another kernel knows of
    c.src[0] = p.x;
    c.ld[0] = p.ldx;
    c.src[1] = p.dy;
    c.ld[1] = p.lddy;
    for (int i = 0; i < c.kBuffers; i++) c.request(i);
    const int col0 = (c.v0 + c.lane) * 8;
    // the scale in shared memory, zeros from the last feature on
    uint4 *gamma = (uint4 *)(smem + ln_params_at((int)(blockDim.x >> 5), R, 2));
    ln_params<R, BULK>(gamma, p.gamma, c.nw * 32 * R, p.cols);
    __syncthreads();
    gamma += c.v0 + c.lane;
    f2 ag[R][4], ab[R][4];
#pragma unroll
    for (int u = 0; u < R; u++) {
#pragma unroll
        for (int e = 0; e < 4; e++) ag[u][e] = ab[u][e] = pair(0.0f, 0.0f);
    }
    const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
    auto rows = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        // the statistics of 32 rows at a time, one per lane, asked for 32 rows ahead
        float mean_next = 0.0f, rstd_next = 0.0f, mean32 = 0.0f, rstd32 = 0.0f;
        auto ask_stats = [&](int i) {
            if (i + c.lane < c.n) {
                mean_next = p.mean[c.row_of(i + c.lane)];
                rstd_next = p.rstd[c.row_of(i + c.lane)];
            }
        };
        ask_stats(0);
        for (int i = 0; i < c.n; i++) {
            if ((i & 31) == 0) {
                mean32 = mean_next;
                rstd32 = rstd_next;
                ask_stats(i + 32);
            }
            const float mean = __shfl_sync(0xFFFFFFFFu, mean32, i & 31), rstd = __shfl_sync(0xFFFFFFFFu, rstd32, i & 31);
            const f2 minus = pair(-mean, -mean), r2 = pair(rstd, rstd);
            uint4 v[2][R];
            c.template take<W>(i, v);
            c.request(i + c.kBuffers);
            f2 h[R][4], gy[R][4];
            f2 s1 = pair(0.0f, 0.0f), s2 = s1;
#pragma unroll
            for (int u = 0; u < R; u++) {
                f2 d[4], g[4];
                widen8(v[0][u], h[u]);
                widen8(v[1][u], d);
                widen8(gamma[32 * u], g);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    h[u][e] = mul2(add2(h[u][e], minus), r2);
                    gy[u][e] = mul2(d[e], g[e]);
                    s1 = add2(s1, gy[u][e]);
                    s2 = fma2(gy[u][e], h[u][e], s2);
                    ag[u][e] = fma2(d[e], h[u][e], ag[u][e]);
                    ab[u][e] = add2(ab[u][e], d[e]);
                }
            }
            float c1 = warp_sum(sum2(s1)), c2 = warp_sum(sum2(s2));
            if (c.nw > 1) {
                float (*r)[16] = red[c.g][i & 1];            // the two are a barrier apart
                if (c.lane == 0) {
                    r[0][c.w] = c1;
                    r[1][c.w] = c2;
                }
                asm volatile("bar.sync %0, %1;" ::"r"(1 + c.g), "r"(c.nw * 32) : "memory");
                c1 = c2 = 0.0f;
#pragma unroll
                for (int q = 0; q < kLnMaxRowWarps / 4; q++) {
                    const float4 a = ((const float4 *)r[0])[q], b = ((const float4 *)r[1])[q];
                    c1 += (a.x + a.y) + (a.z + a.w);
                    c2 += (b.x + b.y) + (b.z + b.w);
                }
            }
            const float m1 = -rstd * (c1 * inv_n), m2 = -rstd * (c2 * inv_n);
            const f2 k1 = pair(m1, m1), k2 = pair(m2, m2);
            uint4 o[R];
#pragma unroll
            for (int u = 0; u < R; u++) {
#pragma unroll
                for (int e = 0; e < 4; e++) gy[u][e] = fma2(gy[u][e], r2, fma2(h[u][e], k2, k1));
                o[u] = round8(gy[u]);
                if (BULK && W) __stcs((uint4 *)(p.dx + (size_t)c.row_of(i) * p.lddx + col0 + 256 * u), o[u]);
            }
            if (!(BULK && W)) c.put(p.dx, p.lddx, i, o);
        }
    };
    if (c.whole(R - 1)) rows(Whole{});
    else rows(Ragged{});
    c.settle();
    // The CTA's column sums, through the ring's memory (not in use any more): a lane holds 8 neighbouring columns, and 8-byte
    // stores 32 bytes apart took 7 us for 8191 features.  Several groups of warps that hold the same features are added in
    // group order.
    const int groups = (int)(blockDim.x >> 5) / c.nw, width = c.nw * 256 * R;
    float *sums = (float *)smem;                     // [2][groups][width]
#pragma unroll
    for (int u = 0; u < R; u++) {
        float4 *g = (float4 *)(sums + c.g * width + (c.v0 + c.lane + 32 * u) * 8), *b = g + groups * width / 4;
        const float2 g0 = halves(ag[u][0]), g1 = halves(ag[u][1]), g2 = halves(ag[u][2]), g3 = halves(ag[u][3]);
        const float2 b0 = halves(ab[u][0]), b1 = halves(ab[u][1]), b2 = halves(ab[u][2]), b3 = halves(ab[u][3]);
        g[0] = make_float4(g0.x, g0.y, g1.x, g1.y);
        g[1] = make_float4(g2.x, g2.y, g3.x, g3.y);
        b[0] = make_float4(b0.x, b0.y, b1.x, b1.y);
        b[1] = make_float4(b2.x, b2.y, b3.x, b3.y);
    }
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; which++) {
        float *out = p.parts + ((size_t)which * gridDim.x + blockIdx.x) * p.colp;
        const float *from = sums + which * groups * width;
        for (int col = threadIdx.x * 4; col < p.colp; col += blockDim.x * 4) {       // colp is a multiple of 8 and at most width
            float4 s = *(const float4 *)(from + col);
            for (int k = 1; k < groups; k++) {
                const float4 t = *(const float4 *)(from + k * width + col);
                s = make_float4(s.x + t.x, s.y + t.y, s.z + t.z, s.w + t.w);
            }
            *(float4 *)(out + col) = s;
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
    for (int e = 0; e < 8; e += 4) {
        *(float4 *)(pg + col + e) = make_float4(ag[e], ag[e + 1], ag[e + 2], ag[e + 3]);
        *(float4 *)(pb + col + e) = make_float4(ab[e], ab[e + 1], ab[e + 2], ab[e + 3]);
    }
}

// dgamma / dbeta: the partial rows added in a fixed order (sixteen warps take every sixteenth row, their sums are
// then added in warp order), rounded to FP16 and inspected for inf/NaN.  blockIdx.y: 0 dgamma, 1 dbeta.
__global__ void __launch_bounds__(512) k_ln_param_grad(const float *__restrict__ parts, int nparts, int cols, int colp,
                                                       uint16_t *__restrict__ dgamma, uint16_t *__restrict__ dbeta,
                                                       uint32_t *nonfinite_flag)
{
    pdl_trigger();
    pdl_wait();
    __shared__ float sh[16][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const float *src = parts + (size_t)blockIdx.y * nparts * colp;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 10
        for (int r = warp; r < nparts; r += 16) s += src[(size_t)r * colp + col];
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0) {
        bool bad = false;
        if (col < cols) {
            s = sh[0][lane];
#pragma unroll
            for (int w = 1; w < 16; w++) s += sh[w][lane];
            const uint32_t h = (uint32_t)__half_as_ushort(__float2half_rn(s));
            bad = half_bits_nonfinite(h);
            (blockIdx.y ? dbeta : dgamma)[col] = (uint16_t)h;
        }
        if (nonfinite_flag && __any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(nonfinite_flag, 1u);
    }
}

constexpr int kLnMaxParts = 148;      // partial rows of the column sums: one CTA on each SM
constexpr int kLnMaxSize = 1 << 30;   // rows and features: what is added to their indexes stays inside 32 bits

int ln_colp(int cols) { return (cols + 7) / 8 * 8; }
int ln_parts(int rows) { return rows < kLnMaxParts ? rows : kLnMaxParts; }

// How rows of c8 vectors are laid over warps: R vectors a lane, row_warps warps a row, groups of them in a CTA (fewer
// where there are not enough rows for all SMs), and the grid: one CTA with all warps on an SM, or as many
// smaller ones as make that up.
struct LnShape {
    int R, row_warps, groups, grid;
};
LnShape ln_shape(int rows, int c8, bool backward)
{
    auto warps = [&](int r) { return backward ? ln_bwd_warps(r) : kLnFwdWarps; };
    LnShape s = {c8 <= 128 ? (c8 + 31) / 32 : 4, 0, 0, 0};
    if (c8 > 128) {
        int best = 0;
        for (int r = 4; r >= 2; r--) {
            const int w = (c8 + 32 * r - 1) / (32 * r), most = warps(r) < kLnMaxRowWarps ? warps(r) : kLnMaxRowWarps;
            const int busy = w <= most ? warps(r) / w * w : 0;
            if (busy > best) { best = busy; s.R = r; }
        }
    }
    const int all = warps(s.R);
    s.row_warps = (c8 + 32 * s.R - 1) / (32 * s.R);
    const int most = all / s.row_warps, spread = (rows + 147) / 148;
    s.groups = spread < most ? spread : most;
    const long ctas = ((long)rows + s.groups - 1) / s.groups;
    const long fit = 148L * (all / (s.groups * s.row_warps));
    s.grid = (int)(ctas < fit ? ctas : fit);
    return s;
}

template <typename P>
cudaError_t ln_run(void (*kern)(const P), int id, const P &p, const LnShape &s, int inputs, cudaStream_t st)
{
    static bool configured[kMaxDevices][8] = {};
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    const int warps = s.groups * s.row_warps;
    const size_t smem = ln_smem(warps, s.row_warps, s.R, inputs);
    if (!configured[dev][id]) {
        const int most = inputs == 1 ? ln_smem(kLnFwdWarps, kLnMaxRowWarps, 4, 1) : ln_smem(12, 12, 4, 2);
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != cudaSuccess) return e;
        configured[dev][id] = true;
    }
    MPT_LAUNCH(kern, dim3((unsigned)s.grid), dim3((unsigned)(warps * 32)), smem, st, p);
    return cudaSuccess;
}

cudaError_t launch_ln_fwd(LnFwd p, cudaStream_t st)
{
    const uintptr_t bits = (uintptr_t)p.x | (uintptr_t)p.y | (uintptr_t)p.gamma | (uintptr_t)p.beta;
    const bool vec = (bits & 15) == 0 && ((p.ldx | p.ldy) & 7) == 0;
    const int c8 = (p.cols + 7) / 8;
    if (c8 <= kLnMaxRowWarps * 128) {
        const LnShape s = ln_shape(p.rows, c8, false);
        p.row_warps = s.row_warps;
        if (s.R == 1) return vec ? ln_run(k_ln_fwd<1, true>, 0, p, s, 1, st) : ln_run(k_ln_fwd<1, false>, 1, p, s, 1, st);
        if (s.R == 2) return vec ? ln_run(k_ln_fwd<2, true>, 2, p, s, 1, st) : ln_run(k_ln_fwd<2, false>, 3, p, s, 1, st);
        if (s.R == 3) return vec ? ln_run(k_ln_fwd<3, true>, 4, p, s, 1, st) : ln_run(k_ln_fwd<3, false>, 5, p, s, 1, st);
        return vec ? ln_run(k_ln_fwd<4, true>, 6, p, s, 1, st) : ln_run(k_ln_fwd<4, false>, 7, p, s, 1, st);
    }
    const int grid = p.rows < 296 ? p.rows : 296;
    if (vec) MPT_LAUNCH(k_ln_fwd_long<true>, dim3((unsigned)grid), dim3(1024), 0, st, p);
    else MPT_LAUNCH(k_ln_fwd_long<false>, dim3((unsigned)grid), dim3(1024), 0, st, p);
    return cudaSuccess;
}

cudaError_t launch_ln_bwd(LnBwd p, uint16_t *dgamma, uint16_t *dbeta, uint32_t *nonfinite_flag, cudaStream_t st)
{
    const uintptr_t bits = (uintptr_t)p.x | (uintptr_t)p.dy | (uintptr_t)p.dx | (uintptr_t)p.gamma;
    const bool vec = (bits & 15) == 0 && ((p.ldx | p.lddy | p.lddx) & 7) == 0;
    const int c8 = (p.cols + 7) / 8;
    int nparts = 0;
    cudaError_t e = cudaSuccess;
    if (p.rows > 0 && c8 <= ln_bwd_warps(4) * 128) {
        const LnShape s = ln_shape(p.rows, c8, true);
        p.row_warps = s.row_warps;
        nparts = s.grid;
        if (s.R == 1) e = vec ? ln_run(k_ln_bwd<1, true>, 0, p, s, 2, st) : ln_run(k_ln_bwd<1, false>, 1, p, s, 2, st);
        else if (s.R == 2) e = vec ? ln_run(k_ln_bwd<2, true>, 2, p, s, 2, st) : ln_run(k_ln_bwd<2, false>, 3, p, s, 2, st);
        else if (s.R == 3) e = vec ? ln_run(k_ln_bwd<3, true>, 4, p, s, 2, st) : ln_run(k_ln_bwd<3, false>, 5, p, s, 2, st);
        else e = vec ? ln_run(k_ln_bwd<4, true>, 6, p, s, 2, st) : ln_run(k_ln_bwd<4, false>, 7, p, s, 2, st);
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
    MPT_LAUNCH(k_ln_param_grad, grid, dim3(512), 0, st, (const float *)p.parts, nparts, p.cols, p.colp, dgamma, dbeta, nonfinite_flag);
    return cudaSuccess;
}

}  // namespace
}  // namespace mpt

using namespace mpt;

extern "C" {

int mpt_layernorm_forward(int rows, int cols, const uint16_t *x_dev, int ldx, const uint16_t *gamma16_dev,
                          const uint16_t *beta16_dev, float eps, uint16_t *y_dev, int ldy, float *mean_dev, float *rstd_dev,
                          uint32_t *status_dev, void *cuda_stream)
{
    // an empty batch has no addresses: what holds rows may be null then, here and in the backward pass
    if (!gamma16_dev || (rows != 0 && (!x_dev || !y_dev || x_dev == y_dev))) return MPT_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || !isfinite(eps)) return MPT_ERR_INVALID_ARG;
    if (rows < 0 || rows > kLnMaxSize || cols < 1 || cols > kLnMaxSize || ldx < cols || ldy < cols) return MPT_ERR_SHAPE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) return MPT_OK;
    const LnFwd p = {rows, cols, 0, x_dev, (size_t)ldx, gamma16_dev, beta16_dev, eps, y_dev, (size_t)ldy, mean_dev, rstd_dev, status_dev};
    return launch_ln_fwd(p, st) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

int mpt_layernorm_workspace_bytes(int rows, int cols, size_t *bytes_out)
{
    if (!bytes_out) return MPT_ERR_INVALID_ARG;
    if (rows < 0 || rows > kLnMaxSize || cols < 1 || cols > kLnMaxSize) return MPT_ERR_SHAPE;
    *bytes_out = (size_t)2 * (size_t)(ln_parts(rows) > 0 ? ln_parts(rows) : 1) * (size_t)ln_colp(cols) * sizeof(float);
    return MPT_OK;
}

int mpt_layernorm_backward(int rows, int cols, const uint16_t *dy_dev, int lddy, const uint16_t *x_dev, int ldx,
                           const uint16_t *gamma16_dev, const float *mean_dev, const float *rstd_dev, uint16_t *dx_dev, int lddx,
                           uint16_t *dgamma16_dev, uint16_t *dbeta16_dev, uint32_t *nonfinite_flag_dev, uint32_t *status_dev,
                           void *workspace_dev, size_t workspace_bytes, void *cuda_stream)
{
    if (!gamma16_dev || !dgamma16_dev || !workspace_dev) return MPT_ERR_INVALID_ARG;
    if (rows != 0 && (!dy_dev || !x_dev || !mean_dev || !rstd_dev || !dx_dev || dx_dev == dy_dev || dx_dev == x_dev)) return MPT_ERR_INVALID_ARG;
    if (rows < 0 || rows > kLnMaxSize || cols < 1 || cols > kLnMaxSize || lddy < cols || ldx < cols || lddx < cols) return MPT_ERR_SHAPE;
    size_t need = 0;
    mpt_layernorm_workspace_bytes(rows, cols, &need);
    if (workspace_bytes < need || ((uintptr_t)workspace_dev & 15) != 0) return MPT_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const LnBwd p = {rows, cols, 0, dy_dev, (size_t)lddy, x_dev, (size_t)ldx, gamma16_dev, mean_dev, rstd_dev, dx_dev, (size_t)lddx,
                     (float *)workspace_dev, ln_colp(cols), status_dev};
    return launch_ln_bwd(p, dgamma16_dev, dbeta16_dev, nonfinite_flag_dev, st) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

}  // extern "C"
