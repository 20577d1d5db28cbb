// Distillation from a teacher's top logits (softmax reductions in FP32 on FP16 logits, gradient multiplied by
// S / B before it is rounded: paper sections 3.2, 3.3).  Per row, with K teacher entries (class, logit):
//
//   q = softmax over the row's entries of t / tau ;  p = softmax over all C classes of z / tau
//   loss = tau^2 sum_j q_j (log q_j - log p_c(j)) ;  dz_v = rn16(tau * (p_v - sum of q_j with c(j) = v) * S / B)
//
// Bound: HBM, 4 bytes a logit (z read once, dz written once).  A row is spread over the warps of one CTA or of a
// cluster of 2, 4 or 8, so that its logits stay in shared memory between the two passes over them.  Every warp is a
// pipeline of its own over its part of every row: bulk copies in, running maximum and sum of exponentials, bulk copy
// out of the gradient formed in place.  The only thing warps exchange is one (reference, sum) pair per row, through
// distributed shared memory and one cluster barrier, whose two halves have the first pass over the NEXT row between
// them; so nothing waits for the slowest warp, and loads and stores are always in flight.  One more warp per CTA
// prepares the teacher's entries while the others work.
// Exponentials are taken twice (once per pass) rather than kept: 2.1 special-function results a logit are 4300
// cycles for 32000 logits of a row, against 5600 cycles that its 128 KB take at an SM's share of HBM.
// Rows too long for the shared memory of 8 CTAs (about 430 000 classes) are read a second time instead, from L2: the
// rows in work at any moment are a few tens of MB.
#include <math.h>

#include "mpt_common.cuh"
#include "tc_ptx.cuh"

namespace mpt {
namespace {

struct DistillArgs {
    const uint16_t *z;
    size_t ldz;
    int B, C;
    const uint16_t *t;
    const int32_t *idx;
    size_t ldt;
    int K;
    float k;             // log2(e) / tau
    float tau;
    float c;             // tau * S / B
    uint16_t *dz;        // may be null
    size_t lddz;
    float *row_loss;
    uint32_t *kerr;
    int nw;              // warps that hold logits (one more prepares the teacher's entries)
    int wv;              // vectors of 8 logits per warp
    int vp;              // vectors per CTA
    int cl;              // CTAs per cluster
    int ns;              // buffers per warp
    int chunk;           // streamed rows: vectors per buffer
};

struct Entry {
    int32_t v;           // class, -1: none
    float q;             // teacher's probability
    float z;             // student's logit
};
constexpr int kEntryBuffers = 3;
constexpr uint32_t kNegInf16 = 0xFC00u;

__device__ __forceinline__ float h2f(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }
__device__ __forceinline__ uint32_t f2h(float x) { return (uint32_t)__half_as_ushort(__float2half_rn(x)); }
__device__ __forceinline__ float wsum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float wmax(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// Running sum of a lane: sum of 2^(z k + b) with b = -max * k as it was rounded, so the pair says exactly what
// was added up.  max = -inf: nothing but -inf (or NaN, which then is in s) so far, b = 0.
struct Run {
    float m = -INFINITY, b = 0.0f, s = 0.0f;
};
__device__ __forceinline__ void run_add8(Run &r, const uint4 x, float k)
{
    const __half2 mx = __hmax2(__hmax2(*(const __half2 *)&x.x, *(const __half2 *)&x.y), __hmax2(*(const __half2 *)&x.z, *(const __half2 *)&x.w));
    const float m = fmaxf(__low2float(mx), __high2float(mx));       // NaN is dropped here and comes back in the sum
    if (m > r.m) {
        const float b = -__fmul_rn(m, k);
        r.s = r.m == -INFINITY ? r.s : r.s * ex2_approx(b - r.b);
        r.m = m;
        r.b = b;
    }
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float a[4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const float2 f = __half22float2(*(const __half2 *)&w[q]);
        a[q] = ex2_approx(fmaf(f.x, k, r.b)) + ex2_approx(fmaf(f.y, k, r.b));
    }
    r.s += (a[0] + a[1]) + (a[2] + a[3]);
}
// The warp's pair: reference e (terms are relative to 2^e), sum.  A lane with e = -inf has nothing or NaN to add.
__device__ __forceinline__ float2 run_warp(const Run &r)
{
    const float e = r.m == -INFINITY ? -INFINITY : -r.b;
    const float E = wmax(e);
    return make_float2(E, wsum(e == -INFINITY ? r.s : r.s * ex2_approx(e - E)));
}
// The row's pair from those of all warps (every lane gets the same bits): p = 2^(z k - x) / y.  The two stay apart:
// with logits near FP16's largest their log2 would be a number of 10^5, known to a hundredth only.
__device__ __forceinline__ float2 row_pair(const float2 *red, int pairs)
{
    const int lane = threadIdx.x & 31;
    float E = -INFINITY;
    for (int i = lane; i < pairs; i += 32) E = fmaxf(E, red[i].x);
    E = wmax(E);
    float s = 0.0f;
    for (int i = lane; i < pairs; i += 32) {
        const float2 p = red[i];
        s += p.x == -INFINITY ? p.y : p.y * ex2_approx(p.x - E);
    }
    return make_float2(E, wsum(s));
}

// Gradient of n vectors in place.
__device__ __forceinline__ void grad_vectors(uint4 *v, int n, float k, float2 pr, float c, bool live)
{
    const int lane = threadIdx.x & 31;
    const float cs = __fdiv_rn(c, pr.y);
#pragma unroll 4
    for (int i = lane; i < n; i += 32) {
        const uint4 x = v[i];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const float2 f = __half22float2(*(const __half2 *)&w[q]);
            o[q] = live ? pack_f16x2(ex2_approx(fmaf(f.x, k, -pr.x)) * cs, ex2_approx(fmaf(f.y, k, -pr.x)) * cs) : 0u;
        }
        v[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}
// The teacher's classes among the logits [first, first + count) that this warp holds at h: their gradient again
// with the probabilities of all entries of that class subtracted (an entry named twice is written twice, alike).
__device__ __forceinline__ void patch_targets(uint16_t *h, int first, int count, const Entry *ent, int K, float k, float2 pr, float c)
{
    const int lane = threadIdx.x & 31;
    for (int j0 = 0; j0 < K; j0 += 32) {
        const int j = j0 + lane;
        const int v = j < K ? ent[j].v : -1;
        unsigned hit = __ballot_sync(0xFFFFFFFFu, v >= 0 && (unsigned)(v - first) < (unsigned)count);
        while (hit) {
            const int src = __ffs((int)hit) - 1;
            hit &= hit - 1;
            const int at = __shfl_sync(0xFFFFFFFFu, v, src);
            float q = 0.0f;
            for (int i = lane; i < K; i += 32)
                if (ent[i].v == at) q += ent[i].q;
            q = wsum(q);
            if (lane == src) h[at - first] = (uint16_t)f2h((__fdiv_rn(ex2_approx(fmaf(ent[j].z, k, -pr.x)), pr.y) - q) * c);
        }
    }
}

// Teacher's entries of a row, by one warp.  Entries whose class is outside [0, C) or whose logit is -inf have no part;
// *live: whether any has.
__device__ __forceinline__ void prepare_entries(const DistillArgs &p, int row, Entry *ent, int *live)
{
    const int lane = threadIdx.x & 31;
    const int32_t *id = p.idx + (size_t)row * p.ldt;
    const uint16_t *tt = p.t + (size_t)row * p.ldt, *zr = p.z + (size_t)row * p.ldz;
    float top = -INFINITY;
    bool any = false;
#pragma unroll 4
    for (int j = lane; j < p.K; j += 32) {
        const int v = id[j];
        const float t = h2f(tt[j]);
        const bool ok = v >= 0 && v < p.C && t != -INFINITY;
        Entry e;
        e.v = ok ? v : -1;
        e.q = t;
        e.z = ok ? h2f(zr[v]) : 0.0f;
        ent[j] = e;
        if (ok) top = fmaxf(top, t);
        any |= ok;
    }
    top = wmax(top);
    any = __any_sync(0xFFFFFFFFu, any);
    float s = 0.0f;
    for (int j = lane; j < p.K; j += 32) {
        const float w = ent[j].v >= 0 ? ex2_approx((ent[j].q - top) * p.k) : 0.0f;
        ent[j].q = w;
        s += w;
    }
    s = wsum(s);
    const float inv = __fdiv_rn(1.0f, s);
    for (int j = lane; j < p.K; j += 32) ent[j].q = ent[j].v >= 0 ? ent[j].q * inv : 0.0f;
    if (lane == 0) *live = any ? 1 : 0;
    __syncwarp();
}
__device__ __forceinline__ void write_loss(const DistillArgs &p, int row, const Entry *ent, bool live, float2 pr)
{
    const int lane = threadIdx.x & 31;
    constexpr float LN2 = 0.69314718055994531f;
    const float l2s = log2f(pr.y);
    float l = 0.0f;
    for (int j = lane; j < p.K; j += 32) {
        const Entry e = ent[j];
        // log2 q - log2 p; a probability of zero (or none) adds nothing
        if (e.v >= 0 && !(e.q == 0.0f)) l += e.q * ((log2f(e.q) + l2s) - fmaf(e.z, p.k, -pr.x));
    }
    l = wsum(l);
    if (lane == 0) p.row_loss[row] = live ? l * LN2 * p.tau * p.tau : 0.0f;
}

__device__ __forceinline__ void bulk_in(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    mbar_arrive_expect_tx(bar, bytes);
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void bulk_out(void *dst, uint32_t src, uint32_t bytes)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}

// Shared memory: buffers [nw][ns][per] of 16-byte vectors | mbarriers [nw][ns] | pairs [2][cl * nw] |
// entries [3][K] | live [3] | abort word
struct Layout {
    uint32_t bars, red, ent, live, abort, total;
};
__host__ __device__ inline Layout layout_of(int nw, int ns, int per, int cl, int K)
{
    Layout l;
    uint32_t at = (uint32_t)nw * (uint32_t)ns * (uint32_t)per * 16u;
    l.bars = at;
    at += (uint32_t)nw * (uint32_t)ns * 8u;
    l.red = at;
    at += 2u * (uint32_t)cl * (uint32_t)nw * 8u;
    l.ent = at;
    at += (uint32_t)kEntryBuffers * (uint32_t)K * (uint32_t)sizeof(Entry);
    l.live = at;
    at += 4u * kEntryBuffers;
    l.abort = at;
    at += 4u;
    l.total = (at + 15u) & ~15u;
    return l;
}

// BULK: rows start on 16-byte boundaries and move by bulk copies (a last, partial vector by element accesses);
// otherwise the warp copies elements.  STREAM: the row does not stay in shared memory; the second pass reads it again.
template <bool BULK, bool STREAM>
__global__ void __launch_bounds__(1024, 1) k_distill(const DistillArgs p)
{
    pdl_trigger();
    pdl_wait();
    extern __shared__ __align__(128) uint8_t smem[];
    const int per = STREAM ? p.chunk : p.wv;
    const Layout L = layout_of(p.nw, p.ns, per, p.cl, p.K);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.cl > 1 ? (int)cluster_ctarank() : 0;
    const int cluster = blockIdx.x / p.cl, clusters = gridDim.x / p.cl;
    const int n_rows = cluster < p.B ? (p.B - 1 - cluster) / clusters + 1 : 0;
    float2 *red = (float2 *)(smem + L.red);
    Entry *entries = (Entry *)(smem + L.ent);
    int *live = (int *)(smem + L.live);
    volatile uint32_t *abort_flag = (volatile uint32_t *)(smem + L.abort);
    const int pairs = p.cl * p.nw;

    if (warp < p.nw && lane == 0)
        for (int s = 0; s < p.ns; s++) mbar_init(smem_u32(smem + L.bars) + 8u * (uint32_t)(warp * p.ns + s), 1);
    if (threadIdx.x == 0) *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    cluster_sync_all();              // every CTA of the cluster runs before anything is written into its shared memory
    if (n_rows == 0) return;         // the same for all CTAs of a cluster

    if (warp == p.nw) {
        // ------------------------------------------------------------ the teacher's entries, the losses
        prepare_entries(p, cluster, entries, live);
        cluster_arrive();
        for (int i = 0; i < n_rows; i++) {
            cluster_wait();
            if (rank == 0) {
                const int b = i % kEntryBuffers;
                write_loss(p, cluster + i * clusters, entries + b * p.K, live[b] != 0, row_pair(red + (i & 1) * pairs, pairs));
            }
            if (i + 1 < n_rows) {
                // after the barrier of row i all warps have finished with row i - 2, whose buffer this is
                const int b = (i + 1) % kEntryBuffers;
                prepare_entries(p, cluster + (i + 1) * clusters, entries + b * p.K, live + b);
                cluster_arrive();
            }
        }
        return;
    }

    // ---------------------------------------------------------------- this warp's part of every row
    const int cv = (p.C + 7) / 8;
    int v0 = rank * p.vp + warp * p.wv;
    const int v_end = min(cv, (rank + 1) * p.vp);
    const int nv = max(0, min(v_end, v0 + p.wv) - v0);
    if (nv == 0) v0 = 0;
    uint4 *buf = (uint4 *)smem + (size_t)warp * p.ns * per;
    const uint32_t bar0 = smem_u32(smem + L.bars) + 8u * (uint32_t)(warp * p.ns);
    bool dead = false;

    // requests vectors [f, f + n) of this warp's part of row i into buffer s (the caller knows that it is free)
    auto request = [&](int i, int s, int f, int n) {
        const int row = cluster + i * clusters;
        const uint16_t *src = p.z + (size_t)row * p.ldz + (size_t)(v0 + f) * 8;
        uint4 *dst = buf + s * per;
        const int whole = min(n, p.C / 8 - (v0 + f));             // n - 1 where the part ends in a partial vector
        if (BULK) {
            if (lane == 0) {                                      // each use of a buffer completes one phase of its barrier
                if (whole > 0) bulk_in(smem_u32(dst), src, (uint32_t)whole * 16u, bar0 + 8u * (uint32_t)s);
                else mbar_arrive(bar0 + 8u * (uint32_t)s);
            }
            if (whole < n && lane < 8) {
                const int e = (v0 + f + whole) * 8 + lane;
                ((uint16_t *)(dst + whole))[lane] = e < p.C ? src[whole * 8 + lane] : (uint16_t)kNegInf16;
            }
        } else {
            for (int e = lane; e < n * 8; e += 32)
                ((uint16_t *)dst)[e] = (v0 + f) * 8 + e < p.C ? src[e] : (uint16_t)kNegInf16;
        }
        __syncwarp();
    };
    // waits for a buffer's n-th use to be filled
    auto arrived = [&](int s, int use) {
        if (BULK) {
            const bool got = mbar_wait(bar0 + 8u * (uint32_t)s, (uint32_t)(use & 1), (volatile uint32_t *)abort_flag);
            if (!__all_sync(0xFFFFFFFFu, got)) {
                if (lane == 0 && p.kerr && !*abort_flag) atomicCAS(p.kerr, 0u, (uint32_t)KERR_WAIT_FULL | 0x40u | ((uint32_t)blockIdx.x << 8));
                *abort_flag = 1u;
                dead = true;
            }
        }
    };
    // writes vectors [f, f + n) of the gradient of row i from buffer s; always commits a bulk group
    auto send = [&](int i, int s, int f, int n) {
        const int row = cluster + i * clusters;
        uint16_t *dst = p.dz + (size_t)row * p.lddz + (size_t)(v0 + f) * 8;
        const uint4 *src = buf + s * per;
        const int whole = min(n, p.C / 8 - (v0 + f));
        if (BULK) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (whole > 0 && !dead) bulk_out(dst, smem_u32(src), (uint32_t)whole * 16u);
                bulk_commit_group();
            }
            if (whole < n && lane < 8 && !dead) {
                const int e = (v0 + f + whole) * 8 + lane;
                if (e < p.C) dst[whole * 8 + lane] = ((const uint16_t *)(src + whole))[lane];
            }
            __syncwarp();
        } else {
            __syncwarp();
            if (!dead)
                for (int e = lane; e < n * 8; e += 32)
                    if ((v0 + f) * 8 + e < p.C) dst[e] = ((const uint16_t *)src)[e];
            __syncwarp();
        }
    };
    auto publish = [&](int i, const float2 pr) {
        float2 *slot = red + (i & 1) * pairs + rank * p.nw + warp;
        if (p.cl == 1) {
            if (lane == 0) *slot = pr;
        } else if (lane < p.cl) {
            const uint32_t to = mapa_u32(smem_u32(slot), (uint32_t)lane);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(pr.x), "f"(pr.y) : "memory");
        }
        __syncwarp();
    };

    if (!STREAM) {
        // buffer of row i: i % ns.  Three buffers: row i + 2 is on its way while row i + 1 is summed and row i is
        // turned into its gradient.  Two: row i + 2 is requested when row i has left.
        auto first_pass = [&](int i) {
            const int s = i % p.ns;
            if (nv > 0) arrived(s, i / p.ns);
            Run r;
#pragma unroll 4
            for (int j = lane; j < nv; j += 32) run_add8(r, buf[s * per + j], p.k);
            return run_warp(r);
        };
        if (nv > 0) {
            request(0, 0, 0, nv);
            if (n_rows > 1) request(1, 1, 0, nv);
        }
        publish(0, first_pass(0));
        cluster_arrive();
        for (int i = 0; i < n_rows; i++) {
            if (p.ns > 2 && i + 2 < n_rows && nv > 0) {
                if (lane == 0) bulk_wait_group_read<0>();          // row i - 1 has left this buffer (sent an iteration ago)
                __syncwarp();
                request(i + 2, (i + 2) % p.ns, 0, nv);
            }
            float2 next = make_float2(0.0f, 0.0f);
            if (i + 1 < n_rows) next = first_pass(i + 1);
            cluster_wait();
            const float2 pr = row_pair(red + (i & 1) * pairs, pairs);
            const int eb = i % kEntryBuffers;
            const bool alive = live[eb] != 0;
            if (i + 1 < n_rows) {
                publish(i + 1, next);
                cluster_arrive();
            }
            if (p.dz && nv > 0) {
                uint4 *v = buf + (i % p.ns) * per;
                grad_vectors(v, nv, p.k, pr, p.c, alive);
                __syncwarp();
                if (alive) patch_targets((uint16_t *)v, v0 * 8, nv * 8, entries + eb * p.K, p.K, p.k, pr, p.c);
                send(i, i % p.ns, 0, nv);
            }
            if (p.ns == 2 && i + 2 < n_rows && nv > 0) {
                if (lane == 0) bulk_wait_group_read<0>();
                __syncwarp();
                request(i + 2, i % 2, 0, nv);
            }
        }
    } else {
        // Chunks of this warp's part go through a ring of ns buffers in the order in which they are used: the first
        // pass over row 0, then for each row i the first pass over row i + 1 and the second over row i.  Requests run
        // ns - 2 chunks ahead, so a buffer's previous gradient has had one chunk's time to leave.
        const int nch = (nv + per - 1) / per;
        const int passes = p.dz ? 2 : 1;
        const int total = nch * n_rows * passes;
        int asked = 0, used = 0;
        auto ask = [&](int q) {           // chunk q of the sequence
            const int pass = q / nch, ch = q - pass * nch;
            int row;
            if (passes == 1 || pass == 0) row = pass;
            else if (pass == 2 * n_rows - 1) row = n_rows - 1;
            else row = (pass & 1) ? (pass + 1) / 2 : pass / 2 - 1;
            request(row, q % p.ns, ch * per, min(per, nv - ch * per));
        };
        auto ahead = [&]() {
            for (; asked < total && asked < used + p.ns - 1; asked++) {
                if (lane == 0) bulk_wait_group_read<1>();
                __syncwarp();
                ask(asked);
            }
        };
        auto first_pass = [&]() {
            Run r;
            for (int ch = 0; ch < nch; ch++, used++) {
                ahead();
                const int n = min(per, nv - ch * per), s = used % p.ns;
                arrived(s, used / p.ns);
#pragma unroll 4
                for (int j = lane; j < n; j += 32) run_add8(r, buf[s * per + j], p.k);
                __syncwarp();
                if (lane == 0) bulk_commit_group();       // an empty group: every chunk counts as one
            }
            return run_warp(r);
        };
        publish(0, first_pass());
        cluster_arrive();
        for (int i = 0; i < n_rows; i++) {
            float2 next = make_float2(0.0f, 0.0f);
            if (i + 1 < n_rows) next = first_pass();
            cluster_wait();
            const float2 pr = row_pair(red + (i & 1) * pairs, pairs);
            const int eb = i % kEntryBuffers;
            const bool alive = live[eb] != 0;
            if (i + 1 < n_rows) {
                publish(i + 1, next);
                cluster_arrive();
            }
            if (p.dz) {
                for (int ch = 0; ch < nch; ch++, used++) {
                    ahead();
                    const int n = min(per, nv - ch * per), s = used % p.ns;
                    arrived(s, used / p.ns);
                    uint4 *v = buf + s * per;
                    grad_vectors(v, n, p.k, pr, p.c, alive);
                    __syncwarp();
                    if (alive) patch_targets((uint16_t *)v, (v0 + ch * per) * 8, n * 8, entries + eb * p.K, p.K, p.k, pr, p.c);
                    send(i, s, ch * per, n);
                }
            }
        }
    }
    if (lane == 0) {
        bulk_wait_group_read<0>();          // shared memory must outlive the copies that read it
        if (dead) {                         // ... and, after a wait that ran out, those still on their way into it (bounded)
            const unsigned long long t0 = global_ns();
            while (global_ns() - t0 < 1000000ull) {}
        }
    }
}

constexpr uint32_t kSmemLimit = 220u * 1024u;
constexpr int kMaxWarps = 31;

template <bool BULK, bool STREAM>
cudaError_t run(const DistillArgs &p, uint32_t smem, cudaStream_t st)
{
    static bool configured[kMaxDevices] = {};
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    auto kern = k_distill<BULK, STREAM>;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const int threads = (p.nw + 1) * 32;
    int per_sm = 2048 / threads;
    const int by_smem = (int)((227u * 1024u) / (smem + 1024u));
    if (by_smem < per_sm) per_sm = by_smem;
    if (per_sm > 16) per_sm = 16;
    if (per_sm < 1) per_sm = 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cl;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.stream = st;
    cfg.attrs = attr;
    // Clusters the device holds with one CTA on each SM: rows are dealt out statically, so a cluster that had to
    // wait for another to end would double the time.
    static int resident[kMaxDevices][9] = {};       // 0 = not asked yet
    if (resident[dev][p.cl] == 0) {
        cfg.gridDim = dim3((unsigned)(148 / p.cl * p.cl));
        cfg.blockDim = dim3(1024);
        cfg.dynamicSmemBytes = kSmemLimit;
        cfg.numAttrs = 1;
        int n = 0;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kern, &cfg);
        if (e != cudaSuccess) return e;
        if (n < 1) return cudaErrorLaunchOutOfResources;
        resident[dev][p.cl] = n;
    }
    int clusters = resident[dev][p.cl] * per_sm;
    if (clusters > p.B) clusters = p.B;
    cfg.gridDim = dim3((unsigned)(clusters * p.cl));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

// Vectors of a CTA over its warps: as few rounds of 32 lanes as 31 warps allow, then no more warps than that needs.
void split_warps(DistillArgs &p, int vectors_per_cta, int unit)
{
    p.vp = vectors_per_cta;
    const int rounds = (p.vp + kMaxWarps * unit - 1) / (kMaxWarps * unit);
    p.wv = (rounds < 1 ? 1 : rounds) * unit;
    p.nw = (p.vp + p.wv - 1) / p.wv;
}

cudaError_t launch_distill(DistillArgs p, cudaStream_t st)
{
    const bool bulk = (((uintptr_t)p.z | (uintptr_t)p.dz) & 15) == 0 && (p.ldz & 7) == 0 && (!p.dz || (p.lddz & 7) == 0);
    const int cv = (p.C + 7) / 8;
    p.chunk = 0;
    for (p.cl = 1; p.cl <= 8; p.cl *= 2) {
        split_warps(p, (cv + p.cl - 1) / p.cl, 32);
        // few long rows: more SMs per row
        if (p.cl < 8 && (long)p.B * p.cl * 2 <= 148 && p.vp >= 512) continue;
        for (p.ns = 3; p.ns >= 2; p.ns--) {
            const uint32_t smem = layout_of(p.nw, p.ns, p.wv, p.cl, p.K).total;
            if (smem <= kSmemLimit) return bulk ? run<true, false>(p, smem, st) : run<false, false>(p, smem, st);
        }
    }
    p.cl = 8;
    p.chunk = 128;
    p.ns = 4;
    split_warps(p, (cv + 7) / 8, p.chunk);
    uint32_t smem = layout_of(p.nw, p.ns, p.chunk, p.cl, p.K).total;
    if (smem > kSmemLimit) {
        p.ns = 3;
        smem = layout_of(p.nw, p.ns, p.chunk, p.cl, p.K).total;
    }
    return bulk ? run<true, true>(p, smem, st) : run<false, true>(p, smem, st);
}

}  // namespace
}  // namespace mpt

using namespace mpt;

extern "C" int mpt_distill_topk(const uint16_t *z_dev, int ldz, int B, int C, const uint16_t *t16_dev, const int32_t *idx_dev,
                                int ldt, int K, float tau, float S, uint16_t *dz_dev, int lddz, float *row_loss_dev,
                                float *loss_dev, uint32_t *status_dev, void *cuda_stream)
{
    if (!z_dev || !t16_dev || !idx_dev || !row_loss_dev || !loss_dev || z_dev == dz_dev) return MPT_ERR_INVALID_ARG;
    if (!(tau > 0.0f) || !isfinite(tau) || !isfinite(1.4426950408889634f / tau) || !isfinite(S)) return MPT_ERR_INVALID_ARG;
    if (B < 0 || C < 1 || C > MPT_DISTILL_MAX_C || K < 1 || K > MPT_DISTILL_MAX_K) return MPT_ERR_SHAPE;
    if (ldz < C || (dz_dev && lddz < C) || ldt < K) return MPT_ERR_SHAPE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    if (B > 0) {
        DistillArgs p = {};
        p.z = z_dev; p.ldz = (size_t)ldz; p.B = B; p.C = C;
        p.t = t16_dev; p.idx = idx_dev; p.ldt = (size_t)ldt; p.K = K;
        p.k = 1.4426950408889634f / tau;
        p.tau = tau;
        p.c = tau * S / (float)B;
        p.dz = dz_dev; p.lddz = (size_t)lddz;
        p.row_loss = row_loss_dev;
        p.kerr = status_dev;
        e = launch_distill(p, st);
    }
    if (e == cudaSuccess) e = launch_loss_mean(row_loss_dev, B, loss_dev, st);
    return e == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}
