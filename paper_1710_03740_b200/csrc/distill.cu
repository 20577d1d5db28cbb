// Distillation from a teacher's top logits (softmax reductions in FP32 on FP16 logits, gradient multiplied by
// S / B before it is rounded: paper sections 3.2, 3.3).  Per row, with K teacher entries (class, logit):
//
//   q = softmax over the row's entries of t / tau ;  p = softmax over all C classes of z / tau
//   loss = tau^2 sum_j q_j (log q_j - log p_c(j)) ;  dz_v = rn16(tau * (p_v - sum of q_j with c(j) = v) * S / B)
//
// Bound: HBM, 4 bytes a logit (z read once, dz written once).  Three kernels, by the length of a row:
//   up to 2048 classes (and 256 entries): k_distill_rows, a warp a row.
//   up to 32768: k_distill, a row spread over up to 16 warps of a CTA.  Each warp sums the exponentials of its part and turns
// them into the gradient; what warps exchange is one (reference, sum) pair per row, through shared memory and an mbarrier; two
// more warps prepare the teacher's entries rows ahead, a further one moves whole rows in and out by bulk copies.  The
// exponentials stay in registers between the two uses, each lane's relative to its own maximum: one special-function result
// and about 6 instructions a logit (4096 x 32000 102 us = 5.1 TB/s, 2001 x 20011 43 us, 4096 x 32001 without a pitch, where
// every row lies differently to 16-byte boundaries, 117 us).
//   longer: k_distill_stream.  A row passes through shared memory twice, the second time from L2 (first reads are marked to
// stay, second reads and the gradient to leave first), and its exponentials are taken twice (512 x 793471 364 to 389 us); where there
// are few rows, or where that evens out the last round, the CTAs of a cluster share it and exchange the pairs through
// distributed shared memory.
#include <math.h>

#include "distill_plan.h"
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
    int nw;              // warps that hold logits (kTeachers more prepare the teacher's entries)
    int wv;              // vectors of 8 logits per warp
    int cv;              // vectors that a row may touch
    int vp;              // vectors per CTA
    int cl;              // CTAs per cluster
    int ns;              // buffers per warp
    int nb_log2;         // buffers for a row's entries: 2^nb_log2
    int per;             // vectors per buffer: wv, or a chunk of it where rows are streamed
    int kept;            // the teacher's classes' logits are kept with the entries (else the row's loss reads them again)
    int same;            // rows of dz lie to 16-byte boundaries as those of z do
};

// Rows are worked on in the 16-byte vectors that they lie in: vector g of row r holds classes 8 g - shift ... + 7, what lies
// before class 0 and behind the last counts as -inf.  A SHIFT of zero for all rows is known at compile time.
template <bool SHIFT>
__device__ __forceinline__ int shift_of(const DistillArgs &p, int row)
{
    return SHIFT ? (int)((((uintptr_t)p.z >> 1) + (size_t)row * p.ldz) & 7) : 0;
}

// A row's teacher entries in shared memory, each array K long: class (-1: none), teacher's probability, the student's
// logit (kept by the warp that holds it while the gradient takes its place), and the teacher's probability of the class
// (q, or of all entries that name it).
// The entries of the classes that warp w of this CTA holds are order[first[w]] ... order[first[w + 1] - 1].
struct Entries {
    int32_t *v;
    float *q, *z, *sum;
    int32_t *order, *first;
};
constexpr int kEntryWords = 5;       // 32-bit words an entry takes
constexpr int kPairBuffers = 4;      // a warp publishes row i + 1 when all have finished with row i - 3
constexpr int kNoClass = -1;
constexpr int kTeachers = 2;         // warps that prepare the teacher's entries, every kTeachers-th row each
constexpr unsigned kNap = 64;        // ns
constexpr int kAhead = 4;            // rows of its own a teacher warp asks for ahead
constexpr int kMaxWarps = 16;        // warps that hold logits: few, so that what each does once per row stays small
constexpr int kMinRounds = 4, kMaxRounds = 8;      // vectors a lane keeps in registers
constexpr int kHalfWarps = 8;        // CTAs of so many warps with logits are compiled to fit twice on an SM
constexpr int kChunk = 256;          // vectors of a buffer where rows are streamed
constexpr int kMaxBatch = 1 << 30;   // what is added to row indexes stays inside 32 bits
constexpr uint32_t kNegInf16 = 0xFC00u;

__device__ __forceinline__ float h2f(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }
__device__ __forceinline__ uint32_t f2h(float x) { return (uint32_t)__half_as_ushort(__float2half_rn(x)); }
__device__ __forceinline__ float wsum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float wmax(float v)      // NaN operands are dropped, as by fmaxf
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// Running sum of a lane: sum of 2^(z k + b) with b = -max * k as it was rounded, so the pair says exactly what
// was added up.  max = -inf: nothing but -inf (or NaN, which then is in s) so far, b = 0.
struct Run {
    float m = -INFINITY, b = 0.0f, s = 0.0f;
};
__device__ __forceinline__ __half2 max8(const uint4 x)
{
    return __hmax2(__hmax2(*(const __half2 *)&x.x, *(const __half2 *)&x.y), __hmax2(*(const __half2 *)&x.z, *(const __half2 *)&x.w));
}
// N vectors at once: one comparison with the running maximum for all of them.
template <int N>
__device__ __forceinline__ void run_add(Run &r, const uint4 (&x)[N], float k)
{
    __half2 mx = max8(x[0]);
#pragma unroll
    for (int u = 1; u < N; u++) mx = __hmax2(mx, max8(x[u]));
    const float m = fmaxf(__low2float(mx), __high2float(mx));       // NaN is dropped here and comes back in the sum
    if (m > r.m) {
        const float b = -__fmul_rn(m, k);
        r.s = r.m == -INFINITY ? r.s : r.s * ex2_approx(b - r.b);
        r.m = m;
        r.b = b;
    }
    float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < N; u++) {
        const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const float2 f = __half22float2(*(const __half2 *)&w[q]);
            a[q] += ex2_approx(fmaf(f.x, k, r.b));
            a[q] += ex2_approx(fmaf(f.y, k, r.b));
        }
    }
    r.s += (a[0] + a[1]) + (a[2] + a[3]);
}
// n vectors of shared memory, lane by lane; the warp's rounds of 32 go four at a time
__device__ __forceinline__ void run_vectors(Run &r, const uint4 *v, int n, float k)
{
    const int lane = threadIdx.x & 31;
    int base = 0;
    for (; base + 128 <= n; base += 128) {
        const uint4 *s = v + base + lane;
        const uint4 x[4] = {s[0], s[32], s[64], s[96]};
        run_add<4>(r, x, k);
    }
    if (base + 64 <= n) {
        const uint4 *s = v + base + lane;
        const uint4 x[2] = {s[0], s[32]};
        run_add<2>(r, x, k);
        base += 64;
    }
    for (int j = base + lane; j < n; j += 32) {
        const uint4 x[1] = {v[j]};
        run_add<1>(r, x, k);
    }
}
// The warp's pair from its lanes': reference e (terms are relative to 2^e), sum.  A lane with e = -inf has nothing or NaN
// to add.
__device__ __forceinline__ float2 warp_pair(float e, float s)
{
    const float E = wmax(e);
    return make_float2(E, wsum(e == -INFINITY ? s : s * ex2_approx(e - E)));
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

// Eight neighbouring gradients of a row to global memory, the first of class `first`; whole: dst is 16-byte aligned
// (always, unless SHIFT).
template <bool SHIFT>
__device__ __forceinline__ void store8(uint16_t *dst, const uint4 v, int first, int C, bool whole)
{
    if ((!SHIFT || (whole && first >= 0)) && first + 8 <= C) {
        __stcs((uint4 *)dst, v);
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 8; e++)
        if ((unsigned)(first + e) < (unsigned)C) dst[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
}
// Gradient of n vectors, 2^(z k - x) * cs with cs = tau S / (B y), from shared memory to dst (class `first` on).
template <int N, bool SHIFT>
__device__ __forceinline__ void grad_store(const uint4 *v, uint16_t *dst, int first, int C, bool whole, float k, float x, float cs)
{
    uint4 in[N];
#pragma unroll
    for (int u = 0; u < N; u++) in[u] = v[32 * u];
#pragma unroll
    for (int u = 0; u < N; u++) {
        const uint32_t w[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const float2 f = __half22float2(*(const __half2 *)&w[q]);
            o[q] = pack_f16x2(ex2_approx(fmaf(f.x, k, -x)) * cs, ex2_approx(fmaf(f.y, k, -x)) * cs);
        }
        store8<SHIFT>(dst + 256 * u, make_uint4(o[0], o[1], o[2], o[3]), first + 256 * u, C, whole);
    }
}
template <bool SHIFT>
__device__ __forceinline__ void grad_vectors(const uint4 *v, int n, uint16_t *dst, int first, int C, bool whole, float k, float2 pr, float cs)
{
    const int lane = threadIdx.x & 31;
    int base = 0;
    for (; base + 128 <= n; base += 128) grad_store<4, SHIFT>(v + base + lane, dst + (base + lane) * 8, first + (base + lane) * 8, C, whole, k, pr.x, cs);
    if (base + 64 <= n) {
        grad_store<2, SHIFT>(v + base + lane, dst + (base + lane) * 8, first + (base + lane) * 8, C, whole, k, pr.x, cs);
        base += 64;
    }
    for (int j = base + lane; j < n; j += 32) grad_store<1, SHIFT>(v + j, dst + j * 8, first + j * 8, C, whole, k, pr.x, cs);
}
// The teacher's classes among the logits [first, first + count) that warp w holds at h: keep their logits ...
__device__ __forceinline__ void keep_targets(const uint16_t *h, int first, int count, const Entries &ent, int w)
{
    for (int j = ent.first[w] + (int)(threadIdx.x & 31); j < ent.first[w + 1]; j += 32) {
        const int i = ent.order[j], at = ent.v[i] - first;
        if ((unsigned)at < (unsigned)count) ent.z[i] = h2f(h[at]);
    }
}
// ... and, when the warp has written the gradients of these classes at dst, write theirs again with the teacher's
// probability of the class subtracted (an entry named twice is written twice, alike).
__device__ __forceinline__ void patch_targets(uint16_t *dst, int first, int count, const Entries &ent, int w, float k, float2 pr, float cs, float c)
{
    for (int j = ent.first[w] + (int)(threadIdx.x & 31); j < ent.first[w + 1]; j += 32) {
        const int i = ent.order[j], at = ent.v[i] - first;
        if ((unsigned)at < (unsigned)count)
            dst[at] = (uint16_t)f2h(fmaf(ex2_approx(fmaf(ent.z[i], k, -pr.x)), cs, -ent.sum[i] * c));
    }
}

// The first entries of a row's list, asked for ahead of their use.
struct ListAhead {
    static constexpr int N = 4;          // a lane
    int v[N];
    uint16_t t[N];
    __device__ __forceinline__ void ask(const DistillArgs &p, int row)
    {
        const size_t at = (size_t)row * p.ldt;
#pragma unroll
        for (int c = 0; c < N; c++) {
            const int j = (int)(threadIdx.x & 31) + 32 * c;
            v[c] = j < p.K ? p.idx[at + j] : kNoClass;
            t[c] = j < p.K ? p.t[at + j] : (uint16_t)kNegInf16;
        }
    }
};
// Teacher's entries of a row, by one warp.  Entries whose class is outside [0, C) or whose logit is -inf have no part;
// returns whether any has.  `rank`: which CTA of the cluster this is.
// Classes named more than once are found with a hash table (open addressing, `slots` words, a
// power of two and at least 2 K); only theirs are added up, over the entries in order.
__device__ __forceinline__ bool prepare_entries(const DistillArgs &p, int row, int rank, int shift, const ListAhead &ahead, const Entries &ent, int *table,
                                                int slots)
{
    const int lane = threadIdx.x & 31;
    const int32_t *id = p.idx + (size_t)row * p.ldt;
    const uint16_t *tt = p.t + (size_t)row * p.ldt;
    for (int i = lane; i < slots; i += 32) table[i] = kNoClass;
    if (lane < kMaxWarps) ent.first[lane] = 0;
    float top = -INFINITY;
    bool any = false;
    __syncwarp();
    auto enter = [&](int j, int v, uint16_t t16) {
        const float t = h2f(t16);
        const bool ok = v >= 0 && v < p.C && t != -INFINITY;
        ent.v[j] = ok ? v : kNoClass;
        ent.q[j] = t;
        if (ok) top = fmaxf(top, t);
        any |= ok;
    };
#pragma unroll
    for (int c = 0; c < ListAhead::N; c++)
        if (lane + 32 * c < p.K) enter(lane + 32 * c, ahead.v[c], ahead.t[c]);
#pragma unroll 4
    for (int j = lane + 32 * ListAhead::N; j < p.K; j += 32) enter(j, id[j], tt[j]);
    top = wmax(top);
    float s = 0.0f;
    bool twice = false;
    // the warp of this CTA that holds class v, kMaxWarps: none
    auto holder = [&](int v) {
        const int at = ((v + shift) >> 3) - rank * p.vp;
        return v >= 0 && at >= 0 && at < p.vp ? at / p.wv : kMaxWarps;
    };
    for (int j = lane; j < p.K; j += 32) {
        const int v = ent.v[j];
        const int hw = holder(v);
        if (hw < kMaxWarps) ent.sum[j] = __int_as_float(atomicAdd(ent.first + hw, 1));      // its place in the warp's list
        float w = 0.0f;
        if (v >= 0) {
            w = ex2_approx((ent.q[j] - top) * p.k);
            for (unsigned h = (unsigned)v * 2654435761u;; h += 1u << 21) {      // the top 11 bits choose the slot
                const int was = atomicCAS(table + ((h >> 21) & (unsigned)(slots - 1)), kNoClass, v);
                if (was == kNoClass) break;
                if (was == v) {
                    twice = true;
                    break;
                }
            }
        }
        ent.q[j] = w;
        s += w;
    }
    s = wsum(s);
    __syncwarp();
    const int n = lane < kMaxWarps ? ent.first[lane] : 0;
    int before = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xFFFFFFFFu, before, o);
        if (lane >= o) before += up;
    }
    __syncwarp();
    if (lane <= kMaxWarps) ent.first[lane] = before - n;      // lane kMaxWarps: all of them
    __syncwarp();
    const float inv = __fdiv_rn(1.0f, s);
    for (int j = lane; j < p.K; j += 32) {
        const int hw = holder(ent.v[j]);
        if (hw < kMaxWarps) ent.order[ent.first[hw] + __float_as_int(ent.sum[j])] = j;
        const float q = ent.v[j] >= 0 ? ent.q[j] * inv : 0.0f;
        ent.q[j] = q;
        ent.sum[j] = q;
    }
    __syncwarp();
    if (__any_sync(0xFFFFFFFFu, twice)) {
        for (int j = lane; j < p.K; j += 32) {
            const int v = ent.v[j];
            float q = 0.0f;
            for (int i = 0; i < p.K; i++)
                if (ent.v[i] == v) q += ent.q[i];
            ent.sum[j] = q;
        }
        __syncwarp();
    }
    return __any_sync(0xFFFFFFFFu, any);
}
__device__ __forceinline__ void write_loss(const DistillArgs &p, int row, const Entries &ent, bool live, float2 pr)
{
    const int lane = threadIdx.x & 31;
    constexpr float LN2 = 0.69314718055994531f;
    const float l2s = log2f(pr.y);
    const uint16_t *zr = p.z + (size_t)row * p.ldz;
    float l = 0.0f;
#pragma unroll 4
    for (int j = lane; j < p.K; j += 32) {
        const float q = ent.q[j];
        const int v = ent.v[j];
        // log2 q - log2 p; a probability of zero (or none) adds nothing
        if (v >= 0 && !(q == 0.0f)) {
            const float z = p.kept ? ent.z[j] : h2f(zr[v]);
            l += q * ((log2f(q) + l2s) - fmaf(z, p.k, -pr.x));
        }
    }
    l = wsum(l);
    if (lane == 0) p.row_loss[row] = live ? l * LN2 * p.tau * p.tau : 0.0f;
}

// Bulk copies with an L2 eviction priority (l2_policy)
__device__ __forceinline__ void bulk_in(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy)
{
    mbar_arrive_expect_tx(bar, bytes);
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void bulk_out(void *dst, uint32_t src, uint32_t bytes, uint64_t policy)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group.L2::cache_hint [%0], [%1], %2, %3;" ::"l"(dst), "r"(src), "r"(bytes),
                 "l"(policy)
                 : "memory");
}

// Shared memory: buffers [nw][ns][per] of 16-byte vectors | entries [nb] | mbarriers: [nw][ns] of the buffers, [4] of
// the pairs, 2 x [nb] of the entries (full, empty) | pairs [4][cl * nw] | hash tables [teachers] | the row's pair [nb] |
// live [nb] | abort word
// mbarriers of the buffers: one per warp and buffer, or two per buffer where a warp of its own moves whole rows
__host__ __device__ inline int buffer_bars(int nw, int ns) { return (nw < 2 ? 2 : nw) * ns; }
struct Layout {
    uint32_t ent, bars, red, table, pair, live, abort, total;
    int slots;
};
__host__ __device__ inline Layout layout_of(int nw, int ns, int per, int cl, int K, int nb)
{
    Layout l;
    uint32_t at = (uint32_t)nw * (uint32_t)ns * (uint32_t)per * 16u;
    l.ent = at;
    at += (uint32_t)nb * ((uint32_t)K * kEntryWords + kMaxWarps + 1u) * 4u;
    at = (at + 7u) & ~7u;
    l.bars = at;
    at += ((uint32_t)buffer_bars(nw, ns) + (uint32_t)kPairBuffers + 2u * (uint32_t)nb) * 8u;
    l.red = at;
    at += (uint32_t)kPairBuffers * (uint32_t)cl * (uint32_t)nw * 8u;
    l.slots = 32;
    while (l.slots < 2 * K) l.slots *= 2;
    l.table = at;
    at += (uint32_t)kTeachers * 4u * (uint32_t)l.slots;
    l.pair = at;
    at += 8u * (uint32_t)nb;
    l.live = at;
    at += 4u * (uint32_t)nb;
    l.abort = at;
    at += 4u;
    l.total = (at + 15u) & ~15u;
    return l;
}

// Bounded wait that sleeps between its tries: a warp that polls takes the issue slots of those that work (and of the
// teacher's warps above all, which everybody then waits for longer).
template <bool CLUSTER>
static __device__ __noinline__ bool wait_asleep(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag)
{
    unsigned long long t0 = 0;
    for (uint32_t it = 0;; ++it) {
        __nanosleep(kNap);
        if (CLUSTER ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity)) return true;
        if ((it & 63u) == 63u) {
            if (*abort_flag) return false;
            const unsigned long long now = global_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > WAIT_LIMIT_NS) return false;
        }
    }
}

// What all warps of a CTA share, and each warp's part of the rows.  ROWS: the CTA's part of a row lies in one buffer of [ns]
// and moves as one copy, in and out, by a warp that does nothing else: what a warp spends on issuing its own copies it spends
// once a row, and all others wait for the slowest.  Otherwise each warp has ns buffers of its own.
template <bool SHIFT, bool ROWS>
struct Cta {
    const DistillArgs &p;
    uint8_t *smem;
    Layout L;
    int warp, lane, rank, cluster, clusters, n_rows, pairs;
    uint32_t bars;
    volatile uint32_t *abort_flag;
    bool dead = false;
    // this warp's part: vectors [v0, v0 + nv) of a row, its buffers and their mbarriers
    int v0, nv;
    uint4 *buf;
    int pitch;           // vectors from one buffer to the next
    uint32_t bar0;

    __device__ __forceinline__ Cta(const DistillArgs &args, uint8_t *s) : p(args), smem(s), L(layout_of(args.nw, args.ns, args.per, args.cl, args.K, 1 << args.nb_log2))
    {
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        rank = !ROWS && p.cl > 1 ? (int)cluster_ctarank() : 0;      // ROWS: no clusters
        cluster = (int)blockIdx.x / p.cl;
        clusters = (int)gridDim.x / p.cl;
        n_rows = cluster < p.B ? (p.B - 1 - cluster) / clusters + 1 : 0;
        pairs = p.cl * p.nw;
        bars = smem_u32(smem + L.bars);
        abort_flag = (volatile uint32_t *)(smem + L.abort);
        const int v_end = min(p.cv, (rank + 1) * p.vp);
        v0 = rank * p.vp + warp * p.wv;
        nv = warp < p.nw ? max(0, min(v_end, v0 + p.wv) - v0) : 0;
        if (nv == 0) v0 = 0;
        buf = (uint4 *)smem + (ROWS ? (size_t)warp * p.wv : (size_t)warp * p.ns * p.per);
        pitch = ROWS ? p.nw * p.wv : p.per;
        bar0 = ROWS ? bars : bars + 8u * (uint32_t)(warp * p.ns);
        if (!ROWS && warp < p.nw && lane == 0)
            for (int i = 0; i < p.ns; i++) mbar_init(bar0 + 8u * (uint32_t)i, 1);
        if (ROWS && threadIdx.x == 0)
            for (int i = 0; i < p.ns; i++) {
                mbar_init(bar0 + 8u * (uint32_t)i, 1);                        // the row has arrived
                mbar_init(written_bar(i), (uint32_t)p.nw);                    // every warp has put its gradient in its place
            }
        if (threadIdx.x == 0) {
            for (int i = 0; i < kPairBuffers; i++) mbar_init(pair_bar(i), (uint32_t)pairs);
            for (int b = 0; b < 1 << p.nb_log2; b++) {
                mbar_init(full_bar(b), 1);
                mbar_init(empty_bar(b), (uint32_t)p.nw);
            }
            *abort_flag = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (p.cl > 1) cluster_sync_all();   // every CTA of the cluster has its barriers before anything arrives there
    }
    __device__ __forceinline__ uint32_t pair_bar(int i) const { return bars + 8u * (uint32_t)(buffer_bars(p.nw, p.ns) + (i & (kPairBuffers - 1))); }
    __device__ __forceinline__ uint32_t full_bar(int b) const { return bars + 8u * (uint32_t)(buffer_bars(p.nw, p.ns) + kPairBuffers + b); }
    __device__ __forceinline__ uint32_t empty_bar(int b) const { return full_bar(b) + (8u << p.nb_log2); }
    __device__ __forceinline__ uint32_t written_bar(int s) const { return bars + 8u * (uint32_t)(p.ns + s); }
    __device__ __forceinline__ Entries entries(int b) const
    {
        float *at = (float *)(smem + L.ent) + b * (kEntryWords * p.K + kMaxWarps + 1);
        return {(int32_t *)at, at + p.K, at + 2 * p.K, at + 3 * p.K, (int32_t *)(at + 4 * p.K), (int32_t *)(at + 5 * p.K)};
    }
    __device__ __forceinline__ float2 *pair_of(int b) const { return (float2 *)(smem + L.pair) + b; }
    __device__ __forceinline__ int *live(int b) const { return (int *)(smem + L.live) + b; }
    __device__ __forceinline__ float2 *red(int i) const { return (float2 *)(smem + L.red) + (i & (kPairBuffers - 1)) * pairs; }
    __device__ __forceinline__ int row_of(int i) const { return cluster + i * clusters; }

    // A wait of the whole warp; one that runs out ends all later ones of this CTA at once.
    template <bool CLUSTER>
    __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity)
    {
        bool got = CLUSTER ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity);
        if (!got) got = wait_asleep<CLUSTER>(bar, parity, abort_flag);
        if (!__all_sync(0xFFFFFFFFu, got)) {
            if (lane == 0 && p.kerr && !*abort_flag) atomicCAS(p.kerr, 0u, (uint32_t)KERR_WAIT_FULL | 0x40u | ((uint32_t)blockIdx.x << 8));
            *abort_flag = 1u;
            dead = true;
        }
    }
    __device__ __forceinline__ int shift(int i) const { return shift_of<SHIFT>(p, row_of(i)); }
    // The class of the first element of this warp's part of row i.
    __device__ __forceinline__ int first_class(int i) const { return v0 * 8 - shift(i); }
    // What lies before the row's first class or behind its last becomes -inf, in vectors [f, f + n) of this warp's part.
    __device__ __forceinline__ void mend(int i, int s, int f, int n)
    {
        const int sh = shift(i), g0 = v0 + f;
        uint16_t *h = (uint16_t *)(buf + s * pitch);
        const bool head = SHIFT && g0 == 0, tail = (g0 + n) * 8 - sh > p.C;
        if (head && lane < sh) h[lane] = (uint16_t)kNegInf16;
        if (tail) {                                  // the last vector, with a shift perhaps one more
            for (int g = SHIFT ? max((p.C + sh) / 8, g0) : g0 + n - 1; g < g0 + n; g++)
                if (lane < 8 && g * 8 - sh + lane >= p.C) h[(g - g0) * 8 + lane] = (uint16_t)kNegInf16;
        }
        if (head || tail) {
            refilled_later();
            __syncwarp();
        }
    }
    // After ordinary stores into a buffer, by the lanes that made them: the bulk copy that refills it comes after them.
    __device__ __forceinline__ static void refilled_later() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
    // Vectors [first, first + n) of row i to dst, which is free; `bar` completes a phase with them.  A vector that is not the
    // row's alone comes with what lies beside the row (mend() replaces that); one that reaches out of the matrix's memory,
    // by elements.
    __device__ __forceinline__ void bring(int i, uint4 *dst, int first, int n, uint32_t bar, uint64_t policy)
    {
        const int row = row_of(i), sh = shift(i);
        const uint16_t *src = p.z + (size_t)row * p.ldz;
        int a = 0, b = n;
        if (SHIFT) {
            const int lo = (size_t)row * p.ldz < (size_t)sh ? 1 : 0;
            const int hi = (p.C + sh + ((size_t)(p.B - 1 - row) * p.ldz >= 7 ? 7 : 0)) / 8;
            a = min(max(lo - first, 0), n);
            b = max(min(hi - first, n), a);
        } else if (row == p.B - 1) b = max(min(n, p.C / 8 - first), 0);
        auto elements = [&](int g) {
            const int c = (first + g) * 8 - sh + lane;
            if (lane < 8) ((uint16_t *)(dst + g))[lane] = (unsigned)c < (unsigned)p.C ? src[c] : (uint16_t)kNegInf16;
        };
        if (a > 0 || b < n) {
            for (int g = 0; g < a; g++) elements(g);
            for (int g = b; g < n; g++) elements(g);
            refilled_later();
            __syncwarp();                            // the arrival below tells of these, too
        }
        if (lane == 0) {
            if (b > a) bulk_in(smem_u32(dst + a), src + ((ptrdiff_t)(first + a) * 8 - sh), (uint32_t)(b - a) * 16u, bar, policy);
            else mbar_arrive(bar);
        }
        __syncwarp();
    }
    // Requests vectors [f, f + n) of this warp's part of row i into buffer s (the caller knows that it is free).
    __device__ __forceinline__ void request(int i, int s, int f, int n, uint64_t policy)
    {
        bring(i, buf + s * pitch, v0 + f, n, bar0 + 8u * (uint32_t)s, policy);
    }
    __device__ __forceinline__ void arrived(int s, uint32_t parity) { wait<false>(bar0 + 8u * (uint32_t)s, parity); }
    // ROWS: the work of the last warp.  Every buffer goes round: a row arrives, its gradient takes its place, leaves, and the
    // row ns further arrives.
    __device__ __forceinline__ void move_rows()
    {
        const uint64_t policy = l2_policy(2);        // every byte is used once
        const int first = rank * p.vp, n = max(0, min(p.cv, first + p.vp) - first);
        auto fetch = [&](int i, int s) { bring(i, (uint4 *)smem + s * pitch, first, n, bar0 + 8u * (uint32_t)s, policy); };
        for (int i = 0; i < p.ns && i < n_rows; i++) fetch(i, i);
        int s = 0;
        uint32_t parity = 0;
        for (int i = 0; i < n_rows; i++) {
            wait<false>(written_bar(s), parity);
            if (p.dz && lane == 0) {
                // the row's own vectors; the owner of a vector that it shares stores its elements itself
                const int sh = shift(i), a = max(sh > 0 ? 1 : 0, first), b = min((p.C + sh) / 8, first + n);
                if (b > a && p.same && !dead)
                    bulk_out(p.dz + (size_t)row_of(i) * p.lddz + ((size_t)a * 8 - sh), smem_u32((uint4 *)smem + s * pitch + (a - first)),
                             (uint32_t)(b - a) * 16u, policy);
                bulk_commit_group();
                bulk_wait_group_read<0>();
            }
            __syncwarp();
            if (i + p.ns < n_rows) fetch(i + p.ns, s);
            if (++s == p.ns) {
                s = 0;
                parity ^= 1u;
            }
        }
    }
    // ROWS: this warp's gradient of row i is in its place in buffer s.
    __device__ __forceinline__ void written(int i, int s)
    {
        if (p.dz) {
            if (SHIFT && !p.same) send(i, s);
            else if (nv > 0 && !dead && (SHIFT || (v0 + nv) * 8 > p.C)) {
                __syncwarp();                        // all lanes' gradients are there
                const int sh = shift(i), last = (p.C + sh) / 8;
                auto elements = [&](int g) {
                    if (g < v0 || g >= v0 + nv || lane >= 8) return;
                    const int c = g * 8 - sh + lane;
                    if ((unsigned)c < (unsigned)p.C) (p.dz + (size_t)row_of(i) * p.lddz)[c] = ((const uint16_t *)(buf + s * pitch + (g - v0)))[lane];
                };
                if (SHIFT && sh > 0) elements(0);
                if (last > 0 || sh == 0) elements(last);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(written_bar(s));
    }
    // Writes this warp's gradient of row i from buffer s, element by element.
    __device__ __forceinline__ void send(int i, int s)
    {
        uint16_t *dst = p.dz + (size_t)row_of(i) * p.lddz;
        const uint16_t *src = (const uint16_t *)(buf + s * pitch);
        const int first = first_class(i);
        __syncwarp();
        if (!dead)
            for (int e = lane; e < nv * 8; e += 32)
                if ((unsigned)(first + e) < (unsigned)p.C) dst[first + e] = src[e];
        __syncwarp();
    }
    // Where this warp's gradient of row i goes (its first vector's place, which may begin before the row).
    __device__ __forceinline__ uint16_t *out(int i) const { return p.dz + (ptrdiff_t)((size_t)row_of(i) * p.lddz) + first_class(i); }
    // Zeros for this warp's part of a row without a teacher.
    __device__ __forceinline__ void send_zeros(int i)
    {
        for (int j = lane; j < nv; j += 32) store8<SHIFT>(out(i) + j * 8, make_uint4(0u, 0u, 0u, 0u), first_class(i) + j * 8, p.C, p.same);
    }
    // This warp's pair of row i to every CTA of the cluster.
    __device__ __forceinline__ void publish(int i, float2 pr)
    {
        float2 *slot = red(i) + rank * p.nw + warp;
        if (ROWS || p.cl == 1) {
            if (lane == 0) {
                *slot = pr;
                mbar_arrive(pair_bar(i));
            }
        } else if (lane < p.cl) {
            const uint32_t to = mapa_u32(smem_u32(slot), (uint32_t)lane);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(pr.x), "f"(pr.y) : "memory");
            mbar_arrive_cluster(mapa_u32(pair_bar(i), (uint32_t)lane));
        }
        __syncwarp();
    }
    // The row's pair, once all warps have published theirs.
    __device__ __forceinline__ float2 collect(int i)
    {
        const uint32_t parity = (uint32_t)(i / kPairBuffers) & 1u;
        if (ROWS || p.cl == 1) wait<false>(pair_bar(i), parity);
        else wait<true>(pair_bar(i), parity);
        return row_pair(red(i), pairs);
    }
    // The teacher's entries of row i.
    __device__ __forceinline__ int open_entries(int i)
    {
        const int b = i & ((1 << p.nb_log2) - 1);
        wait<false>(full_bar(b), (uint32_t)(i >> p.nb_log2) & 1u);
        return b;
    }
    // ... are not needed any more by this warp; with them goes what the row's loss needs of the row.
    __device__ __forceinline__ void close_entries(int b, float2 pr)
    {
        if (warp == 0 && lane == 0) *pair_of(b) = pr;
        __syncwarp();
        if (lane == 0) mbar_arrive(empty_bar(b));
    }
    // Row i's list on its way to L2: with all SMs' copies queued at the memory a load takes longer than a row.
    __device__ __forceinline__ void prefetch_list(int i)
    {
        if (i >= n_rows) return;
        const size_t at = (size_t)row_of(i) * p.ldt;
        for (int j = lane * 32; j < p.K; j += 1024) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.idx + at + j));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.t + at + j));
        }
    }
    // The work of the last kTeachers warps: the entries of every kTeachers-th row, as far ahead as there are buffers, and
    // the row's loss when a buffer comes back.
    __device__ __forceinline__ void teach()
    {
        const int me = warp - p.nw, nb = 1 << p.nb_log2;
        ListAhead ahead;
        if (me < n_rows) ahead.ask(p, row_of(me));
        for (int r = 1; r < kAhead; r++) prefetch_list(me + r * kTeachers);
        for (int i = me; i < n_rows + nb; i += kTeachers) {
            const int b = i & (nb - 1);
            const uint32_t parity = ((uint32_t)(i >> p.nb_log2) & 1u) ^ 1u;
            // this wait is long and nothing hurries: sleep between the tries, the issue slots belong to the others
            for (int tries = 0; tries < 1000000 && !mbar_try_wait(empty_bar(b), parity) && !*abort_flag; tries++) __nanosleep(200);
            wait<false>(empty_bar(b), parity);
            if (i >= nb && rank == 0 && !dead) write_loss(p, row_of(i - nb), entries(b), *live(b) != 0, *pair_of(b));
            if (i < n_rows) {
                __syncwarp();
                prefetch_list(i + kAhead * kTeachers);
                const bool any = prepare_entries(p, row_of(i), rank, shift(i), ahead, entries(b), (int *)(smem + L.table) + me * L.slots, L.slots);
                if (lane == 0) {
                    *live(b) = any ? 1 : 0;
                    mbar_arrive(full_bar(b));
                }
                if (i + kTeachers < n_rows) ahead.ask(p, row_of(i + kTeachers));      // arrives while this warp waits
            }
        }
    }
    // Common end: shared memory outlives the copies that read it, those still on their way into it after a wait that
    // ran out (for a bounded time), and the other CTAs' stores.
    __device__ __forceinline__ void leave()
    {
        if (lane == 0) {
            bulk_wait_group_read<0>();
            if (dead) {
                const unsigned long long t0 = global_ns();
                while (global_ns() - t0 < 1000000ull) {}
            }
        }
        __syncwarp();
        if (p.cl > 1) cluster_sync_all();
    }
};

// Rows whose exponentials stay in registers: R vectors per lane.
// HALF: for CTAs of at most kHalfWarps (+ 3) warps, with the registers that let two of them reside on an SM; the rows of the
// two hide each other's waits (5000 x 8000 79 -> 52 us; with 16 warps the fewer registers cost more: 5000 x 16000 92 -> 112).
template <int R, bool SHIFT, bool HALF>
__global__ void __launch_bounds__((HALF ? 2 * (kHalfWarps + kTeachers + 1) : kMaxWarps + kTeachers + 1) * 32, 1) k_distill(const DistillArgs p)
{
    pdl_trigger();
    extern __shared__ __align__(128) uint8_t smem[];
    Cta<SHIFT, true> c(p, smem);
    pdl_wait();                                       // up to here nothing was read or written that another kernel knows of
    if (c.warp >= p.nw) {
        if (c.warp < p.nw + kTeachers) c.teach();
        else c.move_rows();
        c.leave();
        return;
    }
    const int nv = c.nv;
    int s_use = 0;
    uint32_t parity = 0;
    for (int i = 0; i < c.n_rows; i++) {
        uint4 *v = c.buf + s_use * c.pitch;
        float e[R][8];
        float m = -INFINITY, b = 0.0f, s = 0.0f;
        if (nv > 0) {
            c.arrived(s_use, parity);
            c.mend(i, s_use, 0, nv);
            uint4 x[R];
            __half2 mx = __half2half2(__ushort_as_half((unsigned short)kNegInf16));
#pragma unroll
            for (int u = 0; u < R; u++) {
                const int j = c.lane + 32 * u;
                x[u] = j < nv ? v[j] : make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u);
                mx = __hmax2(mx, max8(x[u]));
            }
            m = fmaxf(__low2float(mx), __high2float(mx));           // NaN is dropped here and comes back in the sum
            b = m == -INFINITY ? 0.0f : -__fmul_rn(m, p.k);
            float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < R; u++) {
                const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const float2 f = __half22float2(*(const __half2 *)&w[q]);
                    e[u][2 * q] = ex2_approx(fmaf(f.x, p.k, b));
                    e[u][2 * q + 1] = ex2_approx(fmaf(f.y, p.k, b));
                    a[q] += e[u][2 * q] + e[u][2 * q + 1];
                }
            }
            s = (a[0] + a[1]) + (a[2] + a[3]);
        }
        c.publish(i, warp_pair(m == -INFINITY ? -INFINITY : -b, s));
        const int eb = c.open_entries(i);
        const Entries ent = c.entries(eb);
        if (nv > 0) keep_targets((const uint16_t *)v, c.first_class(i), nv * 8, ent, c.warp);
        __syncwarp();
        const float2 pr = c.collect(i);
        if (p.dz && nv > 0) {
            const float cs = __fdiv_rn(p.c, pr.y);
            if (*c.live(eb)) {
                // this lane's exponentials are relative to 2^-b: a lane of nothing but -inf has zeros (or NaN)
                const float k = m == -INFINITY ? cs * 0.0f : cs * ex2_approx(-b - pr.x);
#pragma unroll
                for (int u = 0; u < R; u++) {
                    const int j = c.lane + 32 * u;
                    if (j < nv)
                        v[j] = make_uint4(pack_f16x2(e[u][0] * k, e[u][1] * k), pack_f16x2(e[u][2] * k, e[u][3] * k),
                                          pack_f16x2(e[u][4] * k, e[u][5] * k), pack_f16x2(e[u][6] * k, e[u][7] * k));
                }
                __syncwarp();
                patch_targets((uint16_t *)v, c.first_class(i), nv * 8, ent, c.warp, p.k, pr, cs, p.c);
            } else {
                for (int j = c.lane; j < nv; j += 32) v[j] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
        c.written(i, s_use);
        c.close_entries(eb, pr);
        if (++s_use == p.ns) {
            s_use = 0;
            parity ^= 1u;
        }
    }
    c.leave();
}

// Rows that are read twice.  Chunks of this warp's part go through a ring of ns buffers in the order in which they are
// used, first pass and second pass of one row after the other, requested ns - 1 ahead.
template <bool SHIFT>
__global__ void __launch_bounds__((kMaxWarps + kTeachers) * 32, 1) k_distill_stream(const DistillArgs p)
{
    pdl_trigger();
    extern __shared__ __align__(128) uint8_t smem[];
    Cta<SHIFT, false> c(p, smem);
    pdl_wait();                                       // up to here nothing was read or written that another kernel knows of
    if (c.warp >= p.nw) {
        c.teach();
        c.leave();
        return;
    }
    const uint64_t stay = l2_policy(1), go = l2_policy(2);
    const int nv = c.nv, per = p.per, nch = (nv + per - 1) / per;
    const bool twice = p.dz != nullptr;
    int ask_row = 0, ask_ch = 0, ask_pass = 0, s_ask = 0, s_use = 0, ahead = 0;
    uint32_t parity = 0;
    auto ask = [&]() {
        while (ahead < p.ns - 1 && nv > 0 && ask_row < c.n_rows) {
            c.request(ask_row, s_ask, ask_ch * per, min(per, nv - ask_ch * per), ask_pass || !twice ? go : stay);
            s_ask = s_ask + 1 == p.ns ? 0 : s_ask + 1;
            ahead++;
            if (++ask_ch == nch) {
                ask_ch = 0;
                if (twice && !ask_pass) ask_pass = 1;
                else {
                    ask_pass = 0;
                    ask_row++;
                }
            }
        }
    };
    auto consumed = [&]() {
        ahead--;
        if (++s_use == p.ns) {
            s_use = 0;
            parity ^= 1u;
        }
    };
    for (int i = 0; i < c.n_rows; i++) {
        Run r;
        for (int ch = 0; ch < nch; ch++) {
            ask();
            c.arrived(s_use, parity);
            c.mend(i, s_use, ch * per, min(per, nv - ch * per));
            run_vectors(r, c.buf + s_use * per, min(per, nv - ch * per), p.k);
            __syncwarp();
            consumed();
        }
        c.publish(i, warp_pair(r.m == -INFINITY ? -INFINITY : -r.b, r.s));
        ask();
        const float2 pr = c.collect(i);
        const int eb = c.open_entries(i);
        if (twice) {
            const Entries ent = c.entries(eb);
            const bool alive = *c.live(eb) != 0;
            const float cs = __fdiv_rn(p.c, pr.y);
            for (int ch = 0; ch < nch; ch++) {
                ask();
                c.arrived(s_use, parity);
                c.mend(i, s_use, ch * per, min(per, nv - ch * per));
                const int n = min(per, nv - ch * per), first = c.first_class(i) + ch * per * 8;
                const uint4 *v = c.buf + s_use * per;
                uint16_t *dst = c.out(i) + ch * per * 8;
                if (alive && !c.dead) {
                    grad_vectors<SHIFT>(v, n, dst, first, p.C, p.same, p.k, pr, cs);
                    keep_targets((const uint16_t *)v, first, n * 8, ent, c.warp);
                    __syncwarp();              // orders the warp's stores: the targets' come after those around them
                    patch_targets(dst, first, n * 8, ent, c.warp, p.k, pr, cs, p.c);
                }
                __syncwarp();
                consumed();
            }
            if (!alive && !c.dead) c.send_zeros(i);
        }
        c.close_entries(eb, pr);
    }
    c.leave();
}

// Short rows: a warp for each, which also prepares the teacher's entries; nothing is exchanged and the warps of an SM hide each
// other's waits (4096 x 1000 with 8 entries takes 24 us by the kernel above, whose rows pass through four warps of a CTA one
// after the other).  MEAN: the grid is one cluster, which also takes the mean of the losses.
constexpr int kRowWarps = 8;
constexpr int kRowMaxK = 256;         // entries: what shared memory holds for kRowWarps rows
constexpr int kMeanRows = 64;         // rows of a call that one cluster works on, a row a warp (200 rows: 16 us, with two launches 13)
struct RowLayout {
    uint32_t ent, table, total;       // of a warp: the row | entries | hash table
    int slots;
};
__host__ __device__ inline RowLayout row_layout(int cv, int K)
{
    RowLayout l;
    l.ent = (uint32_t)cv * 16u;
    l.slots = 32;
    while (l.slots < 2 * K) l.slots *= 2;
    l.table = l.ent + ((uint32_t)K * kEntryWords + kMaxWarps + 1u) * 4u;
    l.total = (l.table + 4u * (uint32_t)l.slots + 15u) & ~15u;
    return l;
}
template <int R, bool SHIFT, bool MEAN>
__global__ void __launch_bounds__(kRowWarps * 32, R <= 4 ? 3 : 2) k_distill_rows(const DistillArgs p, float *loss)
{
    pdl_trigger();
    pdl_wait();
    extern __shared__ __align__(128) uint8_t smem[];
    const RowLayout L = row_layout(p.cv, p.K);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *mine = smem + (size_t)warp * L.total;
    uint4 *v = (uint4 *)mine;
    float *at = (float *)(mine + L.ent);
    const Entries ent = {(int32_t *)at, at + p.K, at + 2 * p.K, at + 3 * p.K, (int32_t *)(at + 4 * p.K), (int32_t *)(at + 5 * p.K)};
    for (int row = (int)blockIdx.x * kRowWarps + warp; row < p.B; row += (int)gridDim.x * kRowWarps) {
        const int sh = shift_of<SHIFT>(p, row);
        const uint16_t *zr = p.z + (size_t)row * p.ldz;
        ListAhead ahead;
        ahead.ask(p, row);
        uint4 x[R];
#pragma unroll
        for (int u = 0; u < R; u++) {
            const int first = (lane + 32 * u) * 8 - sh;
            if ((!SHIFT || first >= 0) && first + 8 <= p.C) x[u] = __ldcs((const uint4 *)(zr + first));
            else {
                uint32_t w[4] = {0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u};
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if ((unsigned)(first + e) < (unsigned)p.C)
                        w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xFFFFu) | ((uint32_t)zr[first + e] << 16) : (w[e >> 1] & 0xFFFF0000u) | zr[first + e];
                x[u] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        const bool live = prepare_entries(p, row, 0, sh, ahead, ent, (int *)(mine + L.table), L.slots);
        __half2 mx = __half2half2(__ushort_as_half((unsigned short)kNegInf16));
#pragma unroll
        for (int u = 0; u < R; u++) {
            if (lane + 32 * u < p.cv) v[lane + 32 * u] = x[u];
            mx = __hmax2(mx, max8(x[u]));
        }
        const float m = fmaxf(__low2float(mx), __high2float(mx));           // NaN is dropped here and comes back in the sum
        const float b = m == -INFINITY ? 0.0f : -__fmul_rn(m, p.k);
        float a[4] = {0.0f, 0.0f, 0.0f, 0.0f}, e[R][8];
#pragma unroll
        for (int u = 0; u < R; u++) {
            const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const float2 f = __half22float2(*(const __half2 *)&w[q]);
                e[u][2 * q] = ex2_approx(fmaf(f.x, p.k, b));
                e[u][2 * q + 1] = ex2_approx(fmaf(f.y, p.k, b));
                a[q] += e[u][2 * q] + e[u][2 * q + 1];
            }
        }
        const float2 pr = warp_pair(m == -INFINITY ? -INFINITY : -b, (a[0] + a[1]) + (a[2] + a[3]));
        __syncwarp();
        keep_targets((const uint16_t *)v, -sh, p.cv * 8, ent, 0);
        __syncwarp();
        if (p.dz) {
            uint16_t *out = p.dz + (size_t)row * p.lddz;
            const float cs = __fdiv_rn(p.c, pr.y);
            // this lane's exponentials are relative to 2^-b: a lane of nothing but -inf has zeros (or NaN)
            const float k = m == -INFINITY ? cs * 0.0f : cs * ex2_approx(-b - pr.x);
#pragma unroll
            for (int u = 0; u < R; u++)
                if (lane + 32 * u < p.cv)
                    v[lane + 32 * u] = live ? make_uint4(pack_f16x2(e[u][0] * k, e[u][1] * k), pack_f16x2(e[u][2] * k, e[u][3] * k),
                                                         pack_f16x2(e[u][4] * k, e[u][5] * k), pack_f16x2(e[u][6] * k, e[u][7] * k))
                                            : make_uint4(0u, 0u, 0u, 0u);
            __syncwarp();
            if (live) patch_targets((uint16_t *)v, -sh, p.cv * 8, ent, 0, p.k, pr, cs, p.c);
            __syncwarp();
#pragma unroll
            for (int u = 0; u < R; u++) {
                const int first = (lane + 32 * u) * 8 - sh;
                if (lane + 32 * u < p.cv) store8<SHIFT>(out + first, v[lane + 32 * u], first, p.C, p.same);
            }
        }
        write_loss(p, row, ent, live, pr);
        __syncwarp();                               // the entries are the next row's now
    }
    if (MEAN) {
        __shared__ double red[kRowWarps * 32];
        cluster_sync_all();                         // every row's loss is there
        if (blockIdx.x == 0) mean_of_rows(p.row_loss, p.B, loss, red);
    }
}

constexpr uint32_t kSmemLimit = 220u * 1024u;

template <int R, bool SHIFT, bool MEAN>
cudaError_t run_rows(const DistillArgs &p, float *loss, cudaStream_t st)
{
    static bool configured[kMaxDevices] = {};
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    auto kern = k_distill_rows<R, SHIFT, MEAN>;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const long need = ((long)p.B + kRowWarps - 1) / kRowWarps;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 8;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = MEAN ? 2 : 1;
    cfg.gridDim = dim3(MEAN ? 8u : (unsigned)(need < 148 * 8 ? need : 148 * 8));
    cfg.blockDim = dim3(kRowWarps * 32);
    cfg.dynamicSmemBytes = (size_t)kRowWarps * row_layout(p.cv, p.K).total;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kern, p, loss);
}
template <int R, bool SHIFT>
cudaError_t run_rows_mean(const DistillArgs &p, float *loss, bool mean, cudaStream_t st)
{
    return mean ? run_rows<R, SHIFT, true>(p, loss, st) : run_rows<R, SHIFT, false>(p, loss, st);
}
template <bool SHIFT>
cudaError_t launch_rows(const DistillArgs &p, float *loss, bool mean, cudaStream_t st)
{
    const int R = (p.cv + 31) / 32;
    if (R <= 1) return run_rows_mean<1, SHIFT>(p, loss, mean, st);
    if (R <= 2) return run_rows_mean<2, SHIFT>(p, loss, mean, st);
    if (R <= 4) return run_rows_mean<4, SHIFT>(p, loss, mean, st);
    return run_rows_mean<8, SHIFT>(p, loss, mean, st);
}

typedef void (*DistillKernel)(const DistillArgs);

// id: a number of its own for each kernel (what is known about it is kept per device).
cudaError_t configure(DistillKernel kern, int id)
{
    static bool configured[kMaxDevices][16] = {};
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    if (configured[dev][id]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit);
    configured[dev][id] = e == cudaSuccess;
    return e;
}
// Clusters of cl CTAs of the streaming kernel that are resident at once, one CTA on an SM; -1: an error.
int resident_clusters(DistillKernel kern, int cl)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)cl;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(148 / cl * cl));
    cfg.blockDim = dim3((kMaxWarps + kTeachers) * 32);
    cfg.dynamicSmemBytes = kSmemLimit;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return n;
}
// Rows are dealt out statically, so a cluster that had to wait for another to end would double the time: no more clusters
// than are resident at once.  extra: warps besides those that hold logits and the teacher's; most: warps that an SM's registers
// hold.
cudaError_t run(DistillKernel kern, int resident, int extra, int most, const DistillArgs &p, uint32_t smem, cudaStream_t st)
{
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
    const int threads = (p.nw + kTeachers + extra) * 32;
    int per_sm = most * 32 / threads;
    const int by_smem = (int)((227u * 1024u) / (smem + 1024u));
    if (by_smem < per_sm) per_sm = by_smem;
    if (per_sm < 1) per_sm = 1;
    int clusters = resident * per_sm;
    if (clusters > p.B) clusters = p.B;
    cfg.gridDim = dim3((unsigned)(clusters * p.cl));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

template <bool SHIFT>
cudaError_t launch_rounds(int rounds, const DistillArgs &p, uint32_t smem, cudaStream_t st)
{
    static const DistillKernel kern[] = {k_distill<4, SHIFT, false>, k_distill<5, SHIFT, false>, k_distill<6, SHIFT, false>,
                                         k_distill<7, SHIFT, false>, k_distill<8, SHIFT, false>};
    const bool half = rounds == kMinRounds && p.nw <= kHalfWarps;
    const DistillKernel k = half ? k_distill<kMinRounds, SHIFT, true> : kern[rounds - kMinRounds];
    const cudaError_t e = configure(k, (SHIFT ? 8 : 0) + (half ? kMaxRounds - kMinRounds + 1 : rounds - kMinRounds));
    return e != cudaSuccess ? e : run(k, 148, 1, half ? 2 * (kHalfWarps + kTeachers + 1) : kMaxWarps + kTeachers + 1, p, smem, st);
}
// Rows that are read twice: CTAs of a cluster share one (distill_cluster_log2).
template <bool SHIFT>
cudaError_t launch_stream(DistillArgs p, cudaStream_t st)
{
    const DistillKernel kern = k_distill_stream<SHIFT>;
    static int known[kMaxDevices][kDistillClusters] = {};      // of this kernel
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    const cudaError_t e = configure(kern, SHIFT ? 15 : 7);
    if (e != cudaSuccess) return e;
    const int size = distill_cluster_log2(known[dev], p.B, p.C, [&](int cl) { return resident_clusters(kern, cl); });
    if (size < 0) return cudaErrorLaunchOutOfResources;
    p.cl = 1 << size;
    p.kept = p.cl == 1 && p.dz;
    p.vp = (p.cv + p.cl - 1) / p.cl;
    p.wv = (p.vp + kMaxWarps - 1) / kMaxWarps;
    p.nw = (p.vp + p.wv - 1) / p.wv;
    p.ns = 3;
    for (p.per = kChunk; p.per >= 64; p.per -= 64) {      // long teacher lists leave less room
        const uint32_t smem = layout_of(p.nw, p.ns, p.per, p.cl, p.K, 1 << p.nb_log2).total;
        if (smem <= kSmemLimit) return run(kern, known[dev][size], 0, kMaxWarps + kTeachers, p, smem, st);
    }
    return cudaErrorInvalidConfiguration;
}

// `loss` receives the mean, too, if the kernel that suits the call takes it (*mean_done).
cudaError_t launch_distill(DistillArgs p, float *loss, bool *mean_done, cudaStream_t st)
{
    const bool bulk = (((uintptr_t)p.z | (uintptr_t)p.dz) & 15) == 0 && (p.ldz & 7) == 0 && (!p.dz || (p.lddz & 7) == 0);
    // another pitch or base: the vectors' borders lie elsewhere in every row (all C may be touched by one vector more), and where
    // they lie elsewhere in dz, too, the gradient leaves by elements
    p.same = !p.dz || ((((uintptr_t)p.z ^ (uintptr_t)p.dz) & 15) == 0 && ((p.ldz ^ p.lddz) & 7) == 0);
    const int cv = p.cv = bulk ? (p.C + 7) / 8 : (p.C + 14) / 8;
    p.cl = p.kept = 1;
    if (cv <= 256 && p.K <= kRowMaxK) {
        p.nw = 1;
        p.vp = p.wv = cv;
        *mean_done = p.B <= kMeanRows;
        return bulk ? launch_rows<false>(p, loss, *mean_done, st) : launch_rows<true>(p, loss, *mean_done, st);
    }
    p.nb_log2 = p.K <= 256 ? 2 : 1;
    // four vectors a lane, more only where kMaxWarps warps need it
    int rounds = (cv + 32 * kMaxWarps - 1) / (32 * kMaxWarps);
    if (rounds > kMaxRounds) return bulk ? launch_stream<false>(p, st) : launch_stream<true>(p, st);
    if (rounds < kMinRounds) rounds = kMinRounds;
    p.vp = cv;
    p.wv = p.per = rounds * 32;
    p.nw = (cv + p.wv - 1) / p.wv;
    for (p.ns = 3; p.ns >= 2; p.ns--) {
        const uint32_t smem = layout_of(p.nw, p.ns, p.per, 1, p.K, 1 << p.nb_log2).total;
        if (smem <= kSmemLimit) return bulk ? launch_rounds<false>(rounds, p, smem, st) : launch_rounds<true>(rounds, p, smem, st);
    }
    return cudaErrorInvalidConfiguration;
}

}  // namespace
}  // namespace mpt

using namespace mpt;

extern "C" int mpt_distill_topk(const uint16_t *z_dev, int ldz, int B, int C, const uint16_t *t16_dev, const int32_t *idx_dev,
                                int ldt, int K, float tau, float S, uint16_t *dz_dev, int lddz, float *row_loss_dev,
                                float *loss_dev, uint32_t *status_dev, void *cuda_stream)
{
    // an empty batch has no addresses: what holds rows may be null then
    if (!loss_dev || (B != 0 && (!z_dev || !t16_dev || !idx_dev || !row_loss_dev || z_dev == dz_dev))) return MPT_ERR_INVALID_ARG;
    // 65504 log2(e) / tau stays below 2^31, where rounding an exponent's reference is off by 64: sums relative to it cannot
    // overflow
    if (!(tau >= 0x1p-14f && tau <= 0x1p14f) || !isfinite(S)) return MPT_ERR_INVALID_ARG;
    if (B < 0 || B > kMaxBatch || C < 1 || C > MPT_DISTILL_MAX_C || K < 1 || K > MPT_DISTILL_MAX_K) return MPT_ERR_SHAPE;
    if (ldz < C || (dz_dev && lddz < C) || ldt < K) return MPT_ERR_SHAPE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    bool mean_done = false;
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
        e = launch_distill(p, loss_dev, &mean_done, st);
    }
    if (e == cudaSuccess && !mean_done) e = launch_loss_mean(row_loss_dev, B, loss_dev, st);
    return e == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}
