// Group normalisation of a channels-last tensor x [Nb, P, C] with an activation and dropout in the same pass, and its gradients.
//
//   forward    m_g, v_g over P positions and the cg channels of group g;  xh = (x - m) / sqrt(v + eps);  z = xh w + b;
//              y = dropout(act(z))
//   backward   dz = dropout(dy) act'(z);  db_c = sum dz;  dw_c = sum dz xh;  dn = dz w;
//              dx = rstd (dn - mean_g(dn) - xh mean_g(dn xh))
//
// Everything is bound by memory: x (and dy) in, y (dx) out.  A workgroup takes a slab of whole groups of one image, at least
// 128 bytes of every position, so that lines are read whole.  Where a slab of the whole map fits the registers of one
// workgroup ("whole"), it is read once: mean, then the sum of squared distances from that mean, then the result, all from
// registers.  A larger map is cut into chunks of positions: the chunks' statistics come first, each chunk's own mean and squared
// distances from it, joined by the formula for two sets' (no difference of large sums anywhere), and a second launch reads
// x again, from the last-level cache where the tensor fits it.
// Statistics and sums are fp32; the order of every sum is fixed by the shape, so results repeat bit for bit.
#include "around_device.hpp"

namespace hlq {

// How a call is laid out.  A row of `lanes` lanes covers a slab of lanes * ve channels of one position; `rows` rows to a workgroup.
struct GroupNormPlan {
    int ve, lanes, threads, rows, slabs, chunks, nv;
    int64_t chunk_px;
    bool whole;
};

namespace {

constexpr int kMaxSlab = 2048;       // channels of a slab: its sums fill 64 KB of LDS
constexpr int kSlabBytes = 128;      // of a position, at least

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

// widest vector that channels allow, and the smallest slab of whole groups and whole vectors
bool slab_unit(int C, int cg, int *ve, int *unit)
{
    for (int v : {8, 2, 1}) {
        if (C % v) continue;
        const int64_t u = static_cast<int64_t>(cg) / gcd(cg, v) * v;
        if (u <= kMaxSlab && u / v <= 1024) {
            *ve = v, *unit = static_cast<int>(u);
            return true;
        }
    }
    return false;
}

GroupNormPlan plan_for(int64_t Nb, int64_t P, int C, int cg, bool is_f32, bool backward)
{
    GroupNormPlan p{};
    int unit = 0;
    slab_unit(C, cg, &p.ve, &unit);
    const int want = kSlabBytes / (is_f32 ? 4 : 2);
    int slab = (want + unit - 1) / unit * unit;
    if (slab > C) slab = C;          // a multiple of the unit, too
    p.lanes = slab / p.ve;
    p.slabs = (C + slab - 1) / slab;
    // elements a thread holds: forward x; backward x and dz in fp32
    const int few = 16, many = backward ? 32 : 64;
    static const int threads[3] = {256, 512, 1024};
    for (int pass = 0; pass < 2 && !p.whole; ++pass) {
        const int nv = (pass ? many : few) / p.ve;
        for (int t : threads) {
            if (t < p.lanes) continue;
            if (static_cast<int64_t>(t / p.lanes) * nv >= P) {
                p.whole = true, p.threads = t, p.rows = t / p.lanes, p.nv = nv, p.chunks = 1, p.chunk_px = P;
                break;
            }
        }
    }
    if (p.whole) return p;
    // chunks: enough workgroups to fill the chip, at most 256 a slab (every workgroup of the second launch folds them)
    p.threads = p.lanes > 256 ? 1024 : 256;
    p.rows = p.threads / p.lanes;
    const int64_t pairs = Nb > 0 ? Nb * p.slabs : 1;
    int64_t chunks = (2048 + pairs - 1) / pairs;
    const int64_t most = (P + 4 * p.rows - 1) / (4 * p.rows);
    if (chunks > most) chunks = most;
    if (chunks > 256) chunks = 256;
    if (chunks < 1) chunks = 1;
    p.chunk_px = (P + chunks - 1) / chunks;
    p.chunk_px = (p.chunk_px + p.rows - 1) / p.rows * p.rows;
    p.chunks = static_cast<int>((P + p.chunk_px - 1) / p.chunk_px);
    return p;
}

}  // namespace

// ---- where a thread stands --------------------------------------------------------------------
struct Spot {
    int lane, row, rows, ncol, c0, c, ng;      // ncol: channels of a slab; c: first channel of the thread; ng: groups of the slab
    int64_t img;
    int slab, chunk;
    bool on;
};
__device__ __forceinline__ Spot spot_of(const GroupNormArgs &a, const GroupNormPlan &p, int ve, int block)
{
    Spot s;
    s.row = static_cast<int>(threadIdx.x) / p.lanes;
    s.lane = static_cast<int>(threadIdx.x) - s.row * p.lanes;
    s.rows = p.rows;
    s.ncol = p.lanes * ve;
    const int pair = block / p.chunks;
    s.chunk = block - pair * p.chunks;
    s.img = pair / p.slabs;
    s.slab = pair - static_cast<int>(s.img) * p.slabs;
    s.c0 = s.slab * s.ncol;
    s.c = s.c0 + s.lane * ve;
    const int nch = a.C - s.c0 < s.ncol ? a.C - s.c0 : s.ncol;
    s.ng = nch / a.cg;
    s.on = s.row < p.rows && s.c < a.C;
    return s;
}

// LDS: red[rows][ncol] | part[segs][ncol] (its first row is chan where there is one segment only) | chan[ncol] | grp[ncol]
struct Sums {
    float *red, *part, *chan, *grp;
    int segs;
};
__device__ __forceinline__ Sums sums_of(float *lds, const Spot &s, int ve)
{
    Sums m;
    const int T = static_cast<int>(blockDim.x);
    m.segs = T / s.ncol > 1 ? T / s.ncol : 1;
    m.red = lds;
    m.part = lds + s.rows * s.ncol;
    m.chan = m.segs > 1 ? m.part + m.segs * s.ncol : m.part;
    m.grp = m.chan + s.ncol;
    return m;
}
static size_t sums_lds_bytes(const GroupNormPlan &p)
{
    const int ncol = p.lanes * p.ve, segs = p.threads / ncol > 1 ? p.threads / ncol : 1;
    return sizeof(float) * (static_cast<size_t>(p.rows) * ncol + static_cast<size_t>(segs > 1 ? segs : 0) * ncol + 2 * static_cast<size_t>(ncol));
}

// chan[col] = sum over the workgroup's rows of every thread's v (zeros from threads that are not on)
template <int VE>
__device__ __forceinline__ void column_sums(const float *v, const Spot &s, const Sums &m)
{
    const int T = static_cast<int>(blockDim.x), tid = static_cast<int>(threadIdx.x);
    if (s.row < s.rows) {
#pragma unroll
        for (int e = 0; e < VE; ++e) m.red[s.row * s.ncol + s.lane * VE + e] = s.on ? v[e] : 0.0f;
    }
    __syncthreads();
    if (m.segs > 1) {
        const int seg = tid / s.ncol, col = tid - seg * s.ncol;
        if (seg < m.segs) {
            float t = 0.0f;
            for (int r = seg; r < s.rows; r += m.segs) t += m.red[r * s.ncol + col];
            m.part[seg * s.ncol + col] = t;
        }
        __syncthreads();
        if (tid < s.ncol) {
            float t = 0.0f;
            for (int k = 0; k < m.segs; ++k) t += m.part[k * s.ncol + tid];
            m.chan[tid] = t;
        }
    } else {
        for (int col = tid; col < s.ncol; col += T) {
            float t = 0.0f;
            for (int r = 0; r < s.rows; ++r) t += m.red[r * s.ncol + col];
            m.chan[col] = t;
        }
    }
    __syncthreads();
}

// f(g, sum over the channels of group g of chan[col] weight(col)) for every group of the slab, by one thread each
template <typename Weight, typename F>
__device__ __forceinline__ void group_sums(const Spot &s, const float *chan, int cg, Weight weight, F f)
{
    const int tid = static_cast<int>(threadIdx.x), T = static_cast<int>(blockDim.x);
    if (cg <= 64) {
        for (int g = tid; g < s.ng; g += T) {
            float t = 0.0f;
            for (int k = 0; k < cg; ++k) t += chan[g * cg + k] * weight(g * cg + k);
            f(g, t);
        }
    } else {
        for (int g = tid >> 6; g < s.ng; g += T >> 6) {          // a wavefront to a group
            float t = 0.0f;
            for (int k = tid & 63; k < cg; k += 64) t += chan[g * cg + k] * weight(g * cg + k);
            t = lanes_sum<64>(t);
            if ((tid & 63) == 0) f(g, t);
        }
    }
}

// v[e] = table[group of the thread's channel e]
template <int VE>
__device__ __forceinline__ void of_groups(const float *table, int local_c, int cg, float *v)
{
    int g = local_c / cg, rem = local_c - g * cg;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        v[e] = table[g];
        if (++rem == cg) rem = 0, ++g;
    }
}

template <int VE>
__device__ __forceinline__ void load_params(const void *p, bool f32, int c, float otherwise, float *v)
{
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = p ? load_param(p, f32, c + e) : otherwise;
}

// ---- forward ----------------------------------------------------------------------------------

// WHOLE: the slab's map is one tile of rows * NV positions, normalised from registers.  Else: the statistics of a chunk, tile by
// tile, for the second launch: {mean, sum of squared distances} to part[img][chunk][group].
template <typename T, int VE, int NV, bool WHOLE>
__global__ __launch_bounds__(1024) void k_gn_tile(GroupNormArgs a, GroupNormPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    const Spot s = spot_of(a, p, VE, blockIdx.x);
    const Sums m = sums_of(lds, s, VE);
    const int64_t p0 = static_cast<int64_t>(s.chunk) * p.chunk_px;
    const int64_t p1 = WHOLE ? a.P : (p0 + p.chunk_px < a.P ? p0 + p.chunk_px : a.P);
    const T *x = static_cast<const T *>(a.x) + s.img * a.P * a.C + s.c;
    const int64_t step = static_cast<int64_t>(s.rows) * a.C;
    float run_n = 0.0f, run_mean = 0.0f, run_m2 = 0.0f;         // of group threadIdx.x, over the chunk's tiles so far
    for (int64_t t0 = p0; t0 < p1; t0 += static_cast<int64_t>(s.rows) * NV) {
        Raw<T, VE> raw[NV];
        const T *q = x + (t0 + s.row) * a.C;
        const int64_t left = p1 - t0 - s.row;                   // positions from the thread's first to the end, in steps of rows
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            raw[j].zero();
            if (s.on && static_cast<int64_t>(j) * s.rows < left) raw[j].load(q + j * step);
        }
        const float n = static_cast<float>((p1 - t0 < static_cast<int64_t>(s.rows) * NV ? p1 - t0 : static_cast<int64_t>(s.rows) * NV)) *
                        static_cast<float>(a.cg);
        float v[VE], u[VE], mean[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            raw[j].widen(u);
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] += u[e];
        }
        column_sums<VE>(v, s, m);
        group_sums(s, m.chan, a.cg, [](int) { return 1.0f; }, [&](int g, float t) { m.grp[g] = t / n; });
        __syncthreads();
        if (s.on) of_groups<VE>(m.grp, s.lane * VE, a.cg, mean);
        float tile_mean = 0.0f;
        if (!WHOLE && static_cast<int>(threadIdx.x) < s.ng) tile_mean = m.grp[threadIdx.x];
        if (WHOLE && a.mean)
            for (int g = threadIdx.x; g < s.ng; g += blockDim.x) a.mean[s.img * a.groups + s.c0 / a.cg + g] = m.grp[g];
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (s.on && static_cast<int64_t>(j) * s.rows < left) {
                raw[j].widen(u);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float d = u[e] - mean[e];
                    v[e] = __builtin_fmaf(d, d, v[e]);
                }
            }
        }
        column_sums<VE>(v, s, m);
        if constexpr (WHOLE) {
            group_sums(s, m.chan, a.cg, [](int) { return 1.0f; }, [&](int g, float t) {
                const float r = 1.0f / sqrtf(t / n + a.eps);
                m.grp[g] = r;
                if (a.rstd) a.rstd[s.img * a.groups + s.c0 / a.cg + g] = r;
            });
            __syncthreads();
            if (!s.on) return;
            float w[VE], b[VE];
            of_groups<VE>(m.grp, s.lane * VE, a.cg, u);
            load_params<VE>(a.w, a.param_f32, s.c, 1.0f, w);
            load_params<VE>(a.b, a.param_f32, s.c, 0.0f, b);
#pragma unroll
            for (int e = 0; e < VE; ++e) w[e] *= u[e];
            const int64_t at = (s.img * a.P + s.row) * a.C + s.c;
            T *y = static_cast<T *>(a.y) + at;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (static_cast<int64_t>(j) * s.rows < left) {
                    raw[j].widen(u);
#pragma unroll
                    for (int e = 0; e < VE; ++e) u[e] = __builtin_fmaf(u[e] - mean[e], w[e], b[e]);
                    act_values<EXACT, VE>(u, a.act);
                    if (a.drop.below) drop_values<VE>(u, at + j * step, a.drop);
                    Raw<T, VE>::store(y + j * step, u);
                }
            }
        } else {
            group_sums(s, m.chan, a.cg, [](int) { return 1.0f; }, [&](int g, float t) { m.grp[g] = t; });
            __syncthreads();
            if (static_cast<int>(threadIdx.x) < s.ng) {
                const float both = run_n + n, delta = tile_mean - run_mean, share = n / both;
                run_mean += delta * share;
                run_m2 += m.grp[threadIdx.x] + delta * delta * run_n * share;
                run_n = both;
            }
        }
    }
    if (!WHOLE && static_cast<int>(threadIdx.x) < s.ng)
        static_cast<float2 *>(a.ws)[(s.img * p.chunks + s.chunk) * a.groups + s.c0 / a.cg + threadIdx.x] = make_float2(run_mean, run_m2);
}

// Second launch of a map in chunks: the chunks' statistics joined, then the chunk normalised.
template <typename T, int VE, int U>
__global__ __launch_bounds__(1024) void k_gn_apply(GroupNormArgs a, GroupNormPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    const Spot s = spot_of(a, p, VE, blockIdx.x);
    const int tid = static_cast<int>(threadIdx.x), T_ = static_cast<int>(blockDim.x);
    // three floats a thread: count, mean, squared distances of the chunks seg, seg + segs, ... of group g
    float *ln = lds, *lm = lds + T_, *lq = lds + 2 * T_, *gm = lds + 3 * T_, *gr = gm + s.ncol;
    const int segs = T_ / s.ng;
    const int g = tid % s.ng, seg = tid / s.ng;
    const float2 *part = static_cast<const float2 *>(a.ws) + s.img * p.chunks * a.groups + s.c0 / a.cg;
    float n = 0.0f, mean = 0.0f, m2 = 0.0f;
    if (seg < segs) {
        for (int k = seg; k < p.chunks; k += segs) {
            const float2 v = part[static_cast<int64_t>(k) * a.groups + g];
            const int64_t px = k + 1 < p.chunks ? p.chunk_px : a.P - static_cast<int64_t>(k) * p.chunk_px;
            const float nk = static_cast<float>(px) * static_cast<float>(a.cg), both = n + nk, delta = v.x - mean, share = nk / both;
            mean += delta * share;
            m2 += v.y + delta * delta * n * share;
            n = both;
        }
    }
    ln[tid] = n, lm[tid] = mean, lq[tid] = m2;
    __syncthreads();
    if (tid < s.ng) {
        for (int k = 1; k < segs && k < p.chunks; ++k) {
            const int o = k * s.ng + tid;
            const float nk = ln[o], both = n + nk, delta = lm[o] - mean, share = nk / both;
            mean += delta * share;
            m2 += lq[o] + delta * delta * n * share;
            n = both;
        }
        const float r = 1.0f / sqrtf(m2 / n + a.eps);
        gm[tid] = mean, gr[tid] = r;
        if (s.chunk == 0) {
            const int64_t o = s.img * a.groups + s.c0 / a.cg + tid;
            if (a.mean) a.mean[o] = mean;
            if (a.rstd) a.rstd[o] = r;
        }
    }
    __syncthreads();
    if (!s.on) return;
    float mu[VE], w[VE], b[VE], u[VE];
    of_groups<VE>(gm, s.lane * VE, a.cg, mu);
    of_groups<VE>(gr, s.lane * VE, a.cg, u);
    load_params<VE>(a.w, a.param_f32, s.c, 1.0f, w);
    load_params<VE>(a.b, a.param_f32, s.c, 0.0f, b);
#pragma unroll
    for (int e = 0; e < VE; ++e) w[e] *= u[e];
    const int64_t p0 = static_cast<int64_t>(s.chunk) * p.chunk_px, p1 = p0 + p.chunk_px < a.P ? p0 + p.chunk_px : a.P;
    const int64_t step = static_cast<int64_t>(s.rows) * a.C;
    int64_t at = (s.img * a.P + p0 + s.row) * a.C + s.c;
    for (int64_t q = p0 + s.row; q < p1; q += static_cast<int64_t>(U) * s.rows, at += U * step) {
        Raw<T, VE> raw[U];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (q + static_cast<int64_t>(j) * s.rows < p1) raw[j].load(static_cast<const T *>(a.x) + at + j * step);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (q + static_cast<int64_t>(j) * s.rows < p1) {
                raw[j].widen(u);
#pragma unroll
                for (int e = 0; e < VE; ++e) u[e] = __builtin_fmaf(u[e] - mu[e], w[e], b[e]);
                act_values<EXACT, VE>(u, a.act);
                if (a.drop.below) drop_values<VE>(u, at + j * step, a.drop);
                Raw<T, VE>::store(static_cast<T *>(a.y) + at + j * step, u);
            }
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------

// what a thread needs of its channels
template <int VE> struct Channels {
    float mean[VE], rstd[VE], w[VE], b[VE];
    __device__ __forceinline__ void load(const GroupNormArgs &a, const Spot &s)
    {
        int g = s.c / a.cg, rem = s.c - g * a.cg;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            mean[e] = a.mean[s.img * a.groups + g];
            rstd[e] = a.rstd[s.img * a.groups + g];
            if (++rem == a.cg) rem = 0, ++g;
        }
        load_params<VE>(a.w, a.param_f32, s.c, 1.0f, w);
        load_params<VE>(a.b, a.param_f32, s.c, 0.0f, b);
    }
    // xh and dz of elements `at` .. of x and dy
    template <bool EXACT, typename R>
    __device__ __forceinline__ void slope(const GroupNormArgs &a, const R &x, const R &dy, int64_t at, float *xh, float *dz) const
    {
        float z[VE];
        x.widen(xh);
        dy.widen(dz);
        if (a.drop.below) drop_values<VE>(dz, at, a.drop);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            xh[e] = (xh[e] - mean[e]) * rstd[e];
            z[e] = __builtin_fmaf(xh[e], w[e], b[e]);
        }
        act_slopes<EXACT, VE>(z, a.act, dz);
    }
};

// group means of dn and dn xh from the channels' sums: {sum dz, sum dz xh} in chA, chB
template <int VE>
__device__ __forceinline__ void group_means(const GroupNormArgs &a, const Spot &s, const float *chA, const float *chB, float *gA, float *gB,
                                            float *mA, float *mB)
{
    const float inv = 1.0f / (static_cast<float>(a.P) * static_cast<float>(a.cg));
    auto weight = [&](int col) { return a.w ? load_param(a.w, a.param_f32, s.c0 + col) : 1.0f; };
    group_sums(s, chA, a.cg, weight, [&](int g, float t) { gA[g] = t * inv; });
    group_sums(s, chB, a.cg, weight, [&](int g, float t) { gB[g] = t * inv; });
    __syncthreads();
    if (s.on) {
        of_groups<VE>(gA, s.lane * VE, a.cg, mA);
        of_groups<VE>(gB, s.lane * VE, a.cg, mB);
    }
}

// A slab's map in one tile: x stays in registers as it is, dz in fp32.  Channels' sums to part[img][channel].
template <typename T, int VE, int NV>
__global__ __launch_bounds__(1024) void k_gn_grad_tile(GroupNormArgs a, GroupNormPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    const Spot s = spot_of(a, p, VE, blockIdx.x);
    const Sums m = sums_of(lds, s, VE);
    float *chB = m.grp + s.ncol, *gB = chB + s.ncol;
    const int64_t step = static_cast<int64_t>(s.rows) * a.C, at = (s.img * a.P + s.row) * a.C + s.c, left = a.P - s.row;
    Raw<T, VE> x[NV], dy[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        x[j].zero();
        dy[j].zero();
        if (s.on && static_cast<int64_t>(j) * s.rows < left) {
            x[j].load(static_cast<const T *>(a.x) + at + j * step);
            dy[j].load(static_cast<const T *>(a.dy) + at + j * step);
        }
    }
    Channels<VE> ch;
    float dz[NV][VE], A[VE], B[VE], xh[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) A[e] = B[e] = 0.0f;
    if (s.on) {
        ch.load(a, s);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (static_cast<int64_t>(j) * s.rows < left) {
                ch.template slope<EXACT>(a, x[j], dy[j], at + j * step, xh, dz[j]);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    A[e] += dz[j][e];
                    B[e] = __builtin_fmaf(dz[j][e], xh[e], B[e]);
                }
            }
        }
    }
    column_sums<VE>(B, s, m);
    for (int col = threadIdx.x; col < s.ncol; col += blockDim.x) chB[col] = m.chan[col];
    __syncthreads();
    column_sums<VE>(A, s, m);
    for (int col = threadIdx.x; col < s.ncol; col += blockDim.x)
        if (s.c0 + col < a.C) static_cast<float2 *>(a.ws)[s.img * a.C + s.c0 + col] = make_float2(m.chan[col], chB[col]);
    if (!a.y) return;
    float mA[VE], mB[VE];
    group_means<VE>(a, s, m.chan, chB, m.grp, gB, mA, mB);
    if (!s.on) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (static_cast<int64_t>(j) * s.rows < left) {
            x[j].widen(xh);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                xh[e] = (xh[e] - ch.mean[e]) * ch.rstd[e];
                xh[e] = ch.rstd[e] * (dz[j][e] * ch.w[e] - mA[e] - xh[e] * mB[e]);
            }
            Raw<T, VE>::store(static_cast<T *>(a.y) + at + j * step, xh);
        }
    }
}

// Channels' sums of a chunk to part[img][chunk][channel].
template <typename T, int VE, int U>
__global__ __launch_bounds__(1024) void k_gn_grad_sums(GroupNormArgs a, GroupNormPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    const Spot s = spot_of(a, p, VE, blockIdx.x);
    const Sums m = sums_of(lds, s, VE);
    float *chB = m.grp + s.ncol;
    const int64_t p0 = static_cast<int64_t>(s.chunk) * p.chunk_px, p1 = p0 + p.chunk_px < a.P ? p0 + p.chunk_px : a.P;
    const int64_t step = static_cast<int64_t>(s.rows) * a.C;
    float A[VE], B[VE], xh[VE], dz[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) A[e] = B[e] = 0.0f;
    if (s.on) {
        Channels<VE> ch;
        ch.load(a, s);
        int64_t at = (s.img * a.P + p0 + s.row) * a.C + s.c;
        for (int64_t q = p0 + s.row; q < p1; q += static_cast<int64_t>(U) * s.rows, at += U * step) {
            Raw<T, VE> x[U], dy[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (q + static_cast<int64_t>(j) * s.rows < p1) {
                    x[j].load(static_cast<const T *>(a.x) + at + j * step);
                    dy[j].load(static_cast<const T *>(a.dy) + at + j * step);
                }
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (q + static_cast<int64_t>(j) * s.rows < p1) {
                    ch.template slope<EXACT>(a, x[j], dy[j], at + j * step, xh, dz);
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        A[e] += dz[e];
                        B[e] = __builtin_fmaf(dz[e], xh[e], B[e]);
                    }
                }
            }
        }
    }
    column_sums<VE>(B, s, m);
    for (int col = threadIdx.x; col < s.ncol; col += blockDim.x) chB[col] = m.chan[col];
    __syncthreads();
    column_sums<VE>(A, s, m);
    for (int col = threadIdx.x; col < s.ncol; col += blockDim.x)
        if (s.c0 + col < a.C)
            static_cast<float2 *>(a.ws)[(s.img * p.chunks + s.chunk) * a.C + s.c0 + col] = make_float2(m.chan[col], chB[col]);
}

// dw[c], db[c]: the sums of `parts` rows of {sum dz, sum dz xh}, 16 channels a workgroup
__device__ __forceinline__ void gn_param_grads(const GroupNormArgs &a, int64_t parts, int block, float *lds)
{
    const int T = static_cast<int>(blockDim.x), col = threadIdx.x & 15, row = threadIdx.x >> 4, rows = T >> 4, c = block * 16 + col;
    const float2 *part = static_cast<const float2 *>(a.ws);
    float A = 0.0f, B = 0.0f;
    if (c < a.C) {
        int64_t k = row;
        for (; k + 7 * rows < parts; k += 8 * rows) {
            float2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = part[(k + static_cast<int64_t>(i) * rows) * a.C + c];
#pragma unroll
            for (int i = 0; i < 8; ++i) A += v[i].x, B += v[i].y;
        }
        for (; k < parts; k += rows) {
            const float2 v = part[k * a.C + c];
            A += v.x, B += v.y;
        }
    }
    lds[threadIdx.x] = A, lds[T + threadIdx.x] = B;
    __syncthreads();
    for (int h = rows >> 1; h > 0; h >>= 1) {
        if (row < h) {
            lds[threadIdx.x] += lds[threadIdx.x + 16 * h];
            lds[T + threadIdx.x] += lds[T + threadIdx.x + 16 * h];
        }
        __syncthreads();
    }
    if (row == 0 && c < a.C) {
        if (a.db) store_param(a.db, a.param_f32, c, lds[col]);
        if (a.dw) store_param(a.dw, a.param_f32, c, lds[T + col]);
    }
}
__global__ __launch_bounds__(1024) void k_gn_param_grads(GroupNormArgs a, int64_t parts)
{
    extern __shared__ float lds[];
    gn_param_grads(a, parts, blockIdx.x, lds);
}

// Second launch of a map in chunks: dx.  The first `side` workgroups sum the parameters' gradients instead.
template <typename T, int VE, int U>
__global__ __launch_bounds__(1024) void k_gn_grad_apply(GroupNormArgs a, GroupNormPlan p, int side)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    if (static_cast<int>(blockIdx.x) < side) {
        gn_param_grads(a, static_cast<int64_t>(a.Nb) * p.chunks, blockIdx.x, lds);
        return;
    }
    const Spot s = spot_of(a, p, VE, blockIdx.x - side);
    const int tid = static_cast<int>(threadIdx.x), T_ = static_cast<int>(blockDim.x);
    // the chunks' sums of the slab's channels
    const int segs = T_ / s.ncol > 1 ? T_ / s.ncol : 1;
    float *pA = lds, *pB = pA + segs * s.ncol, *gA = pB + segs * s.ncol, *gB = gA + s.ncol;
    const float2 *part = static_cast<const float2 *>(a.ws) + s.img * p.chunks * a.C + s.c0;
    for (int i = tid; i < segs * s.ncol; i += T_) {
        const int seg = i / s.ncol, col = i - seg * s.ncol;
        float A = 0.0f, B = 0.0f;
        if (s.c0 + col < a.C) {
            for (int k = seg; k < p.chunks; k += segs) {
                const float2 v = part[static_cast<int64_t>(k) * a.C + col];
                A += v.x, B += v.y;
            }
        }
        pA[i] = A, pB[i] = B;
    }
    __syncthreads();
    for (int col = tid; col < s.ncol; col += T_) {
        float A = pA[col], B = pB[col];
        for (int k = 1; k < segs; ++k) A += pA[k * s.ncol + col], B += pB[k * s.ncol + col];
        pA[col] = A, pB[col] = B;
    }
    __syncthreads();
    float mA[VE], mB[VE];
    group_means<VE>(a, s, pA, pB, gA, gB, mA, mB);
    if (!s.on) return;
    Channels<VE> ch;
    ch.load(a, s);
    const int64_t p0 = static_cast<int64_t>(s.chunk) * p.chunk_px, p1 = p0 + p.chunk_px < a.P ? p0 + p.chunk_px : a.P;
    const int64_t step = static_cast<int64_t>(s.rows) * a.C;
    int64_t at = (s.img * a.P + p0 + s.row) * a.C + s.c;
    for (int64_t q = p0 + s.row; q < p1; q += static_cast<int64_t>(U) * s.rows, at += U * step) {
        Raw<T, VE> x[U], dy[U];
        float xh[VE], dz[VE];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (q + static_cast<int64_t>(j) * s.rows < p1) {
                x[j].load(static_cast<const T *>(a.x) + at + j * step);
                dy[j].load(static_cast<const T *>(a.dy) + at + j * step);
            }
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (q + static_cast<int64_t>(j) * s.rows < p1) {
                ch.template slope<EXACT>(a, x[j], dy[j], at + j * step, xh, dz);
#pragma unroll
                for (int e = 0; e < VE; ++e) xh[e] = ch.rstd[e] * (dz[e] * ch.w[e] - mA[e] - xh[e] * mB[e]);
                Raw<T, VE>::store(static_cast<T *>(a.y) + at + j * step, xh);
            }
        }
    }
}

// ---- launches ---------------------------------------------------------------------------------

bool group_norm_ok(int C, int cg)
{
    int ve, unit;
    return slab_unit(C, cg, &ve, &unit);
}

size_t group_norm_ws_bytes(int64_t Nb, int64_t P, int C, int groups, bool is_f32, bool backward)
{
    const GroupNormPlan p = plan_for(Nb, P, C, C / groups, is_f32, backward);
    if (backward) return static_cast<size_t>(Nb) * p.chunks * C * sizeof(float2);
    return p.whole ? 0 : static_cast<size_t>(Nb) * p.chunks * groups * sizeof(float2);
}

template <typename T, int VE>
static hipError_t forward(const GroupNormArgs &a, const GroupNormPlan &p, hipStream_t st)
{
    const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(a.Nb) * p.slabs * p.chunks);
    const size_t lds = sums_lds_bytes(p);
    if (p.whole) {
        if (p.nv == 16 / VE) k_gn_tile<T, VE, 16 / VE, true><<<blocks, p.threads, lds, st>>>(a, p);
        else k_gn_tile<T, VE, 64 / VE, true><<<blocks, p.threads, lds, st>>>(a, p);
        return hipGetLastError();
    }
    k_gn_tile<T, VE, 64 / VE, false><<<blocks, p.threads, lds, st>>>(a, p);
    if (const hipError_t e = hipGetLastError()) return e;
    k_gn_apply<T, VE, 4><<<blocks, p.threads, sizeof(float) * (3 * p.threads + 2 * p.lanes * VE), st>>>(a, p);
    return hipGetLastError();
}

template <typename T, int VE>
static hipError_t backward(const GroupNormArgs &a, const GroupNormPlan &p, hipStream_t st)
{
    const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(a.Nb) * p.slabs * p.chunks);
    const size_t ncol = static_cast<size_t>(p.lanes) * VE, lds = sums_lds_bytes(p) + 2 * ncol * sizeof(float);
    const bool params = a.dw || a.db;
    const int side = params ? (a.C + 15) / 16 : 0;
    if (p.whole) {
        if (blocks) {
            if (p.nv == 16 / VE) k_gn_grad_tile<T, VE, 16 / VE><<<blocks, p.threads, lds, st>>>(a, p);
            else k_gn_grad_tile<T, VE, 32 / VE><<<blocks, p.threads, lds, st>>>(a, p);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        if (params) k_gn_param_grads<<<side, 1024, 2 * 1024 * sizeof(float), st>>>(a, a.Nb);
        return hipGetLastError();
    }
    if (blocks) k_gn_grad_sums<T, VE, 2><<<blocks, p.threads, lds, st>>>(a, p);
    if (const hipError_t e = hipGetLastError()) return e;
    const unsigned second = side + (a.y ? blocks : 0);
    const size_t segs = p.threads / ncol > 1 ? p.threads / ncol : 1;
    size_t lds2 = sizeof(float) * (2 * segs * ncol + 2 * ncol);
    if (lds2 < 2 * sizeof(float) * p.threads) lds2 = 2 * sizeof(float) * p.threads;
    if (second) k_gn_grad_apply<T, VE, 2><<<second, p.threads, lds2, st>>>(a, p, side);
    return hipGetLastError();
}

template <typename T>
static hipError_t by_vector(const GroupNormArgs &a, bool back, hipStream_t st)
{
    const GroupNormPlan p = plan_for(a.Nb, a.P, a.C, a.cg, a.is_f32, back);
    if (p.ve == 8) return back ? backward<T, 8>(a, p, st) : forward<T, 8>(a, p, st);
    if (p.ve == 2) return back ? backward<T, 2>(a, p, st) : forward<T, 2>(a, p, st);
    return back ? backward<T, 1>(a, p, st) : forward<T, 1>(a, p, st);
}

hipError_t launch_group_norm(const GroupNormArgs &a, hipStream_t st) { return a.is_f32 ? by_vector<float>(a, false, st) : by_vector<bf16_t>(a, false, st); }
hipError_t launch_group_norm_backward(const GroupNormArgs &a, hipStream_t st) { return a.is_f32 ? by_vector<float>(a, true, st) : by_vector<bf16_t>(a, true, st); }

}  // namespace hlq
