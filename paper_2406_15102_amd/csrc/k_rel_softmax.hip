// Attention map with a learned relative position bias: softmax over the keys of scaled scores plus one value per head and
// relative position, masked, with dropout; and its gradients.
//
//   z = scale s[b,h,q,k] + table[of[rel(q,k)], h] for the keys that q sees;   p = exp(z - max z) / sum exp(z - max z);   P = dropout(p)
//   dp = dropout(dP);   dz = p (dp - sum_k p dp);   dS = scale dz;   dtable[c, h] = sum over b, q, k with of[rel(q,k)] = c of dz
//
// rel(q, k) = u(k) - u(q) + const with u(k) = k on a sequence and u(k) = (k / w) (2 w - 1) + k % w on a grid of width w, so for one
// query distinct keys have distinct relative positions, and a head's bias is a vector that slides along the keys.
//
// Bound by memory: the scores (and dP) in, the map (dS) out; the row is in registers between them and p is computed anew in the
// backward pass, so nothing is kept of the forward pass but the scores.  A row lies in 8, 16, 32 or 64 lanes of a wavefront, or in the
// four wavefronts of a workgroup, 8 to 64 keys a lane.  A workgroup stays with one head: it lays the part of the bias vector that
// its queries reach into LDS, takes a query's bias into registers and goes through the batch with it.  The gradient of the bias is
// summed over the batch in registers, then over the workgroup's queries in LDS (one thread owns a relative position, so
// there are no atomics and the order is fixed), and leaves the workgroup once; a second launch sums the workgroups' vectors by bucket.
#include "around_device.hpp"

namespace hlq {

struct RelPlan {
    int lanes, nv;               // lanes of a row, vectors of 8 keys a lane
    int rows_q, rows_b;          // queries and batches that a workgroup's rows are in one step
    int q_block, q_blocks;       // queries of a workgroup
    int b_chunk, b_chunks;       // batches of a workgroup
    int win;                     // relative positions that a workgroup's queries reach, at most
    bool few;                    // at most 64 buckets: a workgroup sums its relative positions by bucket before it writes them
    int stride;                  // floats that a workgroup writes: 64, or `win`
};

namespace {

constexpr int kThreads = 256;
constexpr int kFewBuckets = 64;                                  // a lane of a wavefront to a bucket
constexpr int kMaxKeysSequence = 16384, kMaxKeysGrid = 4096;     // two vectors of them (u stretches a grid's to two each) in LDS

__host__ __device__ __forceinline__ int rel_u(int k, int gw) { return gw ? k / gw * (2 * gw - 1) + k % gw : k; }
// rel(q, k) = u(k) - u(q) + rel_const
__host__ __device__ __forceinline__ int rel_const(int Q, int K, int gw) { return gw ? rel_u(K - 1, gw) : Q - 1; }

// Place of relative position i of a sequence in LDS: one float of padding to eight, so that lanes that read element e of their eight keys,
// 8 floats apart, meet 64 banks instead of 8.
__host__ __device__ __forceinline__ int padded(int i) { return i + (i >> 3); }

RelPlan rel_plan(const RelArgs &a, bool back)
{
    RelPlan p{};
    if (a.K <= 64) p.lanes = 8, p.nv = 1;
    else if (a.K <= 128) p.lanes = 16, p.nv = 1;
    else if (a.K <= 256) p.lanes = 32, p.nv = 1;
    else if (a.K <= 512) p.lanes = 64, p.nv = 1;
    else if (a.K <= 1024) p.lanes = 64, p.nv = 2;
    else if (a.K <= 2048) p.lanes = 64, p.nv = 4;
    else if (a.K <= 4096) p.lanes = 256, p.nv = 2;
    else if (a.K <= 8192) p.lanes = 256, p.nv = 4;
    else p.lanes = 256, p.nv = 8;
    const int rows = kThreads / p.lanes;
    p.rows_q = rows;
    while (p.rows_q > 1 && p.rows_q / 2 >= a.Q) p.rows_q /= 2;
    p.rows_b = rows / p.rows_q;
    const int q_steps = (a.Q + p.rows_q - 1) / p.rows_q, b_steps = (a.B + p.rows_b - 1) / p.rows_b;
    const int64_t items = static_cast<int64_t>(a.H) * q_steps * b_steps, target = back ? 1024 : 2048;
    int64_t per = (items + target - 1) / target;
    if (per < 1) per = 1;
    int b_per = per < b_steps ? static_cast<int>(per) : b_steps;
    int q_per = static_cast<int>(per / b_per);
    if (q_per < 1) q_per = 1;
    if (q_per > q_steps) q_per = q_steps;
    if (q_per * p.rows_q > 512) q_per = 512 / p.rows_q;         // the reach of a workgroup's queries stays in LDS
    p.q_block = q_per * p.rows_q;
    p.q_blocks = (a.Q + p.q_block - 1) / p.q_block;
    p.b_chunk = b_per * p.rows_b;
    p.b_chunks = (a.B + p.b_chunk - 1) / p.b_chunk;
    // reach of q_block consecutive queries
    const int most = a.grid_w ? (p.q_block + a.grid_w - 1) / a.grid_w * (2 * a.grid_w - 1) + a.grid_w : p.q_block;
    const int all = a.grid_w ? 2 * rel_u(a.K - 1, a.grid_w) + 1 : a.Q + a.K - 1;
    p.win = rel_u(a.K - 1, a.grid_w) + most;
    if (p.win > all) p.win = all;
    p.few = a.n_buckets <= kFewBuckets;
    p.stride = p.few ? kFewBuckets : p.win;
    return p;
}

// LDS of a workgroup, in floats: the bias vector, the sums by relative position (one vector a wavefront where a wavefront is a row; for
// shorter rows one, and the rows' sums over the batch), reductions across the wavefronts.
__host__ __device__ __forceinline__ int rel_vector(const RelPlan &p, int gw) { return (p.lanes >= 64 && !gw ? padded(p.win) + 1 : p.win); }
size_t rel_lds_bytes(const RelPlan &p, int gw, bool back)
{
    const size_t v = rel_vector(p, gw);
    const int rows = kThreads / p.lanes;
    size_t n = v + 16;
    if (back) n += p.lanes == 64 ? 4 * v : v + (rows > 1 ? static_cast<size_t>(rows) * p.lanes * p.nv * 8 : 0);
    return sizeof(float) * n;
}

}  // namespace

// 8 elements from place `at` of a tensor of `total`: whole vectors run over a row's end into the next row, but not over the tensor's
template <typename T>
__device__ __forceinline__ void load_inside(Raw<T, 8> &r, const T *base, int64_t at, int64_t total)
{
    if (at + 8 <= total) {
        r.load(base + at);
    } else {
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = at + e < total ? base[at + e] : T{};
        __builtin_memcpy(&r, v, sizeof(v));
    }
}
// bit e: byte e of the eight is not zero
__device__ __forceinline__ uint32_t load_mask(const uint8_t *base, int64_t at, int64_t total)
{
    uint64_t m = 0;
    if (at + 8 <= total) {
        __builtin_memcpy(&m, base + at, 8);
    } else {
        for (int e = 0; e < 8 && at + e < total; ++e) m |= static_cast<uint64_t>(base[at + e]) << (8 * e);
    }
    const uint64_t low = 0x7F7F7F7F7F7F7F7Full;
    const uint64_t top = (((m & low) + low) | m) & ~low;               // bit 7 of every byte that is not zero
    return static_cast<uint32_t>((top >> 7) * 0x0102040810204080ull >> 56);
}
// the first n of 8
template <typename T>
__device__ __forceinline__ void store_first(T *p, const float *v, int n)
{
    if (n >= 8) {
        Raw<T, 8>::store(p, v);
        return;
    }
    if (n & 4) {
        Raw<T, 2>::store(p, v);
        Raw<T, 2>::store(p + 2, v + 2);
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e >= (n & 4) && e < n) store_one(p + e, v[e]);
}

// zeros for the elements whose bit is not set
__device__ __forceinline__ void keep_bits(Raw<bf16_t, 8> &r, uint32_t bits)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - 2 * i)) >> 31), hi = static_cast<uint32_t>(static_cast<int32_t>(bits << (30 - 2 * i)) >> 31);
        r.w[i] &= (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void keep_bits(Raw<float, 8> &r, uint32_t bits)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.a[i] = (bits >> i) & 1 ? r.a[i] : 0.0f;
        r.b[i] = (bits >> (4 + i)) & 1 ? r.b[i] : 0.0f;
    }
}
// zeros for the elements that dropout drops; what is kept is not scaled.  i a multiple of 8
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void drop_raw(Raw<bf16_t, 8> &r, int64_t i, const DropRule &d)
{
    uint32_t w[4];
    rand_words<4>(static_cast<uint32_t>(i >> 1), d.k0, d.k1, w);
    const u16x2 under = {static_cast<uint16_t>(d.below - 1), static_cast<uint16_t>(d.below - 1)}, one = {1, 1}, none = {0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        // halves at or above `below`: their difference from below - 1, cut at 0, is not 0
        const u16x2 over = __builtin_elementwise_min(__builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, w[k]), under), one);
        const u16x2 keep = none - over;
        r.w[k] &= __builtin_bit_cast(uint32_t, keep);
    }
}
__device__ __forceinline__ void drop_raw(Raw<float, 8> &r, int64_t i, const DropRule &d)
{
    uint32_t w[4];
    rand_words<4>(static_cast<uint32_t>(i >> 1), d.k0, d.k1, w);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const bool lo = (w[k] & 0xFFFFu) >= d.below, hi = (w[k] >> 16) >= d.below;
        if (k < 2) {
            r.a[2 * k] = lo ? r.a[2 * k] : 0.0f;
            r.a[2 * k + 1] = hi ? r.a[2 * k + 1] : 0.0f;
        } else {
            r.b[2 * k - 4] = lo ? r.b[2 * k - 4] : 0.0f;
            r.b[2 * k - 3] = hi ? r.b[2 * k - 3] : 0.0f;
        }
    }
}

// What a workgroup works on, the same for all its threads.
struct RelJob {
    int h, q0, q1, b0, b1, part, rc, rlo, win;
};
__device__ __forceinline__ RelJob rel_job(const RelArgs &a, const RelPlan &p)
{
    RelJob j;
    const int qb = blockIdx.x % p.q_blocks, rest = blockIdx.x / p.q_blocks;
    const int bc = rest / a.H;
    j.h = rest % a.H;
    j.q0 = qb * p.q_block, j.q1 = min(a.Q, j.q0 + p.q_block);
    j.b0 = bc * p.b_chunk, j.b1 = min(a.B, j.b0 + p.b_chunk);
    j.part = qb * p.b_chunks + bc;
    j.rc = rel_const(a.Q, a.K, a.grid_w);
    j.rlo = j.rc - rel_u(j.q1 - 1, a.grid_w);                         // the first relative position that its queries reach
    j.win = j.rc + rel_u(a.K - 1, a.grid_w) - rel_u(j.q0, a.grid_w) - j.rlo + 1;
    return j;
}

// One row's vectors as loaded, and which of their elements the query sees.
template <typename T, int NV, bool BACK> struct RelRow {
    Raw<T, 8> s[NV], d[BACK ? NV : 1];
    uint32_t seen[NV];

    // k0 of vector j is first + 8 * lanes * j; keys from `end` on are not seen (0: nothing is loaded)
    __device__ __forceinline__ void load(const RelArgs &a, int64_t at, int b, int q, int first, int lanes, int end, int64_t total)
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k0 = first + 8 * lanes * j;
            s[j].zero();
            if (BACK) d[j].zero();
            seen[j] = 0;
            if (k0 < end) {
                load_inside(s[j], static_cast<const T *>(a.s), at + k0, total);
                if (BACK) load_inside(d[j], static_cast<const T *>(a.dp), at + k0, total);
                seen[j] = end - k0 >= 8 ? 0xFFu : (1u << (end - k0)) - 1u;
                if (a.mask)
                    seen[j] &= load_mask(a.mask, (static_cast<int64_t>(b % a.mask_batches) * a.mask_rows + (a.mask_rows > 1 ? q : 0)) * a.K + k0,
                                         static_cast<int64_t>(a.mask_batches) * a.mask_rows * a.K);
            }
        }
    }
};

// z = scale s + bias where seen, minus infinity elsewhere: on entry z holds the bias, on return exp(z - top); the sum over the lane
template <typename T, int NV, bool BACK>
__device__ __forceinline__ float rel_scores(const RelRow<T, NV, BACK> &r, float scale, float *z)
{
    const float NONE = -__builtin_inff();
    float top = NONE;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float v[8];
        r.s[j].widen(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = __builtin_fmaf(v[e], scale, z[8 * j + e]);
            z[8 * j + e] = (r.seen[j] >> e) & 1u ? t : NONE;
            top = fmaxf(top, z[8 * j + e]);
        }
    }
    return top;
}

// the bucket's lane adds v: lanes hold (bucket or -1, value), acc of lane l is the sum of bucket l; whole wavefronts only
__device__ __forceinline__ void bucket_add(int c, float v, float &acc)
{
    const int lane = threadIdx.x & 63, c0 = __builtin_amdgcn_readfirstlane(c);
    if (__all(c == c0)) {                            // far distances share a bucket
        v = lanes_sum<64>(v);
        acc += lane == c0 ? v : 0.0f;
    } else {
        for (int i = 0; i < 64; ++i) {
            const int ci = __builtin_amdgcn_readlane(c, i);
            const float vi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), i));
            acc += lane == ci ? vi : 0.0f;
        }
    }
}

// A workgroup's sums by relative position leave it: value(i) of relative position rlo + i, by bucket where they are few.
template <typename Value>
__device__ __forceinline__ void rel_write_sums(const RelArgs &a, const RelPlan &p, const RelJob &job, float *lds, Value value)
{
    const int tid = threadIdx.x;
    float *w = a.ws + (static_cast<int64_t>(job.h) * p.q_blocks * p.b_chunks + job.part) * p.stride;
    if (!p.few) {
        for (int i = tid; i < job.win; i += kThreads) w[i] = value(i);
        return;
    }
    float acc = 0.0f;
    for (int i0 = tid & ~63; i0 < job.win; i0 += kThreads) {
        const int i = i0 + (tid & 63);
        const int c = i < job.win ? a.of[job.rlo + i] : -1;
        bucket_add(c >= 0 && c < a.n_buckets ? c : -1, i < job.win ? value(i) : 0.0f, acc);
    }
    __syncthreads();
    lds[tid] = acc;
    __syncthreads();
    if (tid < 64) w[tid] = (lds[tid] + lds[64 + tid]) + (lds[128 + tid] + lds[192 + tid]);
}

// Rows of up to 256 keys, 8, 16 or 32 lanes each: several to a wavefront.  A query's bias stays in registers through the batch, and so do the
// sums over the batch, which then meet in LDS: a thread sums those of one relative position.
template <typename T, int LANES, bool BACK>
__global__ __launch_bounds__(kThreads) void k_rel_rows(RelArgs a, RelPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int ROWS = kThreads / LANES, WIDTH = LANES * 8;
    const int tid = threadIdx.x, row = tid / LANES, lane = tid % LANES;
    const RelJob job = rel_job(a, p);
    const int gw = a.grid_w;
    float *bias = lds, *accw = bias + p.win, *tile = accw + (BACK ? p.win : 0);
    for (int i = tid; i < job.win; i += kThreads) {
        const int c = a.of[job.rlo + i];
        bias[i] = c >= 0 && c < a.n_buckets ? load_param(a.table, a.param_f32, static_cast<int64_t>(c) * a.H + job.h) : 0.0f;
        if (BACK) accw[i] = 0.0f;
    }
    const int64_t total = static_cast<int64_t>(a.B) * a.H * a.Q * a.K;
    const int Kp = (a.K + 7) & ~7, k0 = lane * 8;
    const int row_q = row % p.rows_q, row_b = row / p.rows_q;
    const float keep = BACK && a.drop.below ? a.drop.scale : 1.0f;
    RelRow<T, 1, BACK> next;
    auto fetch = [&](int qs, int bs) {
        const int q = qs + row_q, b = bs + row_b;
        const bool on = q < job.q1 && b < job.b1;
        const int end = on ? (a.causal ? min(a.K, q + a.K - a.Q + 1) : a.K) : 0;
        next.load(a, ((static_cast<int64_t>(b) * a.H + job.h) * a.Q + q) * a.K, b, q, k0, LANES, end, total);
    };
    fetch(job.q0, job.b0);
    __syncthreads();
    for (int qs = job.q0; qs < job.q1; qs += p.rows_q) {
        const int q = qs + row_q;
        float bv[8], acc[8];
        {
            int i = rel_u(k0, gw) - rel_u(q < job.q1 ? q : job.q1 - 1, gw) + job.rc - job.rlo, kx = gw ? k0 % gw : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                bv[e] = bias[k0 + e < a.K ? i : 0];
                acc[e] = 0.0f;
                ++i;
                if (gw && ++kx == gw) kx = 0, i += gw - 1;
            }
        }
        for (int bs = job.b0; bs < job.b1; bs += p.rows_b) {
            RelRow<T, 1, BACK> r = next;
            if (bs + p.rows_b < job.b1) fetch(qs, bs + p.rows_b);
            else if (qs + p.rows_q < job.q1) fetch(qs + p.rows_q, job.b0);
            const int b = bs + row_b;
            const int64_t line = (static_cast<int64_t>(b) * a.H + job.h) * a.Q + q;
            const bool on = b < job.b1 && q < job.q1 && k0 < a.K;
            float z[8], sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = bv[e];
            float top = lanes_max<LANES>(rel_scores<T, 1, BACK>(r, a.scale, z));
            if (top == -__builtin_inff()) top = 0.0f;                  // a row that sees nothing
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                z[e] = exp_of<EXACT>(z[e] - top);
                sum += z[e];
            }
            sum = lanes_sum<LANES>(sum);
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] *= inv;
            if constexpr (!BACK) {
                if (on) {
                    if (a.drop.below) drop_values<8>(z, line * Kp + k0, a.drop);
                    store_first(static_cast<T *>(a.out) + line * a.K + k0, z, a.K - k0);
                }
            } else {
                float d[8], dot = 0.0f;
                keep_bits(r.d[0], r.seen[0]);                          // whatever stands where nothing is seen
                if (a.drop.below) drop_raw(r.d[0], line * Kp + k0, a.drop);
                r.d[0].widen(d);
#pragma unroll
                for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(z[e], d[e], dot);
                dot = keep * lanes_sum<LANES>(dot);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float dz = z[e] * __builtin_fmaf(d[e], keep, -dot);
                    acc[e] += dz;
                    d[e] = dz * a.scale;
                }
                if (on) store_first(static_cast<T *>(a.out) + line * a.K + k0, d, a.K - k0);
            }
        }
        if constexpr (BACK) {
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[row * WIDTH + k0 + e] = acc[e];
            __syncthreads();
            const int qe = min(job.q1, qs + p.rows_q);
            const int i0 = job.rc - rel_u(qe - 1, gw) - job.rlo, i1 = job.rc + rel_u(a.K - 1, gw) - rel_u(qs, gw) - job.rlo;
            for (int i = i0 + tid; i <= i1; i += kThreads) {
                float t = 0.0f;
                const int rel = job.rlo + i - job.rc;                  // u(k) - u(q)
                for (int y = 0; y < qe - qs; ++y) {
                    int k = rel + qs + y;
                    if (gw) {
                        const int uk = rel + rel_u(qs + y, gw), ky = uk >= 0 ? uk / (2 * gw - 1) : -1, kx = uk - ky * (2 * gw - 1);
                        k = uk >= 0 && kx < gw ? ky * gw + kx : -1;
                    }
                    if (k >= 0 && k < a.K)
                        for (int x = 0; x < p.rows_b; ++x) t += tile[(x * p.rows_q + y) * WIDTH + k];
                }
                accw[i] += t;
            }
            __syncthreads();
        }
    }
    if constexpr (BACK) rel_write_sums(a, p, job, tile, [&](int i) { return accw[i]; });
}

// Longer rows: a wavefront's (LANES = 64), or a workgroup's (LANES = 256).  The bias is read from LDS for every row, and a row's gradient
// of the bias is added to LDS at once, to the wavefront's own vector or, where the workgroup is one row, to the one: a
// row's relative positions are distinct, rows follow one another, so every sum has its order.
template <typename T, int LANES, int NV, bool GRID, bool BACK>
__global__ __launch_bounds__(kThreads) void k_rel_long(RelArgs a, RelPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4, WIDE = LANES == kThreads;
    constexpr int WAVES = kThreads / 64, VECTORS = BACK ? (WIDE ? 1 : WAVES) : 0, STEP = 8 * LANES;
    const int tid = threadIdx.x, row = tid / LANES, first = tid % LANES * 8;
    const RelJob job = rel_job(a, p);
    const int gw = GRID ? a.grid_w : 0;
    const int size = rel_vector(p, gw);
    float *bias = lds, *sums = lds + size, *red = sums + VECTORS * size;
    for (int i = tid; i < job.win; i += kThreads) {
        const int c = a.of[job.rlo + i], at = GRID ? i : padded(i);
        bias[at] = c >= 0 && c < a.n_buckets ? load_param(a.table, a.param_f32, static_cast<int64_t>(c) * a.H + job.h) : 0.0f;
    }
    for (int i = tid; i < VECTORS * size; i += kThreads) sums[i] = 0.0f;
    const int64_t total = static_cast<int64_t>(a.B) * a.H * a.Q * a.K;
    const int Kp = (a.K + 7) & ~7;
    const int row_q = row % p.rows_q, row_b = row / p.rows_q;
    const float keep = BACK && a.drop.below ? a.drop.scale : 1.0f;
    float *mine = sums + (WIDE ? 0 : (tid >> 6) * size);
    auto end_of = [&](int q, int b) {
        return q < job.q1 && b < job.b1 ? (a.causal ? min(a.K, q + a.K - a.Q + 1) : a.K) : 0;
    };
    // f(j, e, place in LDS) for the lane's keys of vector j
    auto places = [&](int j, int q, auto f) {
        const int k0 = first + STEP * j;
        if constexpr (GRID) {
            int i = rel_u(k0, gw) - rel_u(q, gw) + job.rc - job.rlo, kx = k0 % gw;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f(e, k0 + e < a.K ? i : 0, k0 + e < a.K);
                ++i;
                if (++kx == gw) kx = 0, i += gw - 1;
            }
        } else {
            // padded(k0 + shift + e), k0 a multiple of 8 and shift the wavefront's own: 9 k0 / 8 + padded(shift + e)
            const int shift = __builtin_amdgcn_readfirstlane(job.rc - job.rlo - q);
#pragma unroll
            for (int e = 0; e < 8; ++e) f(e, k0 + e < a.K ? k0 + (k0 >> 3) + padded(shift + e) : 0, k0 + e < a.K);
        }
    };
    __syncthreads();
    for (int qs = job.q0; qs < job.q1; qs += p.rows_q) {
        const int q = qs + row_q;
        for (int bs = job.b0; bs < job.b1; bs += p.rows_b) {
            const int b = bs + row_b;
            const bool on = b < job.b1 && q < job.q1;
            const int64_t line = (static_cast<int64_t>(b) * a.H + job.h) * a.Q + q;
            const int end = end_of(q, b);
            RelRow<T, NV, BACK> r;
            r.load(a, line * a.K, b, q, first, LANES, end, total);
            float z[8 * NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) places(j, min(q, job.q1 - 1), [&](int e, int at, bool) { z[8 * j + e] = bias[at]; });
            float top = rel_scores<T, NV, BACK>(r, a.scale, z), sum = 0.0f;
            if constexpr (WIDE) {
                top = lanes_max<64>(top);
                if ((tid & 63) == 0) red[tid >> 6] = top;
                __syncthreads();
                top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
            } else {
                top = lanes_max<LANES>(top);
            }
            if (top == -__builtin_inff()) top = 0.0f;                  // a row that sees nothing
#pragma unroll
            for (int e = 0; e < 8 * NV; ++e) {
                z[e] = exp_of<EXACT>(z[e] - top);
                sum += z[e];
            }
            if constexpr (WIDE) {
                sum = lanes_sum<64>(sum);
                if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
                __syncthreads();
                sum = (red[4] + red[5]) + (red[6] + red[7]);
            } else {
                sum = lanes_sum<LANES>(sum);
            }
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int e = 0; e < 8 * NV; ++e) z[e] *= inv;
            if constexpr (!BACK) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k0 = first + STEP * j;
                    if (on && k0 < a.K) {
                        if (a.drop.below) drop_values<8>(z + 8 * j, line * Kp + k0, a.drop);
                        store_first(static_cast<T *>(a.out) + line * a.K + k0, z + 8 * j, a.K - k0);
                    }
                }
            } else {
                float dot = 0.0f, d[8];
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    keep_bits(r.d[j], r.seen[j]);                      // whatever stands where nothing is seen
                    if (a.drop.below) drop_raw(r.d[j], line * Kp + first + STEP * j, a.drop);
                    r.d[j].widen(d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(z[8 * j + e], d[e], dot);
                }
                if constexpr (WIDE) {
                    dot = lanes_sum<64>(dot);
                    if ((tid & 63) == 0) red[8 + (tid >> 6)] = dot;
                    __syncthreads();
                    dot = keep * ((red[8] + red[9]) + (red[10] + red[11]));
                } else {
                    dot = keep * lanes_sum<LANES>(dot);
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k0 = first + STEP * j;
                    if (!on || k0 >= a.K) continue;
                    r.d[j].widen(d);
                    float dz[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        dz[e] = z[8 * j + e] * __builtin_fmaf(d[e], keep, -dot);
                        d[e] = dz[e] * a.scale;
                    }
                    if (r.seen[j]) {
                        float was[8];
                        places(j, q, [&](int e, int at, bool) { was[e] = mine[at]; });
                        places(j, q, [&](int e, int at, bool in) {
                            if (in) mine[at] = was[e] + dz[e];
                        });
                    }
                    store_first(static_cast<T *>(a.out) + line * a.K + k0, d, a.K - k0);
                }
            }
        }
    }
    if constexpr (BACK) {
        __syncthreads();
        rel_write_sums(a, p, job, lds, [&](int i) {
            const int at = GRID ? i : padded(i);
            float t = sums[at];
#pragma unroll
            for (int v = 1; v < VECTORS; ++v) t += sums[v * size + at];
            return t;
        });
    }
}

// dtable[c, h] of head blockIdx.x where the workgroups have summed by bucket: 16 wavefronts take their rows in turns, a lane a bucket.
__global__ __launch_bounds__(1024) void k_rel_few_buckets(RelArgs a, RelPlan p)
{
    __shared__ float part[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = blockIdx.x, parts = p.q_blocks * p.b_chunks;
    const float *w = a.ws + static_cast<int64_t>(h) * parts * kFewBuckets + lane;
    float t = 0.0f;
    int k = wave;
    for (; k + 7 * 16 < parts; k += 8 * 16) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[(k + 16 * i) * kFewBuckets];
#pragma unroll
        for (int i = 0; i < 8; ++i) t += v[i];
    }
    for (; k < parts; k += 16) t += w[k * kFewBuckets];
    part[wave][lane] = t;
    __syncthreads();
    if (wave == 0 && lane < a.n_buckets) {
        t = part[0][lane];
        for (int i = 1; i < 16; ++i) t += part[i][lane];
        store_param(a.dtable, a.param_f32, static_cast<int64_t>(lane) * a.H + h, t);
    }
}

// The same for many buckets, 64 of them from 64 * blockIdx.x on of head blockIdx.y, from the workgroups' sums by relative position: those that
// belong to the 64 buckets are listed in their order, 1024 at a time; 64 of the list go through the workgroups' vectors together, a wavefront
// to every 16th vector, and then to their buckets, a lane each.
__global__ __launch_bounds__(1024) void k_rel_many_buckets(RelArgs a, RelPlan p, int n_rel)
{
    __shared__ int list[1024], of[1024], count[16];
    __shared__ float part[16][64];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, h = blockIdx.y;
    const int c0 = blockIdx.x * 64, c1 = min(a.n_buckets, c0 + 64);
    const int gw = a.grid_w, rc = rel_const(a.Q, a.K, gw), parts = p.q_blocks * p.b_chunks, ulast = rel_u(a.K - 1, gw);
    const float *w = a.ws + static_cast<int64_t>(h) * parts * p.stride;
    float acc = 0.0f;                                     // of bucket c0 + lane, in wavefront 0
    for (int r0 = 0; r0 < n_rel; r0 += 1024) {
        const int c = r0 + tid < n_rel ? a.of[r0 + tid] : -1;
        const bool in = c >= c0 && c < c1;
        const uint64_t ballot = __ballot(in);
        if (lane == 0) count[wave] = __popcll(ballot);
        __syncthreads();
        int before = 0, all = 0;
        for (int i = 0; i < 16; ++i) {
            before += i < wave ? count[i] : 0;
            all += count[i];
        }
        if (in) {
            const int at = before + __popcll(ballot & ((1ull << lane) - 1));
            list[at] = r0 + tid;
            of[at] = c - c0;
        }
        __syncthreads();
        for (int e0 = 0; e0 < all; e0 += 64) {
            const int r = e0 + lane < all ? list[e0 + lane] : -1;
            float t = 0.0f;
            for (int k = wave; k < parts; k += 16 * 4) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int kk = k + 16 * i, qb = kk / p.b_chunks;
                    const int q0 = qb * p.q_block, q1 = min(a.Q, q0 + p.q_block), at = r - (rc - rel_u(q1 - 1, gw));
                    const bool reach = kk < parts && r >= 0 && at >= 0 && at <= ulast - rel_u(q0, gw) + rel_u(q1 - 1, gw);
                    v[i] = reach ? w[static_cast<int64_t>(kk) * p.stride + at] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) t += v[i];
            }
            part[wave][lane] = t;
            __syncthreads();
            if (wave == 0) {
                t = part[0][lane];
                for (int i = 1; i < 16; ++i) t += part[i][lane];
                bucket_add(r >= 0 ? of[e0 + lane] : -1, t, acc);
            }
            __syncthreads();
        }
    }
    if (wave == 0 && c0 + lane < c1) store_param(a.dtable, a.param_f32, static_cast<int64_t>(c0 + lane) * a.H + h, acc);
}

bool rel_softmax_ok(int K, int grid_w) { return K <= (grid_w ? kMaxKeysGrid : kMaxKeysSequence); }

size_t rel_softmax_ws_bytes(const RelArgs &a)
{
    if (a.B == 0 || a.Q == 0 || a.K == 0) return 0;
    const RelPlan p = rel_plan(a, true);
    return static_cast<size_t>(a.H) * p.q_blocks * p.b_chunks * p.stride * sizeof(float);
}

static hipError_t run(void (*f)(RelArgs, RelPlan), const RelArgs &a, const RelPlan &p, bool back, hipStream_t st)
{
    const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(a.H) * p.q_blocks * p.b_chunks);
    const size_t lds = rel_lds_bytes(p, a.grid_w, back);
    if (lds > 65536)
        if (const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds))) return e;
    f<<<blocks, kThreads, lds, st>>>(a, p);
    return hipGetLastError();
}

template <typename T, bool BACK>
static hipError_t by_length(const RelArgs &a, const RelPlan &p, hipStream_t st)
{
    const bool grid = a.grid_w != 0;
    switch (p.lanes * 16 + p.nv) {
        case 8 * 16 + 1: return run(k_rel_rows<T, 8, BACK>, a, p, BACK, st);
        case 16 * 16 + 1: return run(k_rel_rows<T, 16, BACK>, a, p, BACK, st);
        case 32 * 16 + 1: return run(k_rel_rows<T, 32, BACK>, a, p, BACK, st);
        case 64 * 16 + 1: return run(grid ? k_rel_long<T, 64, 1, true, BACK> : k_rel_long<T, 64, 1, false, BACK>, a, p, BACK, st);
        case 64 * 16 + 2: return run(grid ? k_rel_long<T, 64, 2, true, BACK> : k_rel_long<T, 64, 2, false, BACK>, a, p, BACK, st);
        case 64 * 16 + 4: return run(grid ? k_rel_long<T, 64, 4, true, BACK> : k_rel_long<T, 64, 4, false, BACK>, a, p, BACK, st);
        case 256 * 16 + 2: return run(grid ? k_rel_long<T, 256, 2, true, BACK> : k_rel_long<T, 256, 2, false, BACK>, a, p, BACK, st);
        case 256 * 16 + 4: return run(k_rel_long<T, 256, 4, false, BACK>, a, p, BACK, st);
        default: return run(k_rel_long<T, 256, 8, false, BACK>, a, p, BACK, st);
    }
}

hipError_t launch_rel_softmax(const RelArgs &a, hipStream_t st)
{
    const RelPlan p = rel_plan(a, false);
    return a.is_f32 ? by_length<float, false>(a, p, st) : by_length<bf16_t, false>(a, p, st);
}

hipError_t launch_rel_softmax_backward(const RelArgs &a, hipStream_t st)
{
    RelPlan p{};
    int n_rel = 0;
    if (a.B && a.Q && a.K) {
        p = rel_plan(a, true);
        n_rel = a.grid_w ? 2 * rel_u(a.K - 1, a.grid_w) + 1 : a.Q + a.K - 1;
        if (const hipError_t e = a.is_f32 ? by_length<float, true>(a, p, st) : by_length<bf16_t, true>(a, p, st)) return e;
    }
    if (!a.dtable) return hipSuccess;
    if (p.few) k_rel_few_buckets<<<a.H, 1024, 0, st>>>(a, p);
    else k_rel_many_buckets<<<dim3((a.n_buckets + 63) / 64, a.H), 1024, 0, st>>>(a, p, n_rel);      // without rows: zeros
    return hipGetLastError();
}

}  // namespace hlq
