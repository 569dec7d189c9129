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
};

namespace {

constexpr int kThreads = 256;
constexpr int kMaxKeysSequence = 16384, kMaxKeysGrid = 4096;     // two vectors of them (u stretches a grid's to two each) in LDS

__host__ __device__ __forceinline__ int rel_u(int k, int gw) { return gw ? k / gw * (2 * gw - 1) + k % gw : k; }
// rel(q, k) = u(k) - u(q) + rel_const
__host__ __device__ __forceinline__ int rel_const(int Q, int K, int gw) { return gw ? rel_u(K - 1, gw) : Q - 1; }

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
    return p;
}

size_t rel_lds_bytes(const RelPlan &p, bool back)
{
    const int rows = kThreads / p.lanes;
    const size_t tile = back && rows > 1 ? static_cast<size_t>(rows) * p.lanes * p.nv * 8 : 0;
    return sizeof(float) * (static_cast<size_t>(p.win) * (back ? 2 : 1) + tile + 16);
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
__device__ __forceinline__ uint64_t load_mask(const uint8_t *base, int64_t at, int64_t total)
{
    uint64_t m = 0;
    if (at + 8 <= total) {
        __builtin_memcpy(&m, base + at, 8);
    } else {
        for (int e = 0; e < 8 && at + e < total; ++e) m |= static_cast<uint64_t>(base[at + e]) << (8 * e);
    }
    return m;
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

template <typename T, int LANES, int NV, bool BACK>
__global__ __launch_bounds__(kThreads) void k_rel(RelArgs a, RelPlan p)
{
    extern __shared__ float lds[];
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr bool WIDE = LANES == kThreads;
    constexpr int ROWS = kThreads / LANES, NE = 8 * NV;
    const float NONE = -__builtin_inff();
    const int tid = threadIdx.x, row = tid / LANES, lane = tid % LANES;
    const int qb = blockIdx.x % p.q_blocks, rest = blockIdx.x / p.q_blocks, h = rest % a.H, bc = rest / a.H;
    const int q0 = qb * p.q_block, q1 = min(a.Q, q0 + p.q_block), b0 = bc * p.b_chunk, b1 = min(a.B, b0 + p.b_chunk);
    const int gw = a.grid_w, rc = rel_const(a.Q, a.K, gw);
    const int rlo = rc - rel_u(q1 - 1, gw), win = rc + rel_u(a.K - 1, gw) - rel_u(q0, gw) - rlo + 1;
    float *bias = lds, *accw = lds + p.win, *tile = accw + (BACK ? p.win : 0), *red = tile + (BACK && !WIDE ? ROWS * LANES * NE : 0);
    for (int i = tid; i < win; i += kThreads) {
        const int c = a.of[rlo + i];
        bias[i] = c >= 0 && c < a.n_buckets ? load_param(a.table, a.param_f32, static_cast<int64_t>(c) * a.H + h) : 0.0f;
        if (BACK) accw[i] = 0.0f;
    }
    __syncthreads();
    const T *S = static_cast<const T *>(a.s), *dP = static_cast<const T *>(a.dp);
    T *out = static_cast<T *>(a.out);
    const int64_t total = static_cast<int64_t>(a.B) * a.H * a.Q * a.K;
    const int64_t mask_total = static_cast<int64_t>(a.mask_batches) * a.mask_rows * a.K;
    const int Kp = (a.K + 7) & ~7;
    const int row_q = row % p.rows_q, row_b = row / p.rows_q;
    for (int qs = q0; qs < q1; qs += p.rows_q) {
        const int q = qs + row_q;
        const int seen_end = q >= q1 ? 0 : (a.causal ? min(a.K, q + a.K - a.Q + 1) : a.K);      // keys from here on are not seen
        float bv[NE], acc[NE];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k0 = (j * LANES + lane) * 8;
            int i = rel_u(k0, gw) - rel_u(q < q1 ? q : q1 - 1, gw) + rc - rlo, kx = gw ? k0 % gw : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                bv[8 * j + e] = bias[k0 + e < a.K ? i : 0];
                acc[8 * j + e] = 0.0f;
                ++i;
                if (gw && ++kx == gw) kx = 0, i += gw - 1;
            }
        }
        for (int bs = b0; bs < b1; bs += p.rows_b) {
            const int b = bs + row_b;
            const bool on = b < b1 && q < q1;
            const int64_t r = (static_cast<int64_t>(b) * a.H + h) * a.Q + q, at = r * a.K;
            Raw<T, 8> rs[NV], rd[NV];
            uint64_t mk[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k0 = (j * LANES + lane) * 8;
                rs[j].zero();
                if (BACK) rd[j].zero();
                mk[j] = 0;
                if (on && k0 < seen_end) {
                    load_inside(rs[j], S, at + k0, total);
                    if (BACK) load_inside(rd[j], dP, at + k0, total);
                    mk[j] = ~0ull;
                    if (a.mask) mk[j] = load_mask(a.mask, (static_cast<int64_t>(b % a.mask_batches) * a.mask_rows + (a.mask_rows > 1 ? q : 0)) * a.K + k0, mask_total);
                }
            }
            float z[NE], top = NONE;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k0 = (j * LANES + lane) * 8;
                rs[j].widen(z + 8 * j);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool seen = k0 + e < seen_end && ((mk[j] >> (8 * e)) & 0xFF) != 0;
                    z[8 * j + e] = seen ? __builtin_fmaf(z[8 * j + e], a.scale, bv[8 * j + e]) : NONE;
                    top = fmaxf(top, z[8 * j + e]);
                }
            }
            if constexpr (WIDE) {
                top = lanes_max<64>(top);
                if ((tid & 63) == 0) red[tid >> 6] = top;
                __syncthreads();
                top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
            } else {
                top = lanes_max<LANES>(top);
            }
            if (top == NONE) top = 0.0f;                  // a row that sees nothing
            float pr[NE], sum = 0.0f;
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                pr[e] = exp_of<EXACT>(z[e] - top);
                sum += pr[e];
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
            for (int e = 0; e < NE; ++e) pr[e] *= inv;
            if constexpr (!BACK) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k0 = (j * LANES + lane) * 8;
                    if (on && k0 < a.K) {
                        if (a.drop.below) drop_values<8>(pr + 8 * j, r * Kp + k0, a.drop);
                        store_first(out + at + k0, pr + 8 * j, a.K - k0);
                    }
                }
            } else {
                float dot = 0.0f, dp[NE];
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k0 = (j * LANES + lane) * 8;
                    rd[j].widen(dp + 8 * j);
                    if (a.drop.below) drop_values<8>(dp + 8 * j, r * Kp + k0, a.drop);
#pragma unroll
                    for (int e = 8 * j; e < 8 * j + 8; ++e) {
                        dp[e] = z[e] == NONE ? 0.0f : dp[e];       // whatever stands where nothing is seen
                        dot = __builtin_fmaf(pr[e], dp[e], dot);
                    }
                }
                if constexpr (WIDE) {
                    dot = lanes_sum<64>(dot);
                    if ((tid & 63) == 0) red[8 + (tid >> 6)] = dot;
                    __syncthreads();
                    dot = (red[8] + red[9]) + (red[10] + red[11]);
                } else {
                    dot = lanes_sum<LANES>(dot);
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k0 = (j * LANES + lane) * 8;
#pragma unroll
                    for (int e = 8 * j; e < 8 * j + 8; ++e) {
                        const float dz = z[e] == NONE ? 0.0f : pr[e] * (dp[e] - dot);
                        acc[e] += dz;
                        dp[e] = dz * a.scale;
                    }
                    if (on && k0 < a.K) store_first(out + at + k0, dp + 8 * j, a.K - k0);
                }
            }
        }
        if constexpr (BACK) {
            if constexpr (WIDE) {
                // one query: its keys' relative positions are distinct
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k0 = (j * LANES + lane) * 8;
                    int i = rel_u(k0, gw) - rel_u(q, gw) + rc - rlo, kx = gw ? k0 % gw : 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (k0 + e < a.K) accw[i] += acc[8 * j + e];
                        ++i;
                        if (gw && ++kx == gw) kx = 0, i += gw - 1;
                    }
                }
                __syncthreads();
            } else {
                constexpr int WIDTH = LANES * NE;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) tile[row * WIDTH + (j * LANES + lane) * 8 + e] = acc[8 * j + e];
                }
                __syncthreads();
                const int qe = min(q1, qs + p.rows_q);
                const int i0 = rc - rel_u(qe - 1, gw) - rlo, i1 = rc + rel_u(a.K - 1, gw) - rel_u(qs, gw) - rlo;
                for (int i = i0 + tid; i <= i1; i += kThreads) {
                    float t = 0.0f;
                    const int rel = rlo + i - rc;                   // u(k) - u(q)
                    for (int y = 0; y < qe - qs; ++y) {
                        const int qq = qs + y;
                        int k;
                        if (gw) {
                            const int uk = rel + rel_u(qq, gw), ky = uk >= 0 ? uk / (2 * gw - 1) : -1, kx = uk - ky * (2 * gw - 1);
                            k = uk >= 0 && kx < gw ? ky * gw + kx : -1;
                        } else {
                            k = rel + qq;
                        }
                        if (k >= 0 && k < a.K)
                            for (int x = 0; x < p.rows_b; ++x) t += tile[(x * p.rows_q + y) * WIDTH + k];
                    }
                    accw[i] += t;
                }
                __syncthreads();
            }
        }
    }
    if constexpr (BACK) {
        float *w = a.ws + (static_cast<int64_t>(h) * p.q_blocks * p.b_chunks + qb * p.b_chunks + bc) * p.win;
        for (int i = tid; i < win; i += kThreads) w[i] = accw[i];
    }
}

// dtable[c, h] for `per` buckets from blockIdx.x * per on and head blockIdx.y: relative positions by 1024s, a thread sums the
// workgroups' values of one, a wavefront those of a bucket.
__global__ __launch_bounds__(1024) void k_rel_table_grad(RelArgs a, RelPlan p, int n_rel, int per)
{
    __shared__ float val[1024];
    __shared__ int of[1024];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, h = blockIdx.y;
    const int c0 = blockIdx.x * per, c1 = min(a.n_buckets, c0 + per);
    const int gw = a.grid_w, rc = rel_const(a.Q, a.K, gw), parts = p.q_blocks * p.b_chunks;
    float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};              // of buckets c0 + wave, + 16, + 32, + 48
    for (int r0 = 0; r0 < n_rel; r0 += 1024) {
        const int r = r0 + tid;
        const int c = r < n_rel ? a.of[r] : -1;
        float t = 0.0f;
        if (c >= c0 && c < c1) {
            for (int qb = 0; qb < p.q_blocks; ++qb) {
                const int q0 = qb * p.q_block, q1 = min(a.Q, q0 + p.q_block);
                const int i = r - (rc - rel_u(q1 - 1, gw));
                if (i < 0 || i > rel_u(a.K - 1, gw) - rel_u(q0, gw) + rel_u(q1 - 1, gw)) continue;
                const float *w = a.ws + (static_cast<int64_t>(h) * parts + qb * p.b_chunks) * p.win + i;
                for (int b = 0; b < p.b_chunks; ++b) t += w[static_cast<int64_t>(b) * p.win];
            }
        }
        val[tid] = t;
        of[tid] = c >= c0 && c < c1 ? c : -1;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int want = c0 + wave + 16 * k;
            if (want < c1)
                for (int i = lane; i < 1024; i += 64) sums[k] += of[i] == want ? val[i] : 0.0f;
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = c0 + wave + 16 * k;
        const float t = lanes_sum<64>(sums[k]);
        if (c < c1 && lane == 0) store_param(a.dtable, a.param_f32, static_cast<int64_t>(c) * a.H + h, t);
    }
}

bool rel_softmax_ok(int K, int grid_w) { return K <= (grid_w ? kMaxKeysGrid : kMaxKeysSequence); }

size_t rel_softmax_ws_bytes(const RelArgs &a)
{
    if (a.B == 0 || a.Q == 0 || a.K == 0) return 0;
    const RelPlan p = rel_plan(a, true);
    return static_cast<size_t>(a.H) * p.q_blocks * p.b_chunks * p.win * sizeof(float);
}

template <typename T, int LANES, int NV>
static hipError_t go(const RelArgs &a, const RelPlan &p, bool back, hipStream_t st)
{
    const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(a.H) * p.q_blocks * p.b_chunks);
    const size_t lds = rel_lds_bytes(p, back);
    const void *f = back ? reinterpret_cast<const void *>(k_rel<T, LANES, NV, true>) : reinterpret_cast<const void *>(k_rel<T, LANES, NV, false>);
    if (lds > 65536)
        if (const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds))) return e;
    if (back) k_rel<T, LANES, NV, true><<<blocks, kThreads, lds, st>>>(a, p);
    else k_rel<T, LANES, NV, false><<<blocks, kThreads, lds, st>>>(a, p);
    return hipGetLastError();
}

template <typename T>
static hipError_t by_length(const RelArgs &a, const RelPlan &p, bool back, hipStream_t st)
{
    switch (p.lanes * 16 + p.nv) {
        case 8 * 16 + 1: return go<T, 8, 1>(a, p, back, st);
        case 16 * 16 + 1: return go<T, 16, 1>(a, p, back, st);
        case 32 * 16 + 1: return go<T, 32, 1>(a, p, back, st);
        case 64 * 16 + 1: return go<T, 64, 1>(a, p, back, st);
        case 64 * 16 + 2: return go<T, 64, 2>(a, p, back, st);
        case 64 * 16 + 4: return go<T, 64, 4>(a, p, back, st);
        case 256 * 16 + 2: return go<T, 256, 2>(a, p, back, st);
        case 256 * 16 + 4: return go<T, 256, 4>(a, p, back, st);
        default: return go<T, 256, 8>(a, p, back, st);
    }
}

hipError_t launch_rel_softmax(const RelArgs &a, hipStream_t st)
{
    const RelPlan p = rel_plan(a, false);
    return a.is_f32 ? by_length<float>(a, p, false, st) : by_length<bf16_t>(a, p, false, st);
}

hipError_t launch_rel_softmax_backward(const RelArgs &a, hipStream_t st)
{
    RelPlan p{};
    if (a.B && a.Q && a.K) {
        p = rel_plan(a, true);
        if (const hipError_t e = a.is_f32 ? by_length<float>(a, p, true, st) : by_length<bf16_t>(a, p, true, st)) return e;
    }
    if (!a.dtable) return hipSuccess;
    const int n_rel = a.B && a.Q && a.K ? (a.grid_w ? 2 * rel_u(a.K - 1, a.grid_w) + 1 : a.Q + a.K - 1) : 0;
    const int per = a.n_buckets >= 64 ? 64 : 16;
    k_rel_table_grad<<<dim3((a.n_buckets + per - 1) / per, a.H), 1024, 0, st>>>(a, p, n_rel, per);
    return hipGetLastError();
}

}  // namespace hlq
