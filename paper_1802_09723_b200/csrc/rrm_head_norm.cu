// Group normalisation with an activation, channels last, and its backward pass.
//
// A unit of work is one image's block of whole groups (CB channels): a cluster of blocks takes it, each block a run of its
// pixels.  Forward, a block reads its values once into shared memory, accumulates count, mean and the sum of squared
// distances from the mean (a batch of rows at a time, merged by the pairwise update of Chan, Golub and LeVeque 1983, so
// that a mean far from zero costs no digits), the cluster's blocks merge theirs, and each normalises what it holds: x is
// read once and y written once.  Backward, with z = xhat gamma + beta, dz = dy act'(z) and v = dz gamma,
//   dx = rstd (v - mean(v) - xhat mean(v xhat)),  dgamma = sum(dz xhat),  dbeta = sum(dz),
// the group's two means are sums of gamma times the image's per-channel sums, so a block accumulates the two sums of
// each channel; the images' sums are added up by a second small launch in image order.  A unit too large for the
// cluster's shared memory is read a second time instead (from L2 as far as it reaches).
//
// What bounds it: memory, and for small calls the launch and the cluster's exchange.
#include "rrm_common.cuh"
#include "rrm_head.cuh"
#include <climits>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace rrm {
namespace {

constexpr int NORM_THREADS = 256;
constexpr int NORM_CLUSTER = 8;
constexpr int NORM_MAX_GROUP = 8192;          // channels of one group
constexpr int NORM_MAX_C = 65536;
constexpr int NORM_MAX_PIXELS = 1 << 30;      // row counters are ints
constexpr int NORM_BATCH = 4;                 // rows a thread has in flight

struct NormParams {
    const void *x, *dy;
    const float *gamma, *beta;
    const float* stats_in;
    void *y, *dx;
    float *stats, *dgamma, *dbeta;
    float* sums;                              // [n][c][2] per-image channel sums (n > 1)
    long long x_pixel, x_image, y_pixel, y_image, dx_pixel, dx_image;
    int n, pixels, c, groups, per, cb, blocks_c;
    float eps;
    int act;
    int resident;                             // the unit's values stay in shared memory
};

// what a thread works on: V neighbouring channels (a slot) of every R-th pixel of the block's run
struct NormSpot {
    int image, c0, cb, p0, p1, rank, ranks;
    __device__ explicit NormSpot(const NormParams& p)
    {
        const cg::cluster_group cluster = cg::this_cluster();
        rank = (int)cluster.block_rank();
        ranks = (int)cluster.num_blocks();
        const unsigned unit = blockIdx.x / ranks;
        image = (int)(unit / p.blocks_c);
        c0 = (int)(unit % p.blocks_c) * p.cb;
        cb = min(p.cb, p.c - c0);
        const int share = (p.pixels + ranks - 1) / ranks;
        p0 = min(rank * share, p.pixels);
        p1 = min(p0 + share, p.pixels);
    }
};

template <int V> __device__ __forceinline__ void act_values(int act, float (&z)[V])
{
    switch (act) {                             // one branch for the V values
        case RRM_ACT_NONE: break;
        case RRM_ACT_RELU:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = act_value(RRM_ACT_RELU, z[v]);
            break;
        case RRM_ACT_SILU:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = act_value(RRM_ACT_SILU, z[v]);
            break;
        default:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = act_value(act, z[v]);
    }
}

template <int V> __device__ __forceinline__ void act_slopes(int act, float (&z)[V])
{
    float value;
    switch (act) {
        case RRM_ACT_NONE:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = 1.f;
            break;
        case RRM_ACT_RELU:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = act_slope(RRM_ACT_RELU, z[v], value);
            break;
        case RRM_ACT_SILU:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = act_slope(RRM_ACT_SILU, z[v], value);
            break;
        default:
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = act_slope(act, z[v], value);
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
    #pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Forward.  NS = V / SUB groups share a slot (SUB = V: a slot lies inside one group).
template <typename T, int V, int SUB>
__global__ void __launch_bounds__(NORM_THREADS) norm_kernel(const __grid_constant__ NormParams p)
{
    constexpr int NS = V / SUB;
    extern __shared__ __align__(16) char smem[];
    const NormSpot s(p);
    const cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, slots = s.cb / V, lanes = min(slots, NORM_THREADS), rows = NORM_THREADS / lanes;
    const int row0 = tid / lanes, gb = s.cb / p.per;
    const bool works = row0 < rows;
    const int entries = max(rows * lanes, slots) * NS;
    float* part_mean = reinterpret_cast<float*>(smem);          // [rows][slots][NS]
    float* part_m2 = part_mean + entries;
    float* block_stat = part_m2 + entries;                      // [gb][2] mean, M2 of the block's pixels
    float* final_stat = block_stat + 2 * gb;                    // [gb][2] mean, rstd
    Pack<T, V>* tile = reinterpret_cast<Pack<T, V>*>(smem + ((2 * entries + 4 * gb) * 4 + 15) / 16 * 16);
    const T* x = reinterpret_cast<const T*>(p.x) + s.image * p.x_image + s.c0;

    // ---- the block's mean and sum of squared distances of every group
    for (int sp = 0; sp < slots; sp += lanes) {
        const int slot = sp + tid % lanes;
        if (!works || slot >= slots) continue;
        float count = 0.f, mean[NS], m2[NS];
        #pragma unroll
        for (int i = 0; i < NS; ++i) mean[i] = m2[i] = 0.f;
        for (int px = s.p0 + row0; px < s.p1; px += rows * NORM_BATCH) {
            Pack<T, V> in[NORM_BATCH];
            int got = 0;
            #pragma unroll
            for (int b = 0; b < NORM_BATCH; ++b) {
                const int q = px + b * rows;
                if (q < s.p1) {
                    in[b] = load_pack<T, V>(x + q * p.x_pixel + slot * V);
                    got = b + 1;
                }
            }
            if (p.resident) {
                #pragma unroll
                for (int b = 0; b < NORM_BATCH; ++b)
                    if (b < got) tile[(px + b * rows - s.p0) * slots + slot] = in[b];
            }
            const float m = (float)(got * SUB), inv = 1.f / m, total = count + m, share = m / total;
            #pragma unroll
            for (int i = 0; i < NS; ++i) {
                float sum = 0.f, q = 0.f;
                #pragma unroll
                for (int b = 0; b < NORM_BATCH; ++b)
                    #pragma unroll
                    for (int v = 0; v < SUB; ++v) sum += b < got ? to_f32(in[b].v[i * SUB + v]) : 0.f;
                const float bm = sum * inv;
                #pragma unroll
                for (int b = 0; b < NORM_BATCH; ++b)
                    #pragma unroll
                    for (int v = 0; v < SUB; ++v) {
                        const float t = to_f32(in[b].v[i * SUB + v]) - bm;
                        if (b < got) q = fmaf(t, t, q);
                    }
                const float gap = bm - mean[i];
                mean[i] = fmaf(gap, share, mean[i]);
                m2[i] += q + gap * gap * (count * share);
            }
            count = total;
        }
        #pragma unroll
        for (int i = 0; i < NS; ++i) {
            part_mean[(row0 * slots + slot) * NS + i] = mean[i];
            part_m2[(row0 * slots + slot) * NS + i] = m2[i];
        }
    }
    __syncthreads();
    // a warp a group; row r of the block has seen ceil((pixels - r) / rows) of its pixels
    const int wide = SUB == V ? p.per / V : 1;                  // slots of one group
    const int run = s.p1 - s.p0;
    for (int g = tid / 32; g < gb; g += NORM_THREADS / 32) {
        const int n_e = rows * wide;
        float sum = 0.f, q = 0.f;
        auto at = [&](int e, float& cnt) {
            const int r = e / wide, k = e - r * wide;
            cnt = (float)((run - r + rows - 1) / rows * SUB);
            if (run <= r) cnt = 0.f;
            return SUB == V ? r * slots + g * wide + k : (r * slots + g / NS) * NS + g % NS;
        };
        float cnt;
        for (int e = tid & 31; e < n_e; e += 32) { const int i = at(e, cnt); sum += cnt > 0.f ? cnt * part_mean[i] : 0.f; }
        const float all = (float)run * (float)p.per;
        const float mean = run > 0 ? warp_sum(sum) / all : 0.f;
        for (int e = tid & 31; e < n_e; e += 32) {
            const int i = at(e, cnt);
            const float gap = part_mean[i] - mean;
            if (cnt > 0.f) q += fmaf(cnt * gap, gap, part_m2[i]);
        }
        q = warp_sum(q);
        if ((tid & 31) == 0) { block_stat[2 * g] = mean; block_stat[2 * g + 1] = q; }
    }
    if (s.ranks > 1) cluster.sync(); else __syncthreads();
    // ---- the cluster's
    const int share_px = (p.pixels + s.ranks - 1) / s.ranks;
    for (int g = tid; g < gb; g += NORM_THREADS) {
        float mean = 0.f, q = 0.f;
        for (int r = 0; r < s.ranks; ++r) {
            const int cnt = max(0, min(p.pixels - r * share_px, share_px));
            mean += (float)cnt * cluster.map_shared_rank(block_stat, r)[2 * g];
        }
        mean /= (float)p.pixels;
        for (int r = 0; r < s.ranks; ++r) {
            const int cnt = max(0, min(p.pixels - r * share_px, share_px));
            const float* o = cluster.map_shared_rank(block_stat, r);
            const float gap = o[2 * g] - mean;
            if (cnt > 0) q += fmaf((float)cnt * (float)p.per * gap, gap, o[2 * g + 1]);
        }
        const float rstd = rsqrtf(q / ((float)p.pixels * (float)p.per) + p.eps);
        final_stat[2 * g] = mean;
        final_stat[2 * g + 1] = rstd;
        if (p.stats && s.rank == 0) {
            float* o = p.stats + ((long long)s.image * p.groups + s.c0 / p.per + g) * 2;
            o[0] = mean;
            o[1] = rstd;
        }
    }
    __syncthreads();

    // ---- normalise what the block holds
    T* y = reinterpret_cast<T*>(p.y) + s.image * p.y_image + s.c0;
    for (int sp = 0; sp < slots; sp += lanes) {
        const int slot = sp + tid % lanes;
        if (!works || slot >= slots) continue;
        float mean[NS], scale[V], shift[V];
        #pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int g = (slot * V + i * SUB) / p.per;
            mean[i] = final_stat[2 * g];
            #pragma unroll
            for (int v = 0; v < SUB; ++v) {
                const int ch = s.c0 + slot * V + i * SUB + v;
                scale[i * SUB + v] = final_stat[2 * g + 1] * (p.gamma ? p.gamma[ch] : 1.f);
                shift[i * SUB + v] = p.beta ? p.beta[ch] : 0.f;
            }
        }
        #pragma unroll 2
        for (int px = s.p0 + row0; px < s.p1; px += rows) {
            const Pack<T, V> in = p.resident ? tile[(px - s.p0) * slots + slot] : load_pack<T, V>(x + px * p.x_pixel + slot * V);
            float z[V];
            #pragma unroll
            for (int v = 0; v < V; ++v) z[v] = fmaf(to_f32(in.v[v]) - mean[v / SUB], scale[v], shift[v]);
            act_values<V>(p.act, z);
            Pack<T, V> out;
            #pragma unroll
            for (int v = 0; v < V; ++v) out.v[v] = from_f32<T>(z[v]);
            store_pack<T, V>(y + px * p.y_pixel + slot * V, out);
        }
    }
    if (s.ranks > 1) cluster.sync();                             // no block leaves while another may read its statistics
}

// Backward.
template <typename T, int V, int SUB>
__global__ void __launch_bounds__(NORM_THREADS) norm_backward_kernel(const __grid_constant__ NormParams p)
{
    constexpr int NS = V / SUB;
    extern __shared__ __align__(16) char smem[];
    const NormSpot s(p);
    const cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, slots = s.cb / V, lanes = min(slots, NORM_THREADS), rows = NORM_THREADS / lanes;
    const int row0 = tid / lanes, gb = s.cb / p.per;
    const bool works = row0 < rows;
    const int entries = rows * slots * V;
    float* part_g = reinterpret_cast<float*>(smem);             // [rows][cb] sums of dz xhat
    float* part_b = part_g + entries;                           // [rows][cb] sums of dz
    float* block_sum = part_b + entries;                        // [2][cb] the block's
    float* image_sum = block_sum + 2 * s.cb;                    // [2][cb] the image's
    float* group_mean = image_sum + 2 * s.cb;                   // [gb][2] mean(v), mean(v xhat)
    Pack<T, V>* tile_x = reinterpret_cast<Pack<T, V>*>(smem + ((2 * entries + 4 * s.cb + 2 * gb) * 4 + 15) / 16 * 16);
    Pack<T, V>* tile_d = tile_x + (long long)((p.pixels + s.ranks - 1) / s.ranks) * slots;
    const T* x = reinterpret_cast<const T*>(p.x) + s.image * p.x_image + s.c0;
    const T* dy = reinterpret_cast<const T*>(p.dy) + s.image * p.y_image + s.c0;
    const float* stats = p.stats_in + ((long long)s.image * p.groups + s.c0 / p.per) * 2;

    for (int sp = 0; sp < slots; sp += lanes) {
        const int slot = sp + tid % lanes;
        if (!works || slot >= slots) continue;
        float mean[NS], rstd[NS], gamma[V], beta[V], sg[V], sb[V];
        #pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int g = (slot * V + i * SUB) / p.per;
            mean[i] = stats[2 * g];
            rstd[i] = stats[2 * g + 1];
        }
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            const int ch = s.c0 + slot * V + v;
            gamma[v] = p.gamma ? p.gamma[ch] : 1.f;
            beta[v] = p.beta ? p.beta[ch] : 0.f;
            sg[v] = sb[v] = 0.f;
        }
        for (int px = s.p0 + row0; px < s.p1; px += rows * NORM_BATCH) {
            Pack<T, V> ix[NORM_BATCH], id[NORM_BATCH];
            #pragma unroll
            for (int b = 0; b < NORM_BATCH; ++b) {
                const int q = px + b * rows;
                if (q < s.p1) {
                    ix[b] = load_pack<T, V>(x + q * p.x_pixel + slot * V);
                    id[b] = load_pack<T, V>(dy + q * p.y_pixel + slot * V);
                }
            }
            #pragma unroll
            for (int b = 0; b < NORM_BATCH; ++b) {
                const int q = px + b * rows;
                if (q >= s.p1) continue;
                if (p.resident) {
                    tile_x[(q - s.p0) * slots + slot] = ix[b];
                    tile_d[(q - s.p0) * slots + slot] = id[b];
                }
                float xh[V], z[V];
                #pragma unroll
                for (int v = 0; v < V; ++v) {
                    xh[v] = (to_f32(ix[b].v[v]) - mean[v / SUB]) * rstd[v / SUB];
                    z[v] = fmaf(xh[v], gamma[v], beta[v]);
                }
                act_slopes<V>(p.act, z);
                #pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float dz = to_f32(id[b].v[v]) * z[v];
                    sg[v] = fmaf(dz, xh[v], sg[v]);
                    sb[v] += dz;
                }
            }
        }
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            part_g[row0 * s.cb + slot * V + v] = sg[v];
            part_b[row0 * s.cb + slot * V + v] = sb[v];
        }
    }
    __syncthreads();
    for (int i = tid; i < 2 * s.cb; i += NORM_THREADS) {
        const float* part = i < s.cb ? part_g + i : part_b + (i - s.cb);
        float sum = 0.f;
        #pragma unroll 4
        for (int r = 0; r < rows; ++r) sum += part[r * s.cb];
        block_sum[i] = sum;
    }
    if (s.ranks > 1) cluster.sync(); else __syncthreads();
    for (int i = tid; i < 2 * s.cb; i += NORM_THREADS) {
        float sum = 0.f;
        for (int r = 0; r < s.ranks; ++r) sum += cluster.map_shared_rank(block_sum, r)[i];
        image_sum[i] = sum;
        if (s.rank == 0) {
            const bool g = i < s.cb;
            const int ch = s.c0 + (g ? i : i - s.cb);
            if (p.sums) p.sums[((long long)s.image * p.c + ch) * 2 + (g ? 0 : 1)] = sum;
            else if (g && p.dgamma) p.dgamma[ch] = sum;
            else if (!g && p.dbeta) p.dbeta[ch] = sum;
        }
    }
    __syncthreads();
    for (int g = tid / 32; g < gb; g += NORM_THREADS / 32) {
        float a = 0.f, b = 0.f;
        for (int k = tid & 31; k < p.per; k += 32) {
            const int ch = g * p.per + k;
            const float gamma = p.gamma ? p.gamma[s.c0 + ch] : 1.f;
            a = fmaf(gamma, image_sum[s.cb + ch], a);
            b = fmaf(gamma, image_sum[ch], b);
        }
        a = warp_sum(a);
        b = warp_sum(b);
        const float inv = 1.f / ((float)p.pixels * (float)p.per);
        if ((tid & 31) == 0) { group_mean[2 * g] = a * inv; group_mean[2 * g + 1] = b * inv; }
    }
    __syncthreads();

    T* dx = reinterpret_cast<T*>(p.dx) + s.image * p.dx_image + s.c0;
    for (int sp = 0; sp < slots; sp += lanes) {
        const int slot = sp + tid % lanes;
        if (!works || slot >= slots) continue;
        float mean[NS], rstd[NS], m1[NS], m2[NS], gamma[V], beta[V];
        #pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int g = (slot * V + i * SUB) / p.per;
            mean[i] = stats[2 * g];
            rstd[i] = stats[2 * g + 1];
            m1[i] = group_mean[2 * g];
            m2[i] = group_mean[2 * g + 1];
        }
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            const int ch = s.c0 + slot * V + v;
            gamma[v] = p.gamma ? p.gamma[ch] : 1.f;
            beta[v] = p.beta ? p.beta[ch] : 0.f;
        }
        #pragma unroll 2
        for (int px = s.p0 + row0; px < s.p1; px += rows) {
            const long long at = (long long)(px - s.p0) * slots + slot;
            const Pack<T, V> ix = p.resident ? tile_x[at] : load_pack<T, V>(x + px * p.x_pixel + slot * V);
            const Pack<T, V> id = p.resident ? tile_d[at] : load_pack<T, V>(dy + px * p.y_pixel + slot * V);
            float xh[V], z[V];
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                xh[v] = (to_f32(ix.v[v]) - mean[v / SUB]) * rstd[v / SUB];
                z[v] = fmaf(xh[v], gamma[v], beta[v]);
            }
            act_slopes<V>(p.act, z);
            Pack<T, V> out;
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                const float dv = to_f32(id.v[v]) * z[v] * gamma[v];
                out.v[v] = from_f32<T>(rstd[v / SUB] * (dv - m1[v / SUB] - xh[v] * m2[v / SUB]));
            }
            store_pack<T, V>(dx + px * p.dx_pixel + slot * V, out);
        }
    }
    if (s.ranks > 1) cluster.sync();
}

// The images' channel sums added up, in image order: dgamma and dbeta.
__global__ void norm_sums_kernel(const float* sums, int n, int c, float* dgamma, float* dbeta)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= 2 * c) return;
    float sum = 0.f;
    #pragma unroll 8
    for (int k = 0; k < n; ++k) sum += sums[(long long)k * 2 * c + i];
    float* out = i & 1 ? dbeta : dgamma;
    if (out) out[i >> 1] = sum;
}

struct NormPlan {
    int vec, cb, blocks_c, ranks, resident;
    size_t smem;
};

size_t norm_smem(int cb, int vec, int per, int pixels_per_block, int elem, bool backward, bool resident)
{
    const int slots = cb / vec, lanes = slots < NORM_THREADS ? slots : NORM_THREADS, rows = NORM_THREADS / lanes, gb = cb / per;
    const int sub = per < vec ? per : vec, ns = vec / sub;
    size_t floats;
    if (backward) floats = 2 * (size_t)rows * slots * vec + 4 * (size_t)cb + 2 * gb;
    else floats = 2 * (size_t)(rows * lanes > slots ? rows * lanes : slots) * ns + 4 * (size_t)gb;
    size_t bytes = (floats * 4 + 15) / 16 * 16;
    if (resident) bytes += (size_t)pixels_per_block * cb * elem * (backward ? 2 : 1);
    return bytes;
}

// How a call is cut: channels of a block of channels, blocks of a cluster, and whether a unit stays on chip.
NormPlan norm_plan(const rrm_norm_desc& d, bool backward, int vec)
{
    const int elem = head_elem_bytes(d.dtype), per = d.c / d.groups, base = per > vec ? per : vec, units = d.c / base;
    constexpr size_t ROOM = 227 * 1024, TWO = 113 * 1024;       // dynamic shared memory of one block an SM, and of two
    constexpr int SMS = 148;
    NormPlan best = {};
    // from rows of 128 bytes down to 32, from few blocks a cluster to all: the first cut that fills the SMs and stays on chip
    // with two blocks an SM; failing that the one that leaves most blocks and stays on chip; failing that one read twice
    long long best_score = -1;
    for (int bytes = 128; bytes >= 32; bytes /= 2) {
        const int j = base * elem >= bytes ? 1 : (bytes / (base * elem) < units ? bytes / (base * elem) : units);
        const int cb = base * (j < 1 ? 1 : j), blocks_c = ceil_div(d.c, cb);
        for (int ranks = 1; ranks <= NORM_CLUSTER; ranks *= 2) {
            const int px = ceil_div(d.pixels, ranks);
            const long long blocks = (long long)d.n * blocks_c * ranks;
            const size_t on = norm_smem(cb, vec, per, px, elem, backward, true);
            const bool fits = on <= ROOM, two = on <= TWO;
            if (ranks > 1 && (long long)px * (cb / vec) < NORM_THREADS / 2) continue;       // blocks without work
            const long long score = (fits ? 1000000 : 0) + (two ? 500000 : 0) + (blocks < 2 * SMS ? blocks : 2 * SMS) * 1000 + bytes;
            if (score > best_score) {
                best_score = score;
                best.vec = vec; best.cb = cb; best.blocks_c = blocks_c; best.ranks = ranks; best.resident = fits;
                best.smem = fits ? on : norm_smem(cb, vec, per, px, elem, backward, false);
            }
        }
    }
    return best;
}

int norm_check(rrm_norm_desc& d, bool backward)
{
    if (d.dtype != RRM_F32 && d.dtype != RRM_BF16 && d.dtype != RRM_F16) return RRM_ERR_DTYPE;
    if (!head_act_ok(d.act) || !(d.eps > 0.f) || d.reserved != 0) return RRM_ERR_INVALID_ARG;
    if (d.n < 0 || d.pixels < 0 || d.c < 1 || d.groups < 1 || d.c % d.groups) return RRM_ERR_SHAPE;
    if (d.c > NORM_MAX_C || d.c / d.groups > NORM_MAX_GROUP || d.pixels > NORM_MAX_PIXELS) return RRM_ERR_CAPACITY;
    struct { int64_t *px, *im; bool out; } st[3] = {{&d.x_pixel, &d.x_image, false}, {&d.y_pixel, &d.y_image, !backward}, {&d.dx_pixel, &d.dx_image, true}};
    for (int i = 0; i < (backward ? 3 : 2); ++i) {
        if (*st[i].px == 0) *st[i].px = d.c;
        if (*st[i].im == 0) *st[i].im = *st[i].px * d.pixels;
        if (*st[i].px < 0 || *st[i].im < 0) return RRM_ERR_SHAPE;
        if (st[i].out && d.pixels > 1 && *st[i].px < d.c) return RRM_ERR_SHAPE;
        if (st[i].out && d.n > 1 && d.pixels > 0 && *st[i].im < *st[i].px * (d.pixels - 1) + d.c) return RRM_ERR_SHAPE;
    }
    return RRM_OK;
}

// widest access that all rows allow and that no group boundary cuts unevenly
int norm_vec(const rrm_norm_desc& d, bool backward, const void* const* ptrs, int n_ptrs)
{
    const int elem = head_elem_bytes(d.dtype), per = d.c / d.groups;
    int64_t all = d.c | d.x_pixel | d.x_image | d.y_pixel | d.y_image;
    if (backward) all |= d.dx_pixel | d.dx_image;
    for (int v = 16 / elem; v > 1; v /= 2) {
        if (all % v || (per % v && v % per)) continue;
        bool ok = true;
        for (int i = 0; i < n_ptrs; ++i) ok = ok && !misaligned(ptrs[i], (size_t)v * elem);
        if (ok) return v;
    }
    return 1;
}

template <typename T, int V, int SUB>
cudaError_t norm_launch(const NormParams& p, const NormPlan& o, bool backward, cudaStream_t st)
{
    void (*kernel)(const NormParams) = backward ? norm_backward_kernel<T, V, SUB> : norm_kernel<T, V, SUB>;
    if (o.smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)o.smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((long long)p.n * o.blocks_c * o.ranks));
    cfg.blockDim = dim3(NORM_THREADS);
    cfg.dynamicSmemBytes = o.smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)o.ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = o.ranks > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T>
cudaError_t norm_dispatch16(const NormParams& p, const NormPlan& o, bool backward, cudaStream_t st)
{
    if (o.vec == 8) {
        if (p.per >= 8) return norm_launch<T, 8, 8>(p, o, backward, st);
        if (p.per == 4) return norm_launch<T, 8, 4>(p, o, backward, st);
        if (p.per == 2) return norm_launch<T, 8, 2>(p, o, backward, st);
        return norm_launch<T, 8, 1>(p, o, backward, st);
    }
    if (o.vec >= 4) return p.per >= 4 ? norm_launch<T, 4, 4>(p, o, backward, st) : p.per == 2 ? norm_launch<T, 4, 2>(p, o, backward, st)
                                                                                       : norm_launch<T, 4, 1>(p, o, backward, st);
    if (o.vec == 2) return p.per >= 2 ? norm_launch<T, 2, 2>(p, o, backward, st) : norm_launch<T, 2, 1>(p, o, backward, st);
    return norm_launch<T, 1, 1>(p, o, backward, st);
}

cudaError_t norm_dispatch(int dtype, const NormParams& p, const NormPlan& o, bool backward, cudaStream_t st)
{
    if (dtype == RRM_BF16) return norm_dispatch16<bf16>(p, o, backward, st);
    if (dtype == RRM_F16) return norm_dispatch16<__half>(p, o, backward, st);
    if (o.vec == 4) return p.per >= 4 ? norm_launch<float, 4, 4>(p, o, backward, st) : p.per == 2 ? norm_launch<float, 4, 2>(p, o, backward, st)
                                                                                           : norm_launch<float, 4, 1>(p, o, backward, st);
    if (o.vec == 2) return p.per >= 2 ? norm_launch<float, 2, 2>(p, o, backward, st) : norm_launch<float, 2, 1>(p, o, backward, st);
    return norm_launch<float, 1, 1>(p, o, backward, st);
}

void norm_fill(NormParams& p, const rrm_norm_desc& d, const NormPlan& o)
{
    p.x_pixel = d.x_pixel; p.x_image = d.x_image; p.y_pixel = d.y_pixel; p.y_image = d.y_image;
    p.dx_pixel = d.dx_pixel; p.dx_image = d.dx_image;
    p.n = d.n; p.pixels = d.pixels; p.c = d.c; p.groups = d.groups; p.per = d.c / d.groups; p.cb = o.cb; p.blocks_c = o.blocks_c;
    p.eps = d.eps; p.act = d.act; p.resident = o.resident;
}

}  // namespace
}  // namespace rrm

using namespace rrm;

extern "C" int64_t rrm_group_norm_workspace(const rrm_norm_desc* desc, int backward)
{
    if (!desc) return RRM_ERR_INVALID_ARG;
    rrm_norm_desc d = *desc;
    RRM_TRY(norm_check(d, backward != 0));
    return backward && d.n > 1 ? (int64_t)d.n * d.c * 2 * 4 : 0;
}

extern "C" int rrm_group_norm(const rrm_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y, float* stats,
                              void* workspace, int64_t workspace_bytes, void* stream)
{
    (void)workspace; (void)workspace_bytes;                    // none is needed
    if (!desc) return RRM_ERR_INVALID_ARG;
    rrm_norm_desc d = *desc;
    RRM_TRY(norm_check(d, false));
    if (d.n == 0 || d.pixels == 0) return RRM_OK;
    const int elem = head_elem_bytes(d.dtype);
    if (!x || !y || misaligned(x, elem) || misaligned(y, elem) || misaligned(gamma, 4) || misaligned(beta, 4) || misaligned(stats, 4))
        return RRM_ERR_INVALID_ARG;
    const void* ptrs[2] = {x, y};
    const NormPlan o = norm_plan(d, false, norm_vec(d, false, ptrs, 2));
    if ((long long)d.n * o.blocks_c * o.ranks > INT_MAX) return RRM_ERR_CAPACITY;
    NormParams p = {};
    norm_fill(p, d, o);
    p.x = x; p.gamma = gamma; p.beta = beta; p.y = y; p.stats = stats;
    RRM_CUDA_TRY(norm_dispatch(d.dtype, p, o, false, (cudaStream_t)stream));
    return RRM_OK;
}

extern "C" int rrm_group_norm_backward(const rrm_norm_desc* desc, const void* x, const void* dy, const float* gamma, const float* beta,
                                       const float* stats, void* dx, float* dgamma, float* dbeta, void* workspace,
                                       int64_t workspace_bytes, void* stream)
{
    if (!desc) return RRM_ERR_INVALID_ARG;
    rrm_norm_desc d = *desc;
    RRM_TRY(norm_check(d, true));
    cudaStream_t st = (cudaStream_t)stream;
    if (misaligned(dgamma, 4) || misaligned(dbeta, 4)) return RRM_ERR_INVALID_ARG;
    if (d.n == 0 || d.pixels == 0) {
        if (dgamma) RRM_CUDA_TRY(cudaMemsetAsync(dgamma, 0, (size_t)d.c * 4, st));
        if (dbeta) RRM_CUDA_TRY(cudaMemsetAsync(dbeta, 0, (size_t)d.c * 4, st));
        return RRM_OK;
    }
    const int elem = head_elem_bytes(d.dtype);
    if (!x || !dy || !dx || !stats || misaligned(x, elem) || misaligned(dy, elem) || misaligned(dx, elem) || misaligned(gamma, 4) ||
        misaligned(beta, 4) || misaligned(stats, 4))
        return RRM_ERR_INVALID_ARG;
    const bool sums = d.n > 1 && (dgamma || dbeta);
    if (sums) {
        if (workspace_bytes < (int64_t)d.n * d.c * 2 * 4) return RRM_ERR_CAPACITY;
        if (!workspace || misaligned(workspace, 256)) return RRM_ERR_INVALID_ARG;
    }
    const void* ptrs[3] = {x, dy, dx};
    const NormPlan o = norm_plan(d, true, norm_vec(d, true, ptrs, 3));
    if ((long long)d.n * o.blocks_c * o.ranks > INT_MAX) return RRM_ERR_CAPACITY;
    NormParams p = {};
    norm_fill(p, d, o);
    p.x = x; p.dy = dy; p.gamma = gamma; p.beta = beta; p.stats_in = stats; p.dx = dx;
    p.dgamma = dgamma; p.dbeta = dbeta;
    p.sums = sums ? reinterpret_cast<float*>(workspace) : nullptr;
    RRM_CUDA_TRY(norm_dispatch(d.dtype, p, o, true, st));
    if (sums) {
        norm_sums_kernel<<<ceil_div(2 * d.c, 128), 128, 0, st>>>(p.sums, d.n, d.c, dgamma, dbeta);
        RRM_CUDA_TRY(cudaGetLastError());
    }
    return RRM_OK;
}
