// The gated recurrence over frames, h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(g), and its backward pass.
//
// A frame maps the state v -> f v + b (b = (1 - f) x), or v -> b after a reset; maps compose, (A2, B2) after (A1, B1) being
// (A2 A1, A2 B1 + B2), so the frames can be cut into pieces whose maps are found side by side.  The pieces: a warp takes L
// frames of 32 * V columns (a column: one feature of one stream) into registers, the warps of a block take neighbouring
// pieces, and the blocks of a cluster neighbouring runs of those; warps meet in shared memory, blocks in each other's.  Each
// then starts from its true state and writes its frames: every input is read once and every output written once, in one
// launch, for sequences up to the frames of one cluster.  Longer ones are cut into chunks of that many frames, and a first
// launch finds the chunks' maps (it reads the inputs once more, mostly from L2), a second one, one thread a column, the
// states between the chunks.
//
// Backward, the gradient c that reaches a frame from behind it goes through the map c -> f (c + dh) (0 after a reset), which
// runs over the frames in reverse and composes the same way; its A is the forward one.  dx = (1 - f) (dh + c) and
// dg = f (1 - f) (h_{t-1} - x) (dh + c).  The states h_{t-1} are computed again from g and x: reading the forward pass's h
// would cost a sixth array of traffic and put its rounding (bf16: 2^-9 of h) into a difference.
//
// What bounds it: memory.  3 arrays forward, 5 backward, some 15 and 40 instructions an element.
#include "rrm_common.cuh"
#include "rrm_head.cuh"
#include <climits>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace rrm {
namespace {

constexpr int SCAN_WARPS = 8;          // warps of a block, neighbouring in time
constexpr int SCAN_CLUSTER = 8;        // blocks of a cluster, neighbouring in time

struct ScanParams {
    const void *g, *x, *dh;
    const float *h0, *dlast;           // carry into the first frame / from behind the last one (chunks > 1: found by the carry kernel)
    const uint8_t* reset;
    const int32_t* lengths;
    void *h, *dg, *dx;
    float *last, *dh0;
    float *aggA, *aggF, *aggB;         // [chunks][columns] maps of the chunks: A, forward B, backward B
    float *carryF, *carryB;            // [chunks][columns] state before a chunk, gradient from behind it
    long long g_frame, g_stream, x_frame, x_stream, h_frame, h_stream, dg_frame, dg_stream, dx_frame, dx_stream;
    int frames, n, d, chunks;
    long long columns;                 // n * d
};

// (f, 1 - f): both from the smaller exponential, so that neither cancels
__device__ __forceinline__ void gate(float g, float& keep, float& take)
{
    const float e = __expf(-fabsf(g)), r = __fdividef(1.f, 1.f + e), s = e * r;
    keep = g >= 0.f ? r : s;
    take = g >= 0.f ? s : r;
}

// carry through a map; A < 0 marks a map that lost the state to a reset (0 * carry would keep an infinity or NaN)
__device__ __forceinline__ float through(float A, float B, float carry) { return A < 0.f ? B : fmaf(A, carry, B); }
__device__ __forceinline__ float both(float A, float A2) { return (A < 0.f || A2 < 0.f) ? -1.f : A * A2; }

// What one thread works on: V columns of one stream from frame t0 on.
template <int V> struct ScanSpot {
    long long col;                     // first column (0 if none: `on` is false)
    int n, d, len;
    bool on;
    __device__ ScanSpot(const ScanParams& p, int column_block)
    {
        col = ((long long)column_block * 32 + threadIdx.x) * V;
        on = col < p.columns;
        if (!on) col = 0;
        n = (int)(col / p.d);
        d = (int)(col - (long long)n * p.d);
        len = p.frames;
        if (p.lengths) len = min(max(p.lengths[n], 0), p.frames);
        if (!on) len = 0;
    }
};

// A map per column of the block, one row of 32 * V floats for each warp
template <int V> struct ScanRows { float v[SCAN_WARPS][V][32]; };

// MAPS: only the chunk's map is wanted (first of three launches); BACK: backward.
template <typename T, int V, int L, bool BACK, bool MAPS>
__global__ void __launch_bounds__(SCAN_WARPS * 32) scan_kernel(const __grid_constant__ ScanParams p)
{
    __shared__ ScanRows<V> rowA, rowF, rowB;
    __shared__ float blockA[V][32], blockF[V][32], blockB[V][32];      // the block's own map, read by the cluster
    __shared__ float carryF[V][32], carryB[V][32];                     // state before the block, gradient from behind it
    const int lane = threadIdx.x, w = threadIdx.y, warps = blockDim.y;
    const cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
    const unsigned run = blockIdx.x / ranks;                           // one cluster's: a chunk of one block of columns
    const int chunk = (int)(run % p.chunks);
    const ScanSpot<V> s(p, (int)(run / p.chunks));
    const long long t0 = (((long long)chunk * ranks + rank) * warps + w) * L;
    const int live = (int)max(0ll, min((long long)L, s.len - t0));

    // ---- the piece's inputs, and its map
    Pack<T, V> g[L], x[L], e[BACK ? L : 1];
    unsigned cut = 0;                                                  // bit j: the state is dropped before frame t0 + j
    #pragma unroll
    for (int j = 0; j < L; ++j) {
        if (j < live) {
            const long long t = t0 + j;
            g[j] = load_pack<T, V>(reinterpret_cast<const T*>(p.g) + t * p.g_frame + s.n * p.g_stream + s.d);
            x[j] = load_pack<T, V>(reinterpret_cast<const T*>(p.x) + t * p.x_frame + s.n * p.x_stream + s.d);
            if (BACK) e[j] = load_pack<T, V>(reinterpret_cast<const T*>(p.dh) + t * p.h_frame + s.n * p.h_stream + s.d);
        }
    }
    if (p.reset) {
        #pragma unroll
        for (int j = 0; j < L; ++j)
            if (j < live && p.reset[(t0 + j) * p.n + s.n]) cut |= 1u << j;
    }
    {
        float A[V], F[V], B[V];
        #pragma unroll
        for (int v = 0; v < V; ++v) { A[v] = 1.f; F[v] = 0.f; B[v] = 0.f; }
        #pragma unroll
        for (int j = 0; j < L; ++j) {
            if (j < live) {
                #pragma unroll
                for (int v = 0; v < V; ++v) {
                    float keep, take;
                    gate(to_f32(g[j].v[v]), keep, take);
                    const float b = take * to_f32(x[j].v[v]);
                    // the backward map frame by frame in forward order: B <- B + A f dh, then A <- A f
                    if (cut >> j & 1u) {
                        F[v] = b;
                        A[v] = -1.f;
                    } else {
                        F[v] = fmaf(keep, F[v], b);
                        if (A[v] >= 0.f) {
                            A[v] *= keep;
                            if (BACK) B[v] = fmaf(A[v], to_f32(e[j].v[v]), B[v]);
                        }
                    }
                }
            }
        }
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            rowA.v[w][v][lane] = A[v];
            rowF.v[w][v][lane] = F[v];
            if (BACK) rowB.v[w][v][lane] = B[v];
        }
    }

    // ---- what comes into the block: the chunk's carry through the maps of the cluster's blocks before (behind) this one
    const bool first = w == 0;
    float inF[V], inB[V];
    if (first && !MAPS) {
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            const float* F = p.chunks > 1 ? p.carryF + chunk * p.columns : p.h0;
            inF[v] = s.on && F ? F[s.col + v] : 0.f;
            if (BACK) {
                const float* B = p.chunks > 1 ? p.carryB + chunk * p.columns : p.dlast;
                inB[v] = s.on && B ? B[s.col + v] : 0.f;
            }
        }
    }
    __syncthreads();
    if (ranks > 1 || MAPS) {
        if (first) {
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                float A = 1.f, F = 0.f, B = 0.f;
                for (int i = 0; i < warps; ++i) {
                    const float a = rowA.v[i][v][lane];
                    F = through(a, rowF.v[i][v][lane], F);
                    if (BACK && A >= 0.f) B = fmaf(A, rowB.v[i][v][lane], B);
                    A = both(A, a);
                }
                blockA[v][lane] = A;
                blockF[v][lane] = F;
                if (BACK) blockB[v][lane] = B;
            }
        }
        if (ranks > 1) cluster.sync();
        if (first && !MAPS) {
            for (int r = 0; r < rank; ++r) {
                const float* a = cluster.map_shared_rank(&blockA[0][0], r);
                const float* f = cluster.map_shared_rank(&blockF[0][0], r);
                #pragma unroll
                for (int v = 0; v < V; ++v) inF[v] = through(a[v * 32 + lane], f[v * 32 + lane], inF[v]);
            }
            if (BACK) {
                for (int r = ranks - 1; r > rank; --r) {
                    const float* a = cluster.map_shared_rank(&blockA[0][0], r);
                    const float* b = cluster.map_shared_rank(&blockB[0][0], r);
                    #pragma unroll
                    for (int v = 0; v < V; ++v) inB[v] = through(a[v * 32 + lane], b[v * 32 + lane], inB[v]);
                }
            }
        }
        if (MAPS && first && rank == 0) {
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                float A = 1.f, F = 0.f, B = 0.f;
                for (int r = 0; r < ranks; ++r) {
                    const float a = cluster.map_shared_rank(&blockA[0][0], r)[v * 32 + lane];
                    F = through(a, cluster.map_shared_rank(&blockF[0][0], r)[v * 32 + lane], F);
                    if (BACK && A >= 0.f) B = fmaf(A, cluster.map_shared_rank(&blockB[0][0], r)[v * 32 + lane], B);
                    A = both(A, a);
                }
                if (s.on) {
                    p.aggA[chunk * p.columns + s.col + v] = A;
                    p.aggF[chunk * p.columns + s.col + v] = F;
                    if (BACK) p.aggB[chunk * p.columns + s.col + v] = B;
                }
            }
        }
    }
    if (!MAPS) {
        if (first) {
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                carryF[v][lane] = inF[v];
                if (BACK) carryB[v][lane] = inB[v];
            }
        }
        __syncthreads();

        // ---- from the piece's true state, frame by frame
        float c[V], before[BACK ? L : 1][V];
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            c[v] = carryF[v][lane];
            for (int i = 0; i < w; ++i) c[v] = through(rowA.v[i][v][lane], rowF.v[i][v][lane], c[v]);
        }
        #pragma unroll
        for (int j = 0; j < L; ++j) {
            if (j < live) {
                Pack<T, V> out;
                #pragma unroll
                for (int v = 0; v < V; ++v) {
                    float keep, take;
                    gate(to_f32(g[j].v[v]), keep, take);
                    const bool drop = cut >> j & 1u;
                    const float b = take * to_f32(x[j].v[v]);
                    if (BACK) before[j][v] = drop ? 0.f : c[v];
                    c[v] = drop ? b : fmaf(keep, c[v], b);
                    out.v[v] = from_f32<T>(c[v]);
                }
                if (!BACK) store_pack<T, V>(reinterpret_cast<T*>(p.h) + (t0 + j) * p.h_frame + s.n * p.h_stream + s.d, out);
            }
        }
        if (!BACK && p.last && s.on && (live > 0 ? t0 + live == s.len : (s.len == 0 && t0 == 0))) {
            #pragma unroll
            for (int v = 0; v < V; ++v) p.last[s.col + v] = c[v];
        }
        if (BACK) {
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                c[v] = carryB[v][lane];
                for (int i = warps - 1; i > w; --i) c[v] = through(rowA.v[i][v][lane], rowB.v[i][v][lane], c[v]);
            }
            #pragma unroll
            for (int j = L - 1; j >= 0; --j) {
                if (j < live) {
                    Pack<T, V> og, ox;
                    #pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float keep, take;
                        gate(to_f32(g[j].v[v]), keep, take);
                        const float grad = c[v] + to_f32(e[j].v[v]);
                        og.v[v] = from_f32<T>(grad * (keep * take) * (before[j][v] - to_f32(x[j].v[v])));
                        ox.v[v] = from_f32<T>(grad * take);
                        c[v] = (cut >> j & 1u) ? 0.f : keep * grad;
                    }
                    store_pack<T, V>(reinterpret_cast<T*>(p.dg) + (t0 + j) * p.dg_frame + s.n * p.dg_stream + s.d, og);
                    store_pack<T, V>(reinterpret_cast<T*>(p.dx) + (t0 + j) * p.dx_frame + s.n * p.dx_stream + s.d, ox);
                }
            }
            if (p.dh0 && s.on && t0 == 0) {
                #pragma unroll
                for (int v = 0; v < V; ++v) p.dh0[s.col + v] = c[v];
            }
        }
    }
    if (ranks > 1) cluster.sync();                                     // no block leaves while another may read its maps
}

// The states before the chunks, and the gradients from behind them.
template <bool BACK>
__global__ void scan_carry_kernel(const __grid_constant__ ScanParams p)
{
    const long long col = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (col >= p.columns) return;
    float c = p.h0 ? p.h0[col] : 0.f;
    #pragma unroll 8
    for (int k = 0; k < p.chunks; ++k) {
        p.carryF[k * p.columns + col] = c;
        c = through(p.aggA[k * p.columns + col], p.aggF[k * p.columns + col], c);
    }
    if (BACK) {
        c = p.dlast ? p.dlast[col] : 0.f;
        #pragma unroll 8
        for (int k = p.chunks - 1; k >= 0; --k) {
            p.carryB[k * p.columns + col] = c;
            c = through(p.aggA[k * p.columns + col], p.aggB[k * p.columns + col], c);
        }
    }
}

struct ScanPlan {
    int vec, piece, warps, ranks, chunks;
    int64_t workspace;
};

int scan_plan(const rrm_scan_desc& d, bool backward, int vec, ScanPlan& o)
{
    o.vec = vec;
    o.piece = vec == 1 ? 16 : 8;
    const int pieces = ceil_div(d.frames > 0 ? d.frames : 1, o.piece);
    o.warps = pieces < SCAN_WARPS ? pieces : SCAN_WARPS;
    o.ranks = ceil_div(pieces, SCAN_WARPS);
    if (o.ranks > 4) o.ranks = SCAN_CLUSTER;
    else if (o.ranks == 3) o.ranks = 4;
    o.chunks = ceil_div(pieces, o.warps * o.ranks);
    if (((long long)d.n * d.d / (32 * vec) + 1) * o.chunks * o.ranks > INT_MAX) return RRM_ERR_CAPACITY;
    o.workspace = o.chunks > 1 ? (int64_t)o.chunks * d.n * d.d * 4 * (backward ? 5 : 3) : 0;
    return RRM_OK;
}

bool dense_or(int64_t& stride, int64_t dense)
{
    if (stride == 0) stride = dense;
    return stride >= 0;
}

// checks the sizes and fills in the dense strides
int scan_check(rrm_scan_desc& d, bool backward)
{
    if (d.dtype != RRM_F32 && d.dtype != RRM_BF16 && d.dtype != RRM_F16) return RRM_ERR_DTYPE;
    if (d.frames < 0 || d.n < 1 || d.d < 1) return RRM_ERR_SHAPE;
    if ((long long)d.n * d.d > INT_MAX || (long long)d.frames * d.n > INT_MAX) return RRM_ERR_CAPACITY;
    const int64_t row = d.d;
    struct { int64_t *f, *s; bool used, out; } st[5] = {
        {&d.g_frame, &d.g_stream, true, false}, {&d.x_frame, &d.x_stream, true, false}, {&d.h_frame, &d.h_stream, true, !backward},
        {&d.dg_frame, &d.dg_stream, backward, true}, {&d.dx_frame, &d.dx_stream, backward, true}};
    for (auto& e : st) {
        if (!e.used) continue;
        if (!dense_or(*e.s, row) || !dense_or(*e.f, *e.s * d.n)) return RRM_ERR_SHAPE;
        // rows of an output must not overlap: the streams of a frame lie inside it, or the frames of a stream inside the stream
        if (e.out && !((*e.s >= row && *e.f >= *e.s * (d.n - 1) + row) || (*e.f >= row && *e.s >= *e.f * (d.frames - 1) + row)) &&
            !(d.frames <= 1 && *e.s >= row) && !(d.n == 1 && *e.f >= row))
            return RRM_ERR_SHAPE;
    }
    return RRM_OK;
}

// columns per access: all rows of all arrays begin on a multiple of it
int scan_vec(const rrm_scan_desc& d, bool backward, const void* const* ptrs, int n_ptrs)
{
    const int v = 4, es = head_elem_bytes(d.dtype);
    int64_t all = d.d | d.g_frame | d.g_stream | d.x_frame | d.x_stream | d.h_frame | d.h_stream;
    if (backward) all |= d.dg_frame | d.dg_stream | d.dx_frame | d.dx_stream;
    for (int i = 0; i < n_ptrs; ++i) if (misaligned(ptrs[i], (size_t)v * es)) return 1;
    return all % v == 0 ? v : 1;
}

template <typename T, int V, int L, bool BACK>
cudaError_t scan_launch(const ScanParams& p, const ScanPlan& o, cudaStream_t st)
{
    const long long blocks = (p.columns + 32 * V - 1) / (32 * V) * o.chunks * o.ranks;   // scan_plan has seen that they fit
    const dim3 grid((unsigned)blocks), block(32, o.warps);
    auto run = [&](void (*kernel)(const ScanParams)) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = grid; cfg.blockDim = block; cfg.stream = st;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)o.ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = o.ranks > 1 ? 1 : 0;
        return cudaLaunchKernelEx(&cfg, kernel, p);
    };
    if (o.chunks > 1) {
        cudaError_t e = run(scan_kernel<T, V, L, BACK, true>);
        if (e != cudaSuccess) return e;
        scan_carry_kernel<BACK><<<(unsigned)((p.columns + 127) / 128), 128, 0, st>>>(p);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return run(scan_kernel<T, V, L, BACK, false>);
}

template <bool BACK>
cudaError_t scan_dispatch(int dtype, const ScanParams& p, const ScanPlan& o, cudaStream_t st)
{
    if (dtype == RRM_F32) return o.vec == 4 ? scan_launch<float, 4, 8, BACK>(p, o, st) : scan_launch<float, 1, 16, BACK>(p, o, st);
    if (dtype == RRM_BF16) return o.vec == 4 ? scan_launch<bf16, 4, 8, BACK>(p, o, st) : scan_launch<bf16, 1, 16, BACK>(p, o, st);
    return o.vec == 4 ? scan_launch<__half, 4, 8, BACK>(p, o, st) : scan_launch<__half, 1, 16, BACK>(p, o, st);
}

void scan_fill(ScanParams& p, const rrm_scan_desc& d, const ScanPlan& o, bool backward, void* workspace)
{
    p.frames = d.frames; p.n = d.n; p.d = d.d; p.chunks = o.chunks;
    p.columns = (long long)d.n * d.d;
    p.g_frame = d.g_frame; p.g_stream = d.g_stream; p.x_frame = d.x_frame; p.x_stream = d.x_stream;
    p.h_frame = d.h_frame; p.h_stream = d.h_stream;
    p.dg_frame = d.dg_frame; p.dg_stream = d.dg_stream; p.dx_frame = d.dx_frame; p.dx_stream = d.dx_stream;
    if (o.chunks > 1) {
        float* ws = reinterpret_cast<float*>(workspace);
        const long long part = o.chunks * p.columns;
        p.aggA = ws; p.aggF = ws + part; p.carryF = ws + 2 * part;
        if (backward) { p.aggB = ws + 3 * part; p.carryB = ws + 4 * part; }
    }
}

int scan_workspace_ok(const ScanPlan& o, const void* workspace, int64_t bytes)
{
    if (o.workspace == 0) return RRM_OK;
    if (bytes < o.workspace) return RRM_ERR_CAPACITY;
    if (!workspace || misaligned(workspace, 256)) return RRM_ERR_INVALID_ARG;
    return RRM_OK;
}

}  // namespace
}  // namespace rrm

using namespace rrm;

extern "C" int64_t rrm_gated_scan_workspace(const rrm_scan_desc* desc, int backward)
{
    if (!desc) return RRM_ERR_INVALID_ARG;
    rrm_scan_desc d = *desc;
    RRM_TRY(scan_check(d, backward != 0));
    ScanPlan o;
    RRM_TRY(scan_plan(d, backward != 0, 4, o));                // the wider access has the shorter chunks, so this covers both
    return o.workspace;
}

extern "C" int rrm_gated_scan(const rrm_scan_desc* desc, const void* g, const void* x, const float* h0, const uint8_t* reset,
                              const int32_t* lengths, void* h, float* last, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!desc) return RRM_ERR_INVALID_ARG;
    rrm_scan_desc d = *desc;
    RRM_TRY(scan_check(d, false));
    const int es = head_elem_bytes(d.dtype);
    if (d.frames > 0 && (!g || !x || !h)) return RRM_ERR_INVALID_ARG;
    if (misaligned(g, es) || misaligned(x, es) || misaligned(h, es) || misaligned(h0, 4) || misaligned(last, 4) || misaligned(lengths, 4))
        return RRM_ERR_INVALID_ARG;
    const void* ptrs[3] = {g, x, h};
    ScanPlan o;
    RRM_TRY(scan_plan(d, false, scan_vec(d, false, ptrs, 3), o));
    RRM_TRY(scan_workspace_ok(o, workspace, workspace_bytes));
    ScanParams p = {};
    scan_fill(p, d, o, false, workspace);
    p.g = g; p.x = x; p.h0 = h0; p.reset = reset; p.lengths = lengths; p.h = h; p.last = last;
    RRM_CUDA_TRY(scan_dispatch<false>(d.dtype, p, o, (cudaStream_t)stream));
    return RRM_OK;
}

extern "C" int rrm_gated_scan_backward(const rrm_scan_desc* desc, const void* g, const void* x, const float* h0,
                                       const uint8_t* reset, const int32_t* lengths, const void* dh, const float* dlast, void* dg,
                                       void* dx, float* dh0, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!desc) return RRM_ERR_INVALID_ARG;
    rrm_scan_desc d = *desc;
    RRM_TRY(scan_check(d, true));
    const int es = head_elem_bytes(d.dtype);
    if (d.frames > 0 && (!g || !x || !dh || !dg || !dx)) return RRM_ERR_INVALID_ARG;
    if (misaligned(g, es) || misaligned(x, es) || misaligned(dh, es) || misaligned(dg, es) || misaligned(dx, es) || misaligned(h0, 4) ||
        misaligned(dlast, 4) || misaligned(dh0, 4) || misaligned(lengths, 4))
        return RRM_ERR_INVALID_ARG;
    const void* ptrs[5] = {g, x, dh, dg, dx};
    ScanPlan o;
    RRM_TRY(scan_plan(d, true, scan_vec(d, true, ptrs, 5), o));
    RRM_TRY(scan_workspace_ok(o, workspace, workspace_bytes));
    ScanParams p = {};
    scan_fill(p, d, o, true, workspace);
    p.g = g; p.x = x; p.h0 = h0; p.reset = reset; p.lengths = lengths; p.dh = dh; p.dlast = dlast;
    p.dg = dg; p.dx = dx; p.dh0 = dh0;
    RRM_CUDA_TRY(scan_dispatch<true>(d.dtype, p, o, (cudaStream_t)stream));
    return RRM_OK;
}
