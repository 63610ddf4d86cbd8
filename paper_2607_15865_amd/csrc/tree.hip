// A step of decoding with drafted tokens held as a tree: its plan (positions
// and masks), the acceptance of a path, and the cache rows' ways in and
// together.  All of them move little and are bound by their chains of dependent
// memory and LDS accesses: trees of 8, 64 and 129 nodes take 2.0, 4.0 and 4.8 us to
// plan; 16 sequences of 64 nodes 3.8 to accept, 3.4 to append to a layer of 8 heads of
// 128 (8.4 MB moved, 2.5 TB/s, start and end of a launch in it), and 7.2 to keep in four layers.
#include <algorithm>

#include "kv_attn.h"

namespace {

constexpr int MAXN = W4_TREE_MAX, MAXW = MAXN / 64;

// The node that node i hangs below, or -1.
__device__ __forceinline__ int parent_of(const int32_t* parents, int i) {
    const int p = parents[i];
    return p >= 0 && p < i ? p : -1;
}

// One block per sequence, a thread per node.  Ancestors by pointer doubling: a
// node's set grows by the set of the node that its pointer has reached, and the
// pointer takes that node's; a chain of N is done after log2 N rounds.
template <int W>
__global__ void __launch_bounds__(64 * W) tree_plan_kernel(TreePlanArgs a) {
    __shared__ unsigned long long set[64 * W][W];
    __shared__ int up[64 * W], steps[64 * W];
    const int b = blockIdx.x, i = threadIdx.x, N = a.N;
    const bool on = i < N;
    int p = on ? parent_of(a.parents + (size_t)b * N, i) : -1;
    int n = p >= 0;                                          // steps from node i to its pointer's place, or to the root
    unsigned long long own[W] = {};
#pragma unroll
    for (int w = 0; w < W; w++) own[w] = i / 64 == w ? 1ull << (i % 64) : 0;
    const int ctx = max(a.ctx_lens[b], 0);
    for (;;) {
#pragma unroll
        for (int w = 0; w < W; w++) set[i][w] = own[w];
        up[i] = p;
        steps[i] = n;
        if (!__syncthreads_or(p >= 0)) break;
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < W; w++) own[w] |= set[p][w];
            n += steps[p];
            p = up[p];
        }
        __syncthreads();
    }
    if (!on) return;
    const int words = (N + 63) / 64;
    if (n >= a.window) {                                     // some ancestors are out of the window
        for (int w = 0; w < W; w++)
            for (unsigned long long left = own[w]; left; left &= left - 1) {
                const int bit = __builtin_ctzll(left), s = steps[w * 64 + bit];
                if (n - s >= a.window && ctx + s >= a.sinks) own[w] &= ~(1ull << bit);
            }
    }
    a.pos[(size_t)b * N + i] = ctx + n;
#pragma unroll
    for (int w = 0; w < W; w++)
        if (w < words) a.mask[((size_t)b * N + i) * words + w] = own[w];
}

// One wave per sequence: lane l looks at nodes l, l + 64, .. for a child of the
// path's last node that has the token picked there.  Children come after
// their parents, so the path ends.
__global__ void __launch_bounds__(64) tree_accept_kernel(TreeAcceptArgs a) {
    __shared__ int pick[MAXN];
    const int b = blockIdx.x, lane = threadIdx.x, N = a.N;
    const size_t base = (size_t)b * N;
    int par[MAXW], tok[MAXW];
#pragma unroll
    for (int w = 0; w < MAXW; w++) {
        const int i = w * 64 + lane;
        par[w] = -1;
        if (i < N) {
            par[w] = parent_of(a.parents + base, i);
            tok[w] = a.tokens[base + i];
            pick[i] = a.picks[base + i];
        }
    }
    __syncthreads();
    int cur = 0, len = 0;
    for (;;) {
        if (lane == 0) a.path[base + len] = cur;
        len++;
        const int want = pick[cur];
        int next = -1;
#pragma unroll
        for (int w = MAXW - 1; w >= 0; w--) {
            const unsigned long long fits = __builtin_amdgcn_ballot_w64(par[w] == cur && tok[w] == want);
            if (fits) next = w * 64 + __builtin_ctzll(fits);
        }
        if (next < 0) {
            if (lane == 0) {
                a.n_path[b] = len;
                a.next[b] = want;
            }
            break;
        }
        cur = next;
    }
    for (int t = len + lane; t < N; t += 64) a.path[base + t] = -1;
}

// A thread per 16 bytes of K and of V.
__global__ void __launch_bounds__(256) kv_append_step_kernel(KvSlotArgs a, uint16_t* k, uint16_t* v,
                                                             const uint16_t* k_new, const uint16_t* v_new) {
    const int segs = a.d / 8;
    const long long total = (long long)a.B * a.T * a.nkv * segs;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const int seg = (int)(i % segs);
        const long long row = i / segs;
        const int h = (int)(row % a.nkv), t = (int)(row / a.nkv % a.T), b = (int)(row / a.nkv / a.T);
        const u32x4 kx = reinterpret_cast<const u32x4*>(k_new)[i], vx = reinterpret_cast<const u32x4*>(v_new)[i];
        const long long ctx = a.ctx_lens[b], slot = ctx + t;
        if (ctx < 0 || slot >= a.max_seq) continue;
        const size_t at = (size_t)(b * a.stride_b + h * a.stride_h + slot * a.stride_s) + seg * 8;
        *reinterpret_cast<u32x4*>(k + at) = kx;
        *reinterpret_cast<u32x4*>(v + at) = vx;
    }
}

// A thread moves one 16-byte column of a (cache, sequence, kv head), the path's
// nodes in order.  A path rises (path[t] >= t), so a row that is still to be
// read is never one that was written.
__global__ void __launch_bounds__(256) kv_keep_kernel(KvSlotArgs a, KeepCaches c, const int32_t* path, const int32_t* n_path) {
    constexpr int CB = 8;                                    // rows requested together
    const int segs = a.d / 8, i = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
    if (i >= a.nkv * segs) return;
    const long long ctx = a.ctx_lens[b];
    const int n = min(n_path[b], a.T);
    if (ctx < 0) return;
    uint16_t* const p = c.p[blockIdx.z] + b * a.stride_b + i / segs * a.stride_h + i % segs * 8;
    const int32_t* const from = path + (size_t)b * a.T;
    for (int t0 = 0; t0 < n; t0 += CB) {
        u32x4 x[CB];
        bool go[CB];
#pragma unroll
        for (int j = 0; j < CB; j++) {
            const int t = t0 + j, f = t < n ? from[t] : -1;
            go[j] = f > t && f < a.T && ctx + f < a.max_seq;
            if (go[j]) x[j] = *reinterpret_cast<const u32x4*>(p + (ctx + f) * a.stride_s);
        }
#pragma unroll
        for (int j = 0; j < CB; j++)
            if (go[j]) *reinterpret_cast<u32x4*>(p + (ctx + t0 + j) * a.stride_s) = x[j];
    }
}

}  // namespace

int launch_tree_plan(const TreePlanArgs& a, hipStream_t stream) {
    const int w = (a.N + 63) / 64;
    if (w < 1 || w > MAXW) return -1;
    auto fn = w == 1 ? tree_plan_kernel<1> : w == 2 ? tree_plan_kernel<2> : w == 3 ? tree_plan_kernel<3> : tree_plan_kernel<4>;
    hipLaunchKernelGGL(fn, dim3(a.B), dim3(64 * w), 0, stream, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_tree_accept(const TreeAcceptArgs& a, hipStream_t stream) {
    if (a.N < 1 || a.N > MAXN) return -1;
    hipLaunchKernelGGL(tree_accept_kernel, dim3(a.B), dim3(64), 0, stream, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_append_step(const KvSlotArgs& a, uint16_t* k, uint16_t* v, const uint16_t* k_new, const uint16_t* v_new,
                          hipStream_t stream) {
    const long long total = (long long)a.B * a.T * a.nkv * (a.d / 8);
    const int blocks = (int)std::min<long long>((total + 255) / 256, 8192);
    hipLaunchKernelGGL(kv_append_step_kernel, dim3(blocks), dim3(256), 0, stream, a, k, v, k_new, v_new);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_keep(const KvSlotArgs& a, const KeepCaches& c, int ncaches, const int32_t* path, const int32_t* n_path,
                   hipStream_t stream) {
    if (ncaches < 1 || ncaches > KEEP_CACHES) return -1;
    hipLaunchKernelGGL(kv_keep_kernel, dim3((a.nkv * (a.d / 8) + 255) / 256, a.B, 2 * ncaches), dim3(256), 0, stream, a, c, path,
                       n_path);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int load_tree() { return load_code((const void*)tree_accept_kernel); }
