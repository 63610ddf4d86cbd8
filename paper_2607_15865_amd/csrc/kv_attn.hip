// Grouped-query attention over the bf16 cache with a window, sinks and draft
// trees (kv_attn.h).
#include <algorithm>
#include <climits>

#include "kv_attn.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// A wave per (sequence, query, head), 64 keys at a time: a lane forms the score
// of one key, then sums its D / 64 dims over the keys.
template <int D>
__global__ void __launch_bounds__(64) kv_attn_kernel(KvAttnArgs a) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x, h = blockIdx.x, b = blockIdx.z, r = a.nq / a.nkv;
    const long long i = blockIdx.y;
    const size_t row = (size_t)b * a.N + i;
    const int ctx = min(a.ctx_lens ? a.ctx_lens[b] : a.ctx_base, a.max_ctx);
    uint16_t* const out = a.out + (row * a.nq + h) * D;
    const uint16_t* const k = a.k + b * a.stride_b + h / r * a.stride_h;
    const uint16_t* const v = a.v + b * a.stride_b + h / r * a.stride_h;
    const uint16_t* const q = a.q + (row * a.nq + h) * D;
    const int p = a.tree ? (a.pos ? a.pos[row] : 0) : ctx + (int)i;
    const int low = a.window == INT_MAX ? 0 : max(0, p - (a.window - 1));        // first slot of the window
    const int high = a.tree ? ctx - 1 : p, end = ctx < 0 ? -1 : a.tree ? ctx + a.N - 1 : p;
    float m = -INFINITY, l = 0.f, o[E] = {};
    for (int j0 = 0; j0 <= end; j0 += 64) {
        const int j = j0 + lane;
        bool seen = j <= high && (j >= low || j < a.sinks);
        if (a.tree && j >= ctx && j <= end) seen = a.tree[row * a.words + (j - ctx) / 64] >> (j - ctx) % 64 & 1;
        const float add = seen && a.mask ? a.mask[(size_t)b * a.max_seq + j] : 0.f;
        seen = seen && add != -INFINITY;
        float s = 0.f;
        if (seen)
            for (int e = 0; e < D; e++) s += bf16_bits_to_f32(q[e]) * bf16_bits_to_f32(k[j * a.stride_s + e]);
        s = seen ? s * a.scale + add : -INFINITY;
        const float mn = fmaxf(m, wave_max(s));
        const float mb = mn == -INFINITY ? 0.f : mn;         // (nothing seen so far, or NaN alone)
        const float keep = exp2_hw((m - mb) * LOG2E), w = exp2_hw((s - mb) * LOG2E);
        l = l * keep + wave_sum(w);
        m = mn;
        for (int e = 0; e < E; e++) o[e] *= keep;
        for (unsigned long long left = __builtin_amdgcn_ballot_w64(seen); left; left &= left - 1) {
            const int c = __builtin_ctzll(left);
            for (int e = 0; e < E; e++) o[e] += lane_val(w, c) * bf16_bits_to_f32(v[(j0 + c) * a.stride_s + lane * E + e]);
        }
    }
    for (int e = 0; e < E; e++) out[lane * E + e] = bf16_bits_rne(l == 0.f ? 0.f : o[e] / l);
}

}  // namespace

int launch_kv_attn(const KvAttnArgs& a, hipStream_t stream) {
    auto fn = a.d == 128 ? kv_attn_kernel<128> : kv_attn_kernel<64>;
    for (int n0 = 0; n0 < a.N; n0 += 65535) {
        KvAttnArgs x = a;                                    // (chains of more than 65535 queries: in lots)
        if (n0) {
            x.q += (size_t)n0 * a.nq * a.d;
            x.out += (size_t)n0 * a.nq * a.d;
            x.ctx_base += n0;
            x.max_ctx += n0;
        }
        hipLaunchKernelGGL(fn, dim3(a.nq, std::min(a.N - n0, 65535), a.B), dim3(64), 0, stream, x);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int load_kv_attn() { return load_code((const void*)kv_attn_kernel<128>); }
