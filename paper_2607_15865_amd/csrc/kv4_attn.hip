// Grouped-query attention over the 4-bit key/value cache (layout: kv4.h).
#include "kv4.h"

namespace {

__device__ __forceinline__ float kv4_half(const uint8_t* p) {
    return (float)__builtin_bit_cast(f16, *reinterpret_cast<const uint16_t*>(p));
}

// One block per (row, query head); its four waves take the tiles in turn.
template <int D>
__global__ void __launch_bounds__(256) kv4_attn_kernel(Kv4AttnArgs a) {
    constexpr int NS = D / 32, NV = D / 64;
    __shared__ float qs[D], om[4][D], ml[4][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x, head = blockIdx.y, g = head / (a.nq / a.nkv);
    const int ctx = min(a.ctx_lens ? a.ctx_lens[b] : a.ctx_base + b, a.max_ctx);
    const long long base = (long long)b * a.stride_b + (long long)g * a.stride_h;
    if (tid < D) qs[tid] = bf16_bits_to_f32(a.q[((size_t)b * a.nq + head) * D + tid]);
    __syncthreads();
    const int j = lane & 31, hs = lane >> 5;                 // key of the tile, half of the dims
    const int t = j >> 2 & 1, n16 = (j >> 3) << 2 | (j & 3);
    float m = -INFINITY, l = 0.f, o[NV] = {};
    for (int tile = wave; tile * KV4_TILE <= ctx; tile += 4) {
        const uint8_t* kt = a.k + base + (long long)tile * kv4_tile_bytes(D);
        const uint8_t* vt = a.v + base + (long long)tile * kv4_tile_bytes(D);
        const int key = tile * KV4_TILE + j;
        float sc = 0.f;
#pragma unroll
        for (int s = 0; s < NS; s++) {
            const float ks = kv4_half(kt + kv4_code_bytes(D) + s * 128 + 2 * j);
            const float lo = kv4_half(kt + kv4_code_bytes(D) + s * 128 + 64 + 2 * j);
#pragma unroll
            for (int qq = 0; qq < 2; qq++) {
                const int q4 = 2 * hs + qq;
                const uint32_t w = reinterpret_cast<const uint32_t*>(kt)[(t * 64 + q4 * 16 + n16) * NS + s];
#pragma unroll
                for (int e = 0; e < 8; e++)
                    sc += qs[32 * s + 8 * q4 + e] * __builtin_fmaf((float)(w >> (4 * (e / 2) + 16 * (e % 2)) & 15u), ks, lo);
            }
        }
        sc += __shfl_xor(sc, 32, 64);
        sc *= a.scale;
        bool seen = key <= ctx;
        if (a.mask && seen) {
            const float mk = a.mask[(size_t)b * a.max_seq + key];
            seen = mk != -INFINITY;
            sc += mk;
        }
        sc = seen ? sc : -INFINITY;
        const float mn = fmaxf(m, wave_max(sc));
        const float mb = mn == -INFINITY ? 0.f : mn;
        const float alpha = m == -INFINITY ? 0.f : __expf(m - mb);
        const float p = seen ? __expf(sc - mb) : 0.f;
        l = l * alpha + 0.5f * wave_sum(p);
        m = mn;
#pragma unroll
        for (int i = 0; i < NV; i++) o[i] *= alpha;
        for (int k = 0; k < KV4_TILE; k++) {
            const float pk = __shfl(p, k, 64);
            if (pk == 0.f) continue;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const int dim = lane + 64 * i, db = dim >> 4;
                const uint32_t w = reinterpret_cast<const uint32_t*>(vt)[((db >> 2) * 64 + (k >> 3) * 16 + (dim & 15)) * 4 + (db & 3)];
                const uint8_t* par = vt + kv4_code_bytes(D) + (dim >> 5) * 128 + 2 * k;
                const int e = k & 7;
                o[i] += pk * __builtin_fmaf((float)(w >> (4 * (e / 2) + 16 * (e % 2)) & 15u), kv4_half(par), kv4_half(par + 64));
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV; i++) om[wave][lane + 64 * i] = o[i];
    if (lane == 0) {
        ml[wave][0] = m;
        ml[wave][1] = l;
    }
    __syncthreads();
    if (tid >= D) return;
    float M = -INFINITY, L = 0.f, x = 0.f;
    for (int w = 0; w < 4; w++) M = fmaxf(M, ml[w][0]);
    for (int w = 0; w < 4; w++) {
        const float f = ml[w][0] == -INFINITY ? 0.f : __expf(ml[w][0] - M);
        L += f * ml[w][1];
        x += f * om[w][tid];
    }
    x = L == 0.f ? 0.f : x / L;
    const size_t oi = ((size_t)b * a.nq + head) * D + tid;
    if (a.out_f16) {
        bool bad = false;
        static_cast<f16*>(a.out)[oi] = act_f16(x, bad);
        flag_range(a.err, bad);
    } else {
        static_cast<uint16_t*>(a.out)[oi] = bf16_bits_rne(x);
    }
}

}  // namespace

int launch_kv4_attn(const Kv4AttnArgs& a, hipStream_t stream) {
    const dim3 grid(a.rows, a.nq);
    if (a.d == 128) hipLaunchKernelGGL(kv4_attn_kernel<128>, grid, dim3(256), 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL(kv4_attn_kernel<64>, grid, dim3(256), 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int load_kv4_attn() { return load_code((const void*)kv4_attn_kernel<128>); }
