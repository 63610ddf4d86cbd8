// The 4-bit key/value cache as it is written and read back (layout and
// definition of the codes: kv4.h).
//
// Both kernels are streams: bf16 rows on one side, 5 bits a value on the other.
// A block has one tile of 32 tokens of one (row, kv head): two waves take K (16
// tokens each), two take V.  The lanes of a wave are laid out so that a lane
// holds whole words and, of the parameters, whole groups with one or two lane
// exchanges: for K a lane has the 8 dims of each group that form its words; for
// V, whose words span 8 tokens, it has 8 dims of its token in four dim
// blocks, and the eight lanes of a token block transpose their 8x8 nibbles by three
// exchanges.
#include "kv4.h"

namespace {

// The code of x in a group (lo, s), r = 1 / s roughly: exact.  floor((x - lo) / s)
// by the reciprocal may be one off next to a whole number, where the border
// (k + 1/2) s decides alike from either side.  That border has 16 bits and the
// fma one rounding, so the sign of t - (k + 1/2) s is exact; where it is 0 the part that
// the subtraction t = x - lo lost decides.
__device__ __forceinline__ uint32_t kv4_code(float x, float lo, float s, float r) {
    const float t = x - lo;
    const float kf = __builtin_floorf(t * r);
    const float d = __builtin_fmaf(-(kf + 0.5f), s, t);
    int c = (int)kf;
    if (d > 0.f) {
        c++;
    } else if (d == 0.f) {
        const float z = t - x;                               // (two-sum: x - lo = t + rest)
        const float rest = (x - (t - z)) + (-lo - z);
        c += rest >= 0.f;
    }
    return (uint32_t)(c < 15 ? c : 15);
}

struct Kv4Group {
    float lo, s, r;
    uint16_t lo_bits, s_bits;
    bool bad;
};

// Parameters of a group from its extremes and the largest |x| bits (bf16).  The
// scale is formed in fp64: (hi - lo) / 15 rounded to fp16 is then the nearest.
__device__ __forceinline__ Kv4Group kv4_group(float lo, float hi, uint32_t amax) {
    Kv4Group g;
    g.bad = amax > 0x477Fu;                                  // beyond 65280, the largest bf16 value in fp16
    const f16 s = (f16)(float)(((double)hi - (double)lo) * (1.0 / 15.0));
    g.s = (float)s;
    g.lo = lo;
    g.s_bits = g.bad ? (uint16_t)0x7E00u : __builtin_bit_cast(uint16_t, s);
    g.lo_bits = g.bad ? (uint16_t)0x7E00u : __builtin_bit_cast(uint16_t, (f16)lo);
    g.r = g.s > 0.f ? __builtin_amdgcn_rcpf(g.s) : 0.f;
    return g;
}

// Eight bf16 values as the fp32 values of their fp16 values.
struct Kv4Vals {
    float x[8];
    float lo, hi;
    uint32_t amax;
};
__device__ __forceinline__ Kv4Vals kv4_load8(u32x4 w) {
    Kv4Vals v;
    v.amax = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        v.x[2 * j] = (float)(f16)__uint_as_float(w[j] << 16);
        v.x[2 * j + 1] = (float)(f16)__uint_as_float(w[j] & 0xFFFF0000u);
        v.amax = max(v.amax, max(w[j] & 0x7FFFu, w[j] >> 16 & 0x7FFFu));
    }
    v.lo = v.x[0];
    v.hi = v.x[0];
#pragma unroll
    for (int j = 1; j < 8; j++) {
        v.lo = fminf(v.lo, v.x[j]);
        v.hi = fmaxf(v.hi, v.x[j]);
    }
    return v;
}

__device__ __forceinline__ uint32_t xor_lane(uint32_t v, int m) { return (uint32_t)__shfl_xor((int)v, m, 64); }

// 8x8 nibble transpose over the lanes of an aligned group of eight: nibble j of
// lane i becomes nibble i of lane j.
__device__ __forceinline__ uint32_t nibble_transpose(uint32_t w, int lane) {
    uint32_t p = xor_lane(w, 4);
    w = lane & 4 ? (w & 0xFFFF0000u) | p >> 16 : (w & 0x0000FFFFu) | p << 16;
    p = xor_lane(w, 2);
    w = lane & 2 ? (w & 0xFF00FF00u) | (p >> 8 & 0x00FF00FFu) : (w & 0x00FF00FFu) | (p & 0x00FF00FFu) << 8;
    p = xor_lane(w, 1);
    return lane & 1 ? (w & 0xF0F0F0F0u) | (p >> 4 & 0x0F0F0F0Fu) : (w & 0x0F0F0F0Fu) | (p & 0x0F0F0F0Fu) << 4;
}

// Token (of eight) whose code is nibble n of a V word, and the bit position of element e of a word.
__device__ __forceinline__ int nibble_elem(int n) { return 2 * (n & 3) + (n >> 2); }
__host__ __device__ constexpr int elem_bit(int e) { return 4 * (e / 2) + 16 * (e % 2); }

// What a block works on: tile `tile` of row b, its tokens lo .. hi - 1 (of 32) in the row's run.
struct Kv4Work {
    int b, g, tile, lo, hi;
    int t0;                  // token of the run at the tile's first slot (may be negative)
};
__device__ __forceinline__ bool kv4_work(const Kv4StoreArgs& a, Kv4Work& w) {
    w.b = blockIdx.z;
    w.g = blockIdx.y;
    const int s0 = a.slots_dev ? a.slots_dev[w.b] : a.slots.v[w.b];
    if (s0 < 0 || s0 > a.max_seq - a.T) return false;
    w.tile = s0 / KV4_TILE + blockIdx.x;
    w.t0 = w.tile * KV4_TILE - s0;
    w.lo = max(0, -w.t0);
    w.hi = min(KV4_TILE, a.T - w.t0);
    return w.lo < w.hi;
}

template <int D>
__global__ void __launch_bounds__(256) kv4_append_kernel(Kv4StoreArgs a) {
    constexpr int NS = D / 32;
    Kv4Work w;
    if (!kv4_work(a, w)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long xrow = (long long)w.b * a.x_b + (long long)w.t0 * a.x_t + (long long)w.g * a.x_h;
    const long long base = (long long)w.b * a.stride_b + (long long)w.g * a.stride_h + (long long)w.tile * kv4_tile_bytes(D);
    bool bad = false;
    if (wave < 2) {          // K: lane (token, q4)
        const int q4 = lane & 3, tok = 16 * wave + (lane >> 2);
        const bool on = tok >= w.lo && tok < w.hi;
        u32x4 in[NS];
#pragma unroll
        for (int s = 0; s < NS; s++)
            in[s] = on ? *reinterpret_cast<const u32x4*>(a.k_x + xrow + tok * a.x_t + 32 * s + 8 * q4) : u32x4{0u, 0u, 0u, 0u};
        uint32_t word[NS];
        uint16_t* const par = reinterpret_cast<uint16_t*>(a.k + base + kv4_code_bytes(D));
#pragma unroll
        for (int s = 0; s < NS; s++) {
            Kv4Vals x = kv4_load8(in[s]);
#pragma unroll
            for (int m = 1; m < 4; m *= 2) {
                x.lo = fminf(x.lo, __shfl_xor(x.lo, m, 64));
                x.hi = fmaxf(x.hi, __shfl_xor(x.hi, m, 64));
                x.amax = max(x.amax, xor_lane(x.amax, m));
            }
            const Kv4Group g = kv4_group(x.lo, x.hi, x.amax);
            word[s] = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) word[s] |= kv4_code(x.x[e], g.lo, g.s, g.r) << elem_bit(e);
            if (g.s == 0.f || g.bad) word[s] = 0;
            bad |= g.bad;
            if (on && q4 == s) {
                par[s * 64 + tok] = g.s_bits;
                par[s * 64 + 32 + tok] = g.lo_bits;
            }
        }
        const int t = tok >> 2 & 1, n16 = (tok >> 3) << 2 | (tok & 3);
        uint32_t* const dst = reinterpret_cast<uint32_t*>(a.k + base) + (t * 64 + q4 * 16 + n16) * NS;
        if (on) {
#pragma unroll
            for (int s = 0; s < NS; s++) dst[s] = word[s];
        }
    } else {                 // V: lane (token of a block of 8 in nibble order, dims' upper half of 16, half of D or token block)
        const int j = lane & 7, nhi = lane >> 3 & 1;
        const int hf = NS == 4 ? lane >> 4 & 1 : 0;
        const int blk = NS == 4 ? 2 * (wave - 2) + (lane >> 5) : lane >> 4;    // block of 8 tokens
        if (NS == 2 && wave == 3) return;
        const int tok = 8 * blk + nibble_elem(j);
        const bool on = tok >= w.lo && tok < w.hi;
        u32x4 in[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            in[i] = on ? *reinterpret_cast<const u32x4*>(a.v_x + xrow + tok * a.x_t + 16 * (4 * hf + i) + 8 * nhi)
                       : u32x4{0u, 0u, 0u, 0u};
        u32x4 word;
        uint16_t* const par = reinterpret_cast<uint16_t*>(a.v + base + kv4_code_bytes(D));
#pragma unroll
        for (int p = 0; p < 2; p++) {          // a group: dim blocks 2 p and 2 p + 1, this lane and its neighbour
            const Kv4Vals x0 = kv4_load8(in[2 * p]), x1 = kv4_load8(in[2 * p + 1]);
            float lo = fminf(x0.lo, x1.lo), hi = fmaxf(x0.hi, x1.hi);
            uint32_t amax = max(x0.amax, x1.amax);
            lo = fminf(lo, __shfl_xor(lo, 8, 64));
            hi = fmaxf(hi, __shfl_xor(hi, 8, 64));
            amax = max(amax, xor_lane(amax, 8));
            const Kv4Group g = kv4_group(lo, hi, amax);
            uint32_t w0 = 0, w1 = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                w0 |= kv4_code(x0.x[e], g.lo, g.s, g.r) << (4 * e);
                w1 |= kv4_code(x1.x[e], g.lo, g.s, g.r) << (4 * e);
            }
            if (g.s == 0.f || g.bad) w0 = w1 = 0;
            bad |= g.bad;
            if (on && nhi == 0) {
                par[(2 * hf + p) * 64 + tok] = g.s_bits;
                par[(2 * hf + p) * 64 + 32 + tok] = g.lo_bits;
            }
            word[2 * p] = nibble_transpose(w0, lane);
            word[2 * p + 1] = nibble_transpose(w1, lane);
        }
        // tokens of the block that are written, as nibbles
        uint32_t keep = 0;
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const int tk = 8 * blk + nibble_elem(n);
            if (tk < w.lo || tk >= w.hi) keep |= 0xFu << (4 * n);
        }
        u32x4* const dst = reinterpret_cast<u32x4*>(a.v + base) + (hf * 64 + blk * 16 + 8 * nhi + j);
        if (keep != 0xFFFFFFFFu) {
            if (keep) word = (*dst & keep) | (word & ~keep);
            *dst = word;
        }
    }
    flag_range(a.err, bad);
}

__device__ __forceinline__ uint32_t kv4_pair(uint32_t c0, uint32_t c1, float s, float lo) {
    const float x = __builtin_fmaf((float)c0, s, lo), y = __builtin_fmaf((float)c1, s, lo);
    return (uint32_t)bf16_bits_rne(x) | (uint32_t)bf16_bits_rne(y) << 16;
}

__device__ __forceinline__ float kv4_param(const uint16_t* p) { return (float)__builtin_bit_cast(f16, *p); }

template <int D>
__global__ void __launch_bounds__(256) kv4_read_kernel(Kv4StoreArgs a) {
    constexpr int NS = D / 32;
    Kv4Work w;
    if (!kv4_work(a, w)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long xrow = (long long)w.b * a.x_b + (long long)w.t0 * a.x_t + (long long)w.g * a.x_h;
    const long long base = (long long)w.b * a.stride_b + (long long)w.g * a.stride_h + (long long)w.tile * kv4_tile_bytes(D);
    if (wave < 2) {
        const int q4 = lane & 3, tok = 16 * wave + (lane >> 2);
        if (tok < w.lo || tok >= w.hi) return;
        const int t = tok >> 2 & 1, n16 = (tok >> 3) << 2 | (tok & 3);
        const uint32_t* const src = reinterpret_cast<const uint32_t*>(a.k + base) + (t * 64 + q4 * 16 + n16) * NS;
        const uint16_t* const par = reinterpret_cast<const uint16_t*>(a.k + base + kv4_code_bytes(D));
#pragma unroll
        for (int s = 0; s < NS; s++) {
            const uint32_t c = src[s];
            const float sc = kv4_param(par + s * 64 + tok), lo = kv4_param(par + s * 64 + 32 + tok);
            u32x4 o;
#pragma unroll
            for (int p = 0; p < 4; p++) o[p] = kv4_pair(c >> (4 * p) & 15u, c >> (4 * p + 16) & 15u, sc, lo);
            *reinterpret_cast<u32x4*>(a.k_x + xrow + tok * a.x_t + 32 * s + 8 * q4) = o;
        }
    } else {
        const int j = lane & 7, nhi = lane >> 3 & 1;
        const int hf = NS == 4 ? lane >> 4 & 1 : 0;
        const int blk = NS == 4 ? 2 * (wave - 2) + (lane >> 5) : lane >> 4;
        if (NS == 2 && wave == 3) return;
        const int tok = 8 * blk + nibble_elem(j);
        const bool on = tok >= w.lo && tok < w.hi;
        const uint16_t* const par = reinterpret_cast<const uint16_t*>(a.v + base + kv4_code_bytes(D));
        const u32x4 word = reinterpret_cast<const u32x4*>(a.v + base)[hf * 64 + blk * 16 + 8 * nhi + j];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t c = nibble_transpose(word[i], lane);
            if (!on) continue;
            const int g = 2 * hf + i / 2;
            const float sc = kv4_param(par + g * 64 + tok), lo = kv4_param(par + g * 64 + 32 + tok);
            u32x4 o;
#pragma unroll
            for (int p = 0; p < 4; p++) o[p] = kv4_pair(c >> (8 * p) & 15u, c >> (8 * p + 4) & 15u, sc, lo);
            *reinterpret_cast<u32x4*>(a.v_x + xrow + tok * a.x_t + 16 * (4 * hf + i) + 8 * nhi) = o;
        }
    }
}

// Tiles of the longest run: a run of T slots from slot s0 on has
// (s0 % 32 + T + 31) / 32.
int kv4_run_tiles(const Kv4StoreArgs& a) {
    if (a.slots_dev) return (a.T + 2 * KV4_TILE - 2) / KV4_TILE;
    int n = 1;
    for (int b = 0; b < a.B; b++) {
        const int m = (a.slots.v[b] % KV4_TILE + a.T + KV4_TILE - 1) / KV4_TILE;
        n = m > n ? m : n;
    }
    return n;
}

}  // namespace

int launch_kv4_append(const Kv4StoreArgs& a, hipStream_t stream) {
    const dim3 grid(kv4_run_tiles(a), a.nkv, a.B);
    if (a.d == 128) hipLaunchKernelGGL(kv4_append_kernel<128>, grid, dim3(256), 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL(kv4_append_kernel<64>, grid, dim3(256), 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv4_read(const Kv4StoreArgs& a, hipStream_t stream) {
    const dim3 grid(kv4_run_tiles(a), a.nkv, a.B);
    if (a.d == 128) hipLaunchKernelGGL(kv4_read_kernel<128>, grid, dim3(256), 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL(kv4_read_kernel<64>, grid, dim3(256), 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int load_kv4() { return load_code((const void*)kv4_append_kernel<128>); }
