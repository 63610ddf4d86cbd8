// The 4-bit key/value cache as it is written and read back (layout and
// definition of the codes: kv4.h).
//
// Both kernels are streams: bf16 rows on one side, 5 bits a value on the other.
// A lane has one group (32 dims of one token): the group's extremes, scale and
// codes need no other lane.  A wave has 64 / NS tokens of K or of V.  In memory the NS
// lanes of a token take 16 bytes of each group side by side, and a transpose among them
// gives each its group (a lane that reads its own 64 bytes costs the largest read
// 11 us of 47).  V, whose words span 8 tokens: the eight lanes of a token block
// transpose their 8x8 nibbles, one word of dims each for one word of tokens, in
// three exchanges; a run that ends inside a block replaces its nibbles alone.
//
// Measured, 2 sequences of 16384 tokens, 8 heads of 128 (134 MB of bf16, 42 of cache): append 39 us in a row of
// appends, 35 without the codes' arithmetic (of about 15 operations a value), and 47 in turn with reads; read 38 and 31.
// One token of two heads of 64: 4.3 and 2.8, a kernel's start, chain of loads, exchanges and stores, and end.
#include <type_traits>

#include "kv4.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, false);
}

// The value of lane ^ M.
template <int M>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
    static_assert(M == 1 || M == 2 || M == 4 || M == 8 || M == 16, "");
    if constexpr (M == 1) return dpp_u32<0xB1>(x);
    if constexpr (M == 2) return dpp_u32<0x4E>(x);
    if constexpr (M == 4) return dpp_u32<0x1B>(dpp_u32<0x141>(x));           // mirrored in 8, then in 4
    if constexpr (M == 8) return dpp_u32<0x128>(x);                          // rotated by 8 in 16
    return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401F);            // (lane ^ 16)
}

// 8x8 nibble transpose over the eight lanes that differ in the bits M, 2 M, 4 M of
// their number: nibble j of the lane with bits i becomes nibble i of the lane with bits j.
template <int M>
__device__ __forceinline__ uint32_t nibble_transpose(uint32_t w, int lane) {
    uint32_t p = lane_xor<4 * M>(w);
    w = lane & 4 * M ? (w & 0xFFFF0000u) | p >> 16 : (w & 0x0000FFFFu) | p << 16;
    p = lane_xor<2 * M>(w);
    w = lane & 2 * M ? (w & 0xFF00FF00u) | (p >> 8 & 0x00FF00FFu) : (w & 0x00FF00FFu) | (p & 0x00FF00FFu) << 8;
    p = lane_xor<M>(w);
    return lane & M ? (w & 0xF0F0F0F0u) | (p >> 4 & 0x0F0F0F0Fu) : (w & 0x0F0F0F0Fu) | (p & 0x0F0F0F0Fu) << 4;
}

// Transpose of x[i] among the NS lanes of a token: afterwards (NS 4) x[i] of lane s is
// what x[s] of lane i was; (NS 2) what x[2 s + i / 2] of lane i % 2 was.  For NS 4 it is its own
// inverse; for NS 2 `back` undoes it.
template <int NS, typename T>
__device__ __forceinline__ void group_transpose(T (&x)[4], int lane, bool back = false) {
    auto swap2 = [&](T& p, T& q, auto m) __attribute__((always_inline)) {     // 2x2: off-diagonal elements change lanes
        constexpr int M = decltype(m)::value;
        const bool odd = lane & M;
        constexpr int W = sizeof(T) / 4;
        uint32_t pw[W], qw[W];
        __builtin_memcpy(pw, &p, sizeof(T));
        __builtin_memcpy(qw, &q, sizeof(T));
#pragma unroll
        for (int k = 0; k < W; k++) {
            const uint32_t a = lane_xor<M>(qw[k]), b = lane_xor<M>(pw[k]);
            pw[k] = odd ? a : pw[k];
            qw[k] = odd ? qw[k] : b;
        }
        __builtin_memcpy(&p, pw, sizeof(T));
        __builtin_memcpy(&q, qw, sizeof(T));
    };
    if constexpr (NS == 4) {
        swap2(x[0], x[1], std::integral_constant<int, 1>{});
        swap2(x[2], x[3], std::integral_constant<int, 1>{});
        swap2(x[0], x[2], std::integral_constant<int, 2>{});
        swap2(x[1], x[3], std::integral_constant<int, 2>{});
    } else {
        T t;
        if (back) { t = x[1]; x[1] = x[2]; x[2] = t; }
        swap2(x[0], x[2], std::integral_constant<int, 1>{});
        swap2(x[1], x[3], std::integral_constant<int, 1>{});
        if (!back) { t = x[1]; x[1] = x[2]; x[2] = t; }
    }
}

// Dims of the 16 bytes that a token's lane s takes as its i-th: (NS 4) chunk s of group i; (NS 2) chunk 2 (i % 2) + s of
// group i / 2.
template <int NS>
__device__ __forceinline__ int chunk_dim(int s, int i) { return NS == 4 ? 32 * i + 8 * s : 32 * (i >> 1) + 16 * (i & 1) + 8 * s; }

// Token (of eight) whose code is nibble n of a V word.
__device__ __forceinline__ int nibble_elem(int n) { return 2 * (n & 3) + (n >> 2); }

// A group: its values as fp16 pairs, its parameters, and what the codes need.
struct Kv4Group {
    f16x2 x[16];
    float lo, s, r, zb, half;    // r = 1 / s roughly, zb = - lo r, half = lo + s / 2
    uint32_t params;             // scale bits | offset bits << 16
    bool bad, rare;
};

__device__ __forceinline__ void kv4_group(Kv4Group& g, const u32x4 (&in)[4]) {
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const uint32_t w = in[i / 4][i % 4];
        g.x[i] = __builtin_convertvector(f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)}, f16x2);
    }
    f16x2 mn = g.x[0], mx = g.x[0], nan = g.x[0] * (f16)0.f;
#pragma unroll
    for (int i = 1; i < 16; i++) {
        mn = __builtin_elementwise_min(mn, g.x[i]);
        mx = __builtin_elementwise_max(mx, g.x[i]);
        nan = __builtin_elementwise_fma(g.x[i], f16x2{(f16)0.f, (f16)0.f}, nan);     // (NaN of an infinity or a NaN)
    }
    g.bad = !((float)nan[0] + (float)nan[1] == 0.f);
    const f16 lo = mn[0] < mn[1] ? mn[0] : mn[1], hi = mx[0] > mx[1] ? mx[0] : mx[1];
    // (in fp64 the quotient rounded to fp16 is the nearest)
    const f16 s = (f16)(float)(((double)(float)hi - (double)(float)lo) * (1.0 / 15.0));
    g.lo = g.bad ? 0.f : (float)lo;
    g.s = g.bad ? 0.f : (float)s;
    g.r = g.s > 0.f ? __builtin_amdgcn_rcpf(g.s) : 0.f;
    g.zb = -g.lo * g.r;
    g.half = __builtin_fmaf(0.5f, g.s, g.lo);
    // The borders lo + (k + 1/2) s have to be fp32 numbers: multiples of half the scale's last place (2^-12 s at least) and
    // of the offset's (2^-11 |lo|), of magnitude up to the values'.  And a scale rounded among fp16's subnormals can ask for
    // codes above 15.
    const float top = fmaxf(__builtin_fabsf(g.lo), __builtin_fabsf((float)hi));
    g.rare = !g.bad && (top > 2048.f * g.s || (g.lo != 0.f && __builtin_fabsf(g.lo) < 0x1p-11f * top) || g.s < 0x1p-14f);
    g.params = g.bad ? 0x7E007E00u : (uint32_t)__builtin_bit_cast(uint16_t, s) | (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16;
}

// The code of x, exact for every group.  floor((x - lo) / s) by the reciprocal may be one off
// next to a whole number, where the border (k + 1/2) s decides alike from either
// side.  That border has 16 bits and the fma one rounding, so the sign of t - (k + 1/2) s is
// exact; where it is 0 the part that the subtraction t = x - lo lost decides.
__device__ __forceinline__ float kv4_code_rare(float x, float lo, float s) {
    if (s == 0.f) return 0.f;
    const float t = x - lo, r = __builtin_amdgcn_rcpf(s);
    const float kf = __builtin_floorf(t * r), d = __builtin_fmaf(-(kf + 0.5f), s, t);
    const float z = t - x;                                   // (two-sum: x - lo = t + rest)
    const float rest = (x - (t - z)) + (-lo - z);
    return fminf(kf + (d > 0.f || (d == 0.f && rest >= 0.f) ? 1.f : 0.f), 15.f);
}

// Codes of values 8 w .. + 7 of the group, value e at nibble e.  The same idea as kv4_code_rare with the border as a value:
// k = floor of about (x - lo) / s, and k + 1 from lo + (k + 1/2) s on.
__device__ __forceinline__ uint32_t kv4_word(const Kv4Group& g, int w) {
    float c[8];
    float one = 1.f;                                         // (opaque: x - .. widens x in the same operation)
    asm("" : "+v"(one));
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const f16 x = g.x[4 * w + e / 2][e % 2];
        const float k = __builtin_floorf(__builtin_fmaf((float)x, g.r, g.zb));
        const float d = __builtin_fmaf((float)x, one, -__builtin_fmaf(k, g.s, g.half));
        c[e] = k + __builtin_amdgcn_fmed3f(__builtin_fmaf(d, 0x1p40f, 1.f), 0.f, 1.f);        // (1 if d >= 0, else 0)
    }
    if (g.rare) {
#pragma unroll
        for (int e = 0; e < 8; e++) c[e] = kv4_code_rare((float)g.x[4 * w + e / 2][e % 2], g.lo, g.s);
    }
    // four codes are summed up as one number below 2^16
    const float a0 = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[3], 16.f, c[2]), 16.f, c[1]), 16.f, c[0]);
    const float a1 = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[7], 16.f, c[6]), 16.f, c[5]), 16.f, c[4]);
    return g.bad ? 0u : (uint32_t)a0 | (uint32_t)a1 << 16;
}

// A wave's work: K or V of 64 / NS tokens (from tok0 of a tile) of a (row, kv head).
struct Kv4Work {
    int b, g, tile, lo, hi;      // tokens lo .. hi - 1 of the tile's 32 are in the row's run
    int t0;                      // token of the run at the tile's first slot (may be negative)
    int tok0;
    bool v;
};
template <int D>
__device__ __forceinline__ bool kv4_work(const Kv4StoreArgs& a, Kv4Work& w) {
    constexpr int WPT = D / 64;                              // waves per tile of K (or V)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), item = wave / (2 * WPT);
    w.b = blockIdx.z;
    w.g = blockIdx.y;
    w.v = wave / WPT % 2;
    w.tok0 = wave % WPT * (KV4_TILE / WPT);
    int s0;
    if (a.slots_dev) {
        s0 = a.slots_dev[w.b];
        asm volatile("" : "+v"(s0));                         // (two loads, not one from a chosen address)
    } else {
        s0 = a.slots.v[w.b];
    }
    s0 = __builtin_amdgcn_readfirstlane(s0);
    if (s0 < 0 || s0 > a.max_seq - a.T) return false;
    w.tile = s0 / KV4_TILE + blockIdx.x * (2 / WPT) + item;
    w.t0 = w.tile * KV4_TILE - s0;
    w.lo = max(0, -w.t0);
    w.hi = min(KV4_TILE, a.T - w.t0);
    return max(w.lo, w.tok0) < min(w.hi, w.tok0 + KV4_TILE / WPT);
}

// Lane (token, group lane % NS): tokens in order for K, for V in nibble order in blocks of 8.
template <int D>
struct Kv4Lane {
    static constexpr int NS = D / 32;
    int tok, s, j, blk;
    __device__ __forceinline__ Kv4Lane(const Kv4Work& w) {
        const int lane = threadIdx.x & 63;
        s = lane % NS;
        j = lane / NS % 8;
        blk = w.tok0 / 8 + lane / (8 * NS);
        tok = w.v ? 8 * blk + nibble_elem(j) : w.tok0 + lane / NS;
    }
    // K: first word of lane (n16, q4) of the token
    __device__ __forceinline__ int k_word(int q4) const {
        return ((tok >> 2 & 1) * 64 + q4 * 16 + ((tok >> 3) << 2 | (tok & 3))) * NS;
    }
    // V: words of dim blocks 2 s, 2 s + 1 (two in a row) of lane (j, q4 = blk), and 8 lanes on
    __device__ __forceinline__ int v_word() const { return ((s >> 1) * 64 + blk * 16 + j) * 4 + 2 * (s & 1); }
};

template <int D>
__global__ void __launch_bounds__(256) kv4_append_kernel(Kv4StoreArgs a) {
    constexpr int NS = D / 32;
    Kv4Work w;
    if (!kv4_work<D>(a, w)) return;
    const int lane = threadIdx.x & 63;
    const Kv4Lane<D> at(w);
    const bool on = at.tok >= w.lo && at.tok < w.hi;
    const uint16_t* const x = (w.v ? a.v_x : a.k_x) + ((long long)w.b * a.x_b + (long long)w.g * a.x_h +
                                                       (long long)(w.t0 + at.tok) * a.x_t);
    uint8_t* const tile = (w.v ? a.v : a.k) + ((long long)w.b * a.stride_b + (long long)w.g * a.stride_h +
                                               (long long)w.tile * kv4_tile_bytes(D));
    u32x4 in[4];
#pragma unroll
    for (int i = 0; i < 4; i++) in[i] = on ? *reinterpret_cast<const u32x4*>(x + chunk_dim<NS>(at.s, i)) : u32x4{0u, 0u, 0u, 0u};
    // V: nibbles (tokens) of this block's words that stay as they are
    uint32_t keep = 0;
    u32x2 old[2] = {u32x2{0u, 0u}, u32x2{0u, 0u}};
    uint32_t* const vw = reinterpret_cast<uint32_t*>(tile) + at.v_word();
    if (w.v && (w.lo > w.tok0 || w.hi < w.tok0 + 64 / NS)) {
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const int tk = 8 * at.blk + nibble_elem(n);
            if (tk < w.lo || tk >= w.hi) keep |= 0xFu << (4 * n);
        }
        if (keep != 0 && keep != 0xFFFFFFFFu) {
            old[0] = *reinterpret_cast<const u32x2*>(vw);
            old[1] = *reinterpret_cast<const u32x2*>(vw + 32);
        }
    }
    group_transpose<NS>(in, lane);
    Kv4Group g;
    kv4_group(g, in);
    if (on) {
        uint16_t* const par = reinterpret_cast<uint16_t*>(tile + kv4_code_bytes(D)) + at.s * 64 + at.tok;
        par[0] = (uint16_t)g.params;
        par[32] = (uint16_t)(g.params >> 16);
    }
    if (!w.v) {              // K words hold values 0, 2, 4, 6 in their lower half: values 8 i .. + 7 in that order
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const f16x2 p0 = g.x[i], p1 = g.x[i + 1], p2 = g.x[i + 2], p3 = g.x[i + 3];
            g.x[i] = f16x2{p0[0], p1[0]};
            g.x[i + 1] = f16x2{p2[0], p3[0]};
            g.x[i + 2] = f16x2{p0[1], p1[1]};
            g.x[i + 3] = f16x2{p2[1], p3[1]};
        }
    }
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; i++) c[i] = kv4_word(g, i);
    if (w.v) {
#pragma unroll
        for (int i = 0; i < 4; i++) c[i] = nibble_transpose<NS>(c[i], lane);           // dim 32 s + 8 i + j
        if (keep != 0xFFFFFFFFu) {
            *reinterpret_cast<u32x2*>(vw) = u32x2{(old[0][0] & keep) | (c[0] & ~keep), (old[0][1] & keep) | (c[2] & ~keep)};
            *reinterpret_cast<u32x2*>(vw + 32) = u32x2{(old[1][0] & keep) | (c[1] & ~keep), (old[1][1] & keep) | (c[3] & ~keep)};
        }
    } else {
        uint32_t* const kw = reinterpret_cast<uint32_t*>(tile);        // (word i: q4 = i of group s)
        if constexpr (NS == 4) {
            group_transpose<4>(c, lane);                                // group i of q4 = s
            if (on) *reinterpret_cast<u32x4*>(kw + at.k_word(at.s)) = u32x4{c[0], c[1], c[2], c[3]};
        } else {
            group_transpose<2>(c, lane);                                // group i % 2 of q4 = 2 s + i / 2
            if (on) {
                *reinterpret_cast<u32x2*>(kw + at.k_word(2 * at.s)) = u32x2{c[0], c[1]};
                *reinterpret_cast<u32x2*>(kw + at.k_word(2 * at.s + 1)) = u32x2{c[2], c[3]};
            }
        }
    }
    flag_range(a.err, g.bad);
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
    if (!kv4_work<D>(a, w)) return;
    const int lane = threadIdx.x & 63;
    const Kv4Lane<D> at(w);
    const bool on = at.tok >= w.lo && at.tok < w.hi;
    uint16_t* const x = (w.v ? a.v_x : a.k_x) + ((long long)w.b * a.x_b + (long long)w.g * a.x_h +
                                                 (long long)(w.t0 + at.tok) * a.x_t);
    const uint8_t* const tile = (w.v ? a.v : a.k) + ((long long)w.b * a.stride_b + (long long)w.g * a.stride_h +
                                                     (long long)w.tile * kv4_tile_bytes(D));
    const uint16_t* const par = reinterpret_cast<const uint16_t*>(tile + kv4_code_bytes(D)) + at.s * 64 + at.tok;
    const float s = kv4_param(par), lo = kv4_param(par + 32);
    uint32_t c[4];                                           // natural nibble order (K: the cache's order)
    if (w.v) {
        const uint32_t* const vw = reinterpret_cast<const uint32_t*>(tile) + at.v_word();
        const u32x2 p = *reinterpret_cast<const u32x2*>(vw), q = *reinterpret_cast<const u32x2*>(vw + 32);
        c[0] = nibble_transpose<NS>(p[0], lane);
        c[1] = nibble_transpose<NS>(q[0], lane);
        c[2] = nibble_transpose<NS>(p[1], lane);
        c[3] = nibble_transpose<NS>(q[1], lane);
    } else {
        const uint32_t* const kw = reinterpret_cast<const uint32_t*>(tile);
        if constexpr (NS == 4) {
            const u32x4 p = *reinterpret_cast<const u32x4*>(kw + at.k_word(at.s));
#pragma unroll
            for (int i = 0; i < 4; i++) c[i] = p[i];
        } else {
            const u32x2 p = *reinterpret_cast<const u32x2*>(kw + at.k_word(2 * at.s));
            const u32x2 q = *reinterpret_cast<const u32x2*>(kw + at.k_word(2 * at.s + 1));
            c[0] = p[0]; c[1] = p[1]; c[2] = q[0]; c[3] = q[1];
        }
        group_transpose<NS>(c, lane, true);
    }
    const int d0 = w.v ? 8 : 4, d1 = w.v ? 4 : 16;           // bits from pair to pair, between a pair's codes
    u32x4 o[4];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int p = 0; p < 4; p++) o[i][p] = kv4_pair(c[i] >> (d0 * p) & 15u, c[i] >> (d0 * p + d1) & 15u, s, lo);
    group_transpose<NS>(o, lane, true);
    if (on) {
#pragma unroll
        for (int i = 0; i < 4; i++) *reinterpret_cast<u32x4*>(x + chunk_dim<NS>(at.s, i)) = o[i];
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
    const int per = a.d == 64 ? 2 : 1;                       // tiles per block
    const dim3 grid((kv4_run_tiles(a) + per - 1) / per, a.nkv, a.B);
    if (a.d == 128) hipLaunchKernelGGL(kv4_append_kernel<128>, grid, dim3(256), 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL(kv4_append_kernel<64>, grid, dim3(256), 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv4_read(const Kv4StoreArgs& a, hipStream_t stream) {
    const int per = a.d == 64 ? 2 : 1;                       // tiles per block
    const dim3 grid((kv4_run_tiles(a) + per - 1) / per, a.nkv, a.B);
    if (a.d == 128) hipLaunchKernelGGL(kv4_read_kernel<128>, grid, dim3(256), 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL(kv4_read_kernel<64>, grid, dim3(256), 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int load_kv4() { return load_code((const void*)kv4_append_kernel<128>); }
