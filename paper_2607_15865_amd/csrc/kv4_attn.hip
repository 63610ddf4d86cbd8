// Grouped-query attention over the 4-bit key/value cache (layout: kv4.h).
//
// Decode: one query per sequence, the work split over keys.  The codes go to the
// matrix cores as they are: a 4-bit code masked out of its word is a subnormal
// fp16 number, c 2^-24 (or 16 c 2^-24 for the nibbles in bits 4..7, whose
// partners are divided by 16), which the 16x16x32 fp16 MFMA takes exactly.  The
// group's scale and offset are applied outside the products, in fp32:
//     q . K_j = sum_g (s_jg sum_{d in g} q_d c_jd + lo_jg sum_{d in g} q_d),
//     out_d   = sum_j (p_j s_jg) c_jd + sum_j p_j lo_jg        (d in g).
// For that the 16 columns of the score tile stand for (head, group) pairs: column
// (h, g) holds head h's query in group g's dims and zeros elsewhere, so one chain
// of MFMAs leaves the sums of every group apart in one accumulator.  A row of
// the output tile is such a pair too: P'_(h,g) j = p_hj s_jg, of which the dims
// of group g are used.  The matrix cores do 4 times (d = 128) the needed work
// and are idle most of the time all the same; the vector units, which have
// little to spare at 5 bits a value, unpack a code in 5/8 of an operation and
// scale per score and weight instead of per value.
#include <algorithm>

#include "kv4.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;

// ---------------------------------------------------------------- decode

constexpr int DW = 8;            // waves per block
constexpr long long kMaxShares = 1024;   // beyond one per (row, kv head), of a launch
constexpr int kCus = 256;
constexpr int MAXR = 8;          // query heads per kv head

// Eight codes of a word as fp16 multiples of 2^-24: elements 0, 1, 4, 5 are
// c 2^-24, elements 2, 3, 6, 7 are 16 c 2^-24.
__device__ __forceinline__ f16x8 code_frag(uint32_t w) {
    const uint32_t w8 = w >> 8;
    const u32x4 r{w & 0x000F000Fu, w & 0x00F000F0u, w8 & 0x000F000Fu, w8 & 0x00F000F0u};
    return __builtin_bit_cast(f16x8, r);
}

// Over lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max_quarters(float v) {
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float sum_quarters(float v) {
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// h x + y, h widened in the operation.
__device__ __forceinline__ float mix_fma(f16 h, float x, float y) { return __builtin_fmaf((float)h, x, y); }

template <int N>                 // lanes xor 1 .. N / 2, N = 2 or 4
__device__ __forceinline__ float group_max(float v) {
    v = fmaxf(v, dpp_mov<0xB1>(v));
    if (N == 4) v = fmaxf(v, dpp_mov<0x4E>(v));
    return v;
}
template <int N>
__device__ __forceinline__ float group_sum(float v) {
    v += dpp_mov<0xB1>(v);
    if (N == 4) v += dpp_mov<0x4E>(v);
    return v;
}

// Output elements off, off + 1: sums x, y over the sum of the weights.
__device__ __forceinline__ void put_pair(const Kv4AttnArgs& a, size_t off, float x, float y, float lt, bool& bad) {
    const float u = lt == 0.f ? 0.f : x / lt, v = lt == 0.f ? 0.f : y / lt;              // (NaN stays)
    uint32_t w;
    if (a.out_f16) {
        const f16 h0 = act_f16(u, bad), h1 = act_f16(v, bad);
        w = (uint32_t)__builtin_bit_cast(uint16_t, h0) | (uint32_t)__builtin_bit_cast(uint16_t, h1) << 16;
    } else {
        w = (uint32_t)bf16_bits_rne(u) | (uint32_t)bf16_bits_rne(v) << 16;
    }
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + off) = w;
}

// One block: a share (a.per tiles) of one (row, kv head), all r query heads of the
// group.  Wave w of 8 takes tiles w, w + 8, .. of the share on its own; the next
// tile's K is requested when this one's scores are formed and its V when its
// output is, into the same registers, so that two blocks fit a CU (CT 1; 16 rows of up to 32768 keys of 8 heads of
// 128, 480 to 500 MB, take 96 to 100 us, 5.0 TB/s; the device reads at 5.9 at most).  The first
// tile's requests do not wait for the context length: a share's place is fixed by
// the longest context, and blocks past a row's own end leave.  CT column tiles of 16 /
// NS heads.  Softmax: the maximum of a head moves only when a score passes it by
// more than 2 (all lanes of the wave then agree on the new one), so weights stay
// below e^2.  Weights times scales are a pair of fp16 numbers, hi + lo: s c and lo of a
// value near 0 cancel, so P' rounded once would leave 2^-12 of the group's range.
// They are multiplied by ef = 2^10 so that small ones keep their digits; if one
// passes the fp16 range after all (a scale above 8), ef drops to 1 for the rest of
// the share: e^2 times the largest scale (8704: bf16 values that fp16 has
// end at 65280) is 64314.
template <int D, int CT>
__global__ void __launch_bounds__(64 * DW, CT == 1 ? 4 : 2) kv4_decode_kernel(Kv4AttnArgs a) {
    constexpr int NS = D / 32, NDB = D / 16, HC = 16 / NS, PS = 8 / NS;
    constexpr int TB = kv4_tile_bytes(D), CB = kv4_code_bytes(D);
    extern __shared__ __attribute__((aligned(16))) float ored[];          // [DW][r][D]
    __shared__ float gst[DW][MAXR][2], glo[DW][MAXR][NS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hk = blockIdx.x, part = blockIdx.y, b = blockIdx.z, r = a.r;
    const int n16 = lane & 15, q4 = lane >> 4, g = n16 % NS;
    const long long base = (long long)b * a.stride_b + (long long)hk * a.stride_h;
    const uint8_t* const kb = a.k + base;
    const uint8_t* const vb = a.v + base;
    const float* const mrow = a.mask ? a.mask + (size_t)b * a.max_seq : nullptr;
    // key of score i (NS 4: tile i; NS 2: tile i / 2) of this lane, of 32
    auto score_key = [&](int i) { return NS == 4 ? 8 * q4 + 4 * i + g : 8 * q4 + 4 * (i >> 1) + 2 * (i & 1) + g; };

    uint32_t kc[2][NS];              // words of score tiles 0 and 1
    u32x4 vc[NS / 2];                // words of dim blocks 0 .. 3 (4 .. 7)
    f16x8 ks, kl, vs, vl;            // scale and offset of group g, tokens 8 q4 .. + 7
    float mk[PS];                    // mask of this lane's scores
    const int paro = CB + g * 128 + q4 * 16;
    auto load_k = [&](int tile) __attribute__((always_inline)) {
        const uint8_t* kt = kb + (long long)tile * TB;
#pragma unroll
        for (int t = 0; t < 2; t++) {
            if constexpr (NS == 4) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(kt + (t * 64 + lane) * 16);
#pragma unroll
                for (int s = 0; s < NS; s++) kc[t][s] = w[s];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2*>(kt + (t * 64 + lane) * 8);
                kc[t][0] = w[0];
                kc[t][1] = w[1];
            }
        }
        ks = *reinterpret_cast<const f16x8*>(kt + paro);
        kl = *reinterpret_cast<const f16x8*>(kt + paro + 64);
        if (mrow) {
#pragma unroll
            for (int i = 0; i < PS; i++) mk[i] = mrow[min(tile * KV4_TILE + score_key(i), a.max_ctx)];
        }
    };
    auto load_v = [&](int tile) __attribute__((always_inline)) {
        const uint8_t* vt = vb + (long long)tile * TB;
#pragma unroll
        for (int i = 0; i < NS / 2; i++) vc[i] = *reinterpret_cast<const u32x4*>(vt + (i * 64 + lane) * 16);
        vs = *reinterpret_cast<const f16x8*>(vt + paro);
        vl = *reinterpret_cast<const f16x8*>(vt + paro + 64);
    };
    const int tile0 = part * a.per;
    int tile = tile0 + wave;
    int ctx = a.ctx_lens ? a.ctx_lens[b] : a.ctx_base + b;
    if (tile * KV4_TILE <= a.max_ctx) {
        load_k(tile);
        load_v(tile);
    }

    // ---- queries: head ct HC + n16 / NS, dims 32 g + 8 q4 .. + 7, times 2^qe (the head's largest becomes 2^14 ..)
    f16x8 qf[CT][NS];
    float qs[CT], f2[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        const int h = ct * HC + n16 / NS;
        u32x4 w{0u, 0u, 0u, 0u};
        if (h < r) w = *reinterpret_cast<const u32x4*>(a.q + ((size_t)b * a.nq + hk * r + h) * D + 32 * g + 8 * q4);
        float x[8], mx = 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            mx = fmaxf(mx, fmaxf(__builtin_fabsf(x[2 * i]), __builtin_fabsf(x[2 * i + 1])));
        }
        mx = max_quarters(group_max<NS>(mx));
        // exponent field of the largest; 2^qe and 2^-qe are both normal numbers
        const int qe = max(-113, min(126, 141 - (int)(__float_as_uint(mx) >> 23)));
        const float up = __uint_as_float((uint32_t)(127 + qe) << 23);
        f2[ct] = __uint_as_float((uint32_t)(127 - qe) << 23);
        f16x8 fr;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float v = x[e] * up;
            sum += v;
            fr[e] = (f16)(e & 2 ? v * 0.0625f : v);
        }
        qs[ct] = sum_quarters(sum) * 0x1p-24f;
#pragma unroll
        for (int s = 0; s < NS; s++) qf[ct][s] = g == s ? fr : f16x8{};
    }
    const float f1 = a.scale * 0x1p24f;

    ctx = min(ctx, a.max_ctx);
    const int ntiles = (ctx + KV4_TILE) / KV4_TILE;             // of ctx + 1 keys
    const int n = max(1, (ntiles + a.per - 1) / a.per);         // shares of this row
    const size_t slot = (((size_t)b * a.nkv + hk) * a.nsplit + part) * r;      // of the share's state
    float2* const pst = reinterpret_cast<float2*>(a.part + (size_t)a.rows * a.nq * a.nsplit * D) + slot;
    if (part >= n) {
        if (tid < r) pst[tid] = float2{-INFINITY, 0.f};
        return;
    }
    const int tile1 = min(tile0 + a.per, ntiles);

    f32x4 o[CT][NDB];
    float m[CT], l[CT], olo[CT][2];  // olo: sums of the offsets, of keys whose weights are held as they are, and / 16
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
#pragma unroll
        for (int i = 0; i < NDB; i++) o[ct][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m[ct] = -INFINITY;
        l[ct] = olo[ct][0] = olo[ct][1] = 0.f;
    }
    float ef = 1024.f;

    for (; tile < tile1; tile += DW) {
        f32x4 acc[CT][2];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) acc[ct][0] = acc[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; s++)
#pragma unroll
            for (int t = 0; t < 2; t++) {
                const f16x8 kf = code_frag(kc[t][s]);
#pragma unroll
                for (int ct = 0; ct < CT; ct++) acc[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[ct][s], acc[ct][t], 0, 0, 0);
            }
        const bool special = mrow || (tile + 1) * KV4_TILE > ctx + 1;       // some key may be hidden
        float p[CT][PS];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) {
#pragma unroll
            for (int t = 0; t < 2; t++) {
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; j++)
                    v[j] = mix_fma(ks[4 * t + j], acc[ct][t][j], mix_fma(kl[4 * t + j], qs[ct], 0.f));
                // sums over the groups (lanes g): lane g keeps the key 4 t + g (NS 2: keys 4 t + g, 4 t + 2 + g)
                const bool b0 = lane & 1;
                const float r0 = (b0 ? v[1] : v[0]) + dpp_mov<0xB1>(b0 ? v[0] : v[1]);
                const float r1 = (b0 ? v[3] : v[2]) + dpp_mov<0xB1>(b0 ? v[2] : v[3]);
                if constexpr (NS == 4) {
                    const bool b1 = lane & 2;
                    p[ct][t] = ((b1 ? r1 : r0) + dpp_mov<0x4E>(b1 ? r0 : r1)) * f1 * f2[ct];
                } else {
                    p[ct][2 * t] = r0 * f1 * f2[ct];
                    p[ct][2 * t + 1] = r1 * f1 * f2[ct];
                }
            }
            if (special) {
                int lim = ctx;
                asm volatile("" : "+s"(lim));                   // (a branch, not selects on every tile)
#pragma unroll
                for (int i = 0; i < PS; i++) {
                    bool seen = tile * KV4_TILE + score_key(i) <= lim;
                    if (mrow) {
                        seen = seen && mk[i] != -INFINITY;
                        p[ct][i] += mk[i];
                    }
                    p[ct][i] = seen ? p[ct][i] : -INFINITY;
                }
            }
        }
        if (tile + DW < tile1) load_k(tile + DW);
        f16x8 pf[CT], pl[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) {
            float mx = p[ct][0];
#pragma unroll
            for (int i = 1; i < PS; i++) mx = fmaxf(mx, p[ct][i]);
            if (__builtin_amdgcn_ballot_w64(mx > m[ct] + 2.f) != 0) {
                const float mn = fmaxf(m[ct], max_quarters(group_max<NS>(mx)));
                const float alpha = exp2_hw((m[ct] - (mn == -INFINITY ? 0.f : mn)) * LOG2E);
                l[ct] *= alpha;
                olo[ct][0] *= alpha;
                olo[ct][1] *= alpha;
                m[ct] = mn;
                // register j of lane (., q4) is row 4 q4 + j, of head (4 q4 + j) / NS
                const float a0 = __shfl(alpha, 4 * q4, 64), a1 = NS == 4 ? a0 : __shfl(alpha, 4 * q4 + 2, 64);
#pragma unroll
                for (int i = 0; i < NDB; i++) {
                    o[ct][i][0] *= a0;
                    o[ct][i][1] *= a0;
                    o[ct][i][2] *= a1;
                    o[ct][i][3] *= a1;
                }
            }
            const float mb = m[ct] == -INFINITY ? 0.f : m[ct];
            // weights, times ef and, of keys whose codes come times 16 (element & 2), / 16
            float u[PS];
#pragma unroll
            for (int i = 0; i < PS; i++) {
                const float w = exp2_hw((p[ct][i] - mb) * LOG2E);
                l[ct] += w;
                u[i] = w * ((NS == 4 ? g & 2 : i & 1) ? ef * 0.0625f : ef);
            }
            // P'_(h,g) of keys 8 q4 + e: weights from the lanes that hold them
            float w[8];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                if constexpr (NS == 4) {
                    w[4 * t + 0] = dpp_mov<0x00>(u[t]);
                    w[4 * t + 1] = dpp_mov<0x55>(u[t]);
                    w[4 * t + 2] = dpp_mov<0xAA>(u[t]);
                    w[4 * t + 3] = dpp_mov<0xFF>(u[t]);
                } else {
                    w[4 * t + 0] = dpp_mov<0xA0>(u[2 * t]);
                    w[4 * t + 1] = dpp_mov<0xF5>(u[2 * t]);
                    w[4 * t + 2] = dpp_mov<0xA0>(u[2 * t + 1]);
                    w[4 * t + 3] = dpp_mov<0xF5>(u[2 * t + 1]);
                }
            }
            f16x8 cs = vs, cl = vl;
            if (special) {                                      // (hidden keys may hold NaN)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    float z = w[e];
                    asm volatile("" : "+v"(z));
                    cs[e] = z == 0.f ? (f16)0.f : cs[e];
                    cl[e] = z == 0.f ? (f16)0.f : cl[e];
                }
            }
            float ps[8];
#pragma unroll
            for (int e = 0; e < 8; e++) ps[e] = mix_fma(cs[e], w[e], 0.f);
            const float pmax = fmaxf(fmaxf(fmaxf(ps[0], ps[1]), fmaxf(ps[2], ps[3])), fmaxf(fmaxf(ps[4], ps[5]), fmaxf(ps[6], ps[7])));
            if (__builtin_amdgcn_ballot_w64(pmax > 65504.f) != 0) {
                float down = 0x1p-10f;
                asm volatile("" : "+v"(down));
                ef = 1.f;
#pragma unroll
                for (int c2 = 0; c2 < CT; c2++) {
                    olo[c2][0] *= down;
                    olo[c2][1] *= down;
#pragma unroll
                    for (int i = 0; i < NDB; i++)
#pragma unroll
                        for (int e = 0; e < 4; e++) o[c2][i][e] *= down;
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    ps[e] *= down;
                    w[e] *= down;
                    if (ct == 1) {
                        pf[0][e] = (f16)((float)pf[0][e] * down);
                        pl[0][e] = (f16)((float)pl[0][e] * down);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                olo[ct][e >> 1 & 1] = mix_fma(cl[e], w[e], olo[ct][e >> 1 & 1]);
                olo[ct][e >> 1 & 1] = mix_fma(cl[e + 1], w[e + 1], olo[ct][e >> 1 & 1]);
                const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(ps[e], ps[e + 1]));
                const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(ps[e] - (float)hi[0], ps[e + 1] - (float)hi[1]));
                pf[ct][e] = hi[0]; pf[ct][e + 1] = hi[1];
                pl[ct][e] = lo[0]; pl[ct][e + 1] = lo[1];
            }
        }
#pragma unroll
        for (int i = 0; i < NDB; i++) {
            const f16x8 vf = code_frag(vc[i / 4][i % 4]);
#pragma unroll
            for (int ct = 0; ct < CT; ct++) {
                o[ct][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pf[ct], vf, o[ct][i], 0, 0, 0);
                o[ct][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl[ct], vf, o[ct][i], 0, 0, 0);
            }
        }
        if (tile + DW < tile1) load_v(tile + DW);
    }

    // ---- the waves' states meet in LDS
    const float eo = ef == 1.f ? 1.f : 0x1p-10f;                // 1 / ef
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        l[ct] = sum_quarters(group_sum<NS>(l[ct]));
        const float lo = sum_quarters(olo[ct][0] + 16.f * olo[ct][1]) * eo;
        const int h = ct * HC + n16 / NS;
        if (q4 == 0 && h < r) {
            glo[wave][h][g] = lo;
            if (g == 0) {
                gst[wave][h][0] = m[ct];
                gst[wave][h][1] = l[ct];
            }
        }
#pragma unroll
        for (int i = 0; i < NDB; i++)
#pragma unroll
            for (int j = i / 2; j < 4; j += NS) {               // the rows of dim block i's group
                const int ho = ct * HC + (4 * q4 + j) / NS;
                if (ho < r) ored[(wave * r + ho) * D + 16 * i + n16] = o[ct][i][j] * (0x1p24f * eo);
            }
    }
    __syncthreads();
    // one share: the output; more: its state, [row, kv head][share][r heads][D] outputs, then [..][r] (max, sum)
    float* const po = a.part + slot * D;
    bool bad = false;
    for (int idx = tid; idx < r * (D / 2); idx += 64 * DW) {
        const int i = idx / (D / 2), d = 2 * (idx % (D / 2));
        float M = -INFINITY;
        for (int w = 0; w < DW; w++) M = fmaxf(M, gst[w][i][0]);
        float x = 0.f, y = 0.f, lt = 0.f;
        for (int w = 0; w < DW; w++) {
            const float sc = gst[w][i][0] == -INFINITY ? 0.f : exp2_hw((gst[w][i][0] - M) * LOG2E);
            const float2 v = *reinterpret_cast<const float2*>(ored + (w * r + i) * D + d);
            x += sc * (v.x + glo[w][i][d / 32]);
            y += sc * (v.y + glo[w][i][d / 32]);
            lt += sc * gst[w][i][1];
        }
        if (a.nsplit == 1) {
            put_pair(a, ((size_t)b * a.nq + hk * r) * D + 2 * idx, x, y, lt, bad);
        } else {
            *reinterpret_cast<float2*>(po + 2 * idx) = float2{x, y};
            if (d == 0) pst[i] = float2{M, lt};
        }
    }
    flag_range(a.err, bad);
}

// Merges the shares of a row and head: one block each, wave w takes shares w, w +
// 4, ..; their order does not depend on timing.
template <int D>
__global__ void __launch_bounds__(256) kv4_decode_merge_kernel(Kv4AttnArgs a) {
    constexpr int CB = 4, E = D / 64;        // shares of a wave requested together, dims of a lane
    __shared__ float sm[4][2 + E][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hk = blockIdx.x, i = blockIdx.y, b = blockIdx.z, n = a.nsplit;
    const size_t slot = ((size_t)b * a.nkv + hk) * n * a.r + i;
    const float* const po = a.part + slot * D + E * lane;
    const float2* const pst = reinterpret_cast<const float2*>(a.part + (size_t)a.rows * a.nq * n * D) + slot;
    float M = -INFINITY, L = 0.f, acc[E] = {};
    for (int c0 = wave; c0 < n; c0 += 4 * CB) {
        float2 s[CB];
        float v[CB][E];
#pragma unroll
        for (int c = 0; c < CB; c++) {
            const size_t o = (size_t)min(c0 + 4 * c, n - 1) * a.r;
            s[c] = pst[o];
#pragma unroll
            for (int e = 0; e < E; e++) v[c][e] = po[o * D + e];
        }
        float Mn = M;
#pragma unroll
        for (int c = 0; c < CB; c++) {
            // a share past the row's end has (-inf, 0) and no output
            const bool none = c0 + 4 * c >= n || (s[c].x == -INFINITY && s[c].y == 0.f);
            if (none) s[c] = float2{-INFINITY, 0.f};
#pragma unroll
            for (int e = 0; e < E; e++) v[c][e] = none ? 0.f : v[c][e];
            Mn = fmaxf(Mn, s[c].x);
        }
        const float Mb = Mn == -INFINITY ? 0.f : Mn, keep = exp2_hw((M - Mb) * LOG2E);
        L *= keep;
#pragma unroll
        for (int e = 0; e < E; e++) acc[e] *= keep;
#pragma unroll
        for (int c = 0; c < CB; c++) {
            const float w = exp2_hw((s[c].x - Mb) * LOG2E);
            L += w * s[c].y;
#pragma unroll
            for (int e = 0; e < E; e++) acc[e] += w * v[c][e];
        }
        M = Mn;
    }
    sm[wave][0][lane] = M;
    sm[wave][1][lane] = L;
#pragma unroll
    for (int e = 0; e < E; e++) sm[wave][2 + e][lane] = acc[e];
    __syncthreads();
    if (wave) return;
    const float Mn = fmaxf(fmaxf(sm[0][0][lane], sm[1][0][lane]), fmaxf(sm[2][0][lane], sm[3][0][lane]));
    const float Mb = Mn == -INFINITY ? 0.f : Mn;
    L = 0.f;
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const float f = exp2_hw((sm[w][0][lane] - Mb) * LOG2E);
        L += f * sm[w][1][lane];
#pragma unroll
        for (int e = 0; e < E; e++) acc[e] += f * sm[w][2 + e][lane];
    }
    bool bad = false;
    const size_t off = ((size_t)b * a.nq + hk * a.r + i) * D + E * lane;
    if constexpr (E == 2) {
        put_pair(a, off, acc[0], acc[1], L, bad);
    } else {
        const float next = __shfl_down(acc[0], 1, 64);
        if (!(lane & 1)) put_pair(a, off, acc[0], next, L, bad);
    }
    flag_range(a.err, bad);
}

// ---------------------------------------------------------------- prefill

// Rows are the (query, head) pairs of one kv head's group, r per query in
// order, so a block's 256 rows are full whatever r is; wave w has rows 32 w ..
// + 31.  Keys come in stages of 64: every thread unpacks two words of K and two
// of V (d = 64: one) to fp16, s c + lo rounded once, and writes them to LDS in the
// order of the 32x32x16 MFMAs' operand registers, 16 bytes a lane, where all
// eight waves read them.  Scores are formed transposed, S^T = K Q^T, with the
// keys of a tile in an order (bits 2 and 3 of the row index swapped) that leaves the weights
// in the operand layout of P^T; a V word holds 8 tokens of one dim and is, once
// unpacked, an operand of O^T = V^T P^T as it stands.  A lane owns one row: the
// online softmax needs a lane exchange only when a maximum moves, which it does when a
// score passes it by more than 8 (log2 units; weights stay below 2^8, in fp16).
// Keys, values and weights rounded to fp16 (2^-11 each) are what lets the matrix units take a stage in one product each;
// the rounding of the output to bf16 (2^-8) hides them: against 64 bits the outputs are off by 0.00170 in the mean, and
// 0.00166 where those are fp32.
//
// Work is dealt out in one of two ways (kv4_prefill_plan).  In pieces (a.pf_chunk):
// every row tile's stages are cut into as many equal parts as it has runs of pf_chunk, one
// block each, the longest tiles first.  Or in a line: the stages of all row tiles of
// all kv heads follow each other and the blocks cut them into equal runs, so that
// long work ends everywhere at once.  A row tile with more than one part leaves their states in
// the workspace, and a second launch merges them in order.
//
// Measured, 2011 queries of 28 heads of 4 behind 14001 tokens: 475 to 540 us by
// the card's clock; 522, 0.83 PFLOP/s, where a library product of two 8192^2 fp16
// matrices ran at 1.13.  With all CUs at work a stage takes 2.4 us (d = 64: 2.1).  In a build without the exponentials 449, without the expansion
// 430, with neither 426, without the first product 428: the halves overlap, and
// the clock at the power limit bounds what is left.
constexpr int PF_W = 8;                      // waves per block
constexpr int PF_ROWS = 32 * PF_W;
constexpr int PF_KST = 64;                   // keys per stage

__host__ __device__ inline int pf_stages(int q, int R, int r, int hist) {     // of row tile q
    const int last = (q + 1) * PF_ROWS < R ? (q + 1) * PF_ROWS - 1 : R - 1;
    return (hist + last / r) / PF_KST + 1;
}

// A kv head's row tiles in the order in which work is dealt out, with their shares of it: parts, last tile first
// (a.pf_chunk), or stages.
__device__ __forceinline__ int pf_tile(const Kv4AttnArgs& a, int i, int nqt) { return a.pf_chunk ? nqt - 1 - i : i; }
__device__ __forceinline__ int pf_weight(const Kv4AttnArgs& a, int i, int nqt, int R, int r) {
    const int st = pf_stages(pf_tile(a, i, nqt), R, r, a.ctx_base);
    return a.pf_chunk ? (st + a.pf_chunk - 1) / a.pf_chunk : st;
}

// x, the same in all lanes, in scalar registers.
__device__ __forceinline__ long long scalar(long long x) {
    return (long long)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                       (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// The entry i that has unit u of a kv head (u below the head's sum), and its first; whole waves call it.
__device__ __forceinline__ void pf_find(const Kv4AttnArgs& a, int R, int r, long long u, int& i, long long& first) {
    const int lane = threadIdx.x & 63, nqt = (R + PF_ROWS - 1) / PF_ROWS;
    first = 0;
    for (int i0 = 0;; i0 += 64) {
        int x = i0 + lane < nqt ? pf_weight(a, i0 + lane, nqt, R, r) : 0;
        const int own = x;
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {              // inclusive sums over the lanes
            const int y = __shfl_up(x, off, 64);
            x += lane >= off ? y : 0;
        }
        const unsigned long long past = __builtin_amdgcn_ballot_w64(first + x > u);
        if (past != 0 || i0 + 64 >= nqt) {
            const int l = past != 0 ? __builtin_ctzll(past) : 0;
            i = i0 + l;
            first += __builtin_amdgcn_readlane(x - own, l);
            return;
        }
        first += __builtin_amdgcn_readlane(x, 63);
    }
}

template <int D>
constexpr int PF_NREG = 2 + 16 * (D / 32);   // floats of a lane's state: maximum, sum, output

__device__ __forceinline__ float max_xor32(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

__device__ __forceinline__ int key_perm(int x) { return (x & ~12) | (x & 4) << 1 | (x & 8) >> 1; }   // swap bits 2 and 3

template <int D, int N>
__device__ __forceinline__ void pf_put(const Kv4AttnArgs& a, size_t off, const float (&x)[N], bool& bad) {   // 4 dims
    uint2 w;
    if (a.out_f16) {
        f16 v[4];
#pragma unroll
        for (int j = 0; j < 4; j++) v[j] = act_f16(x[j], bad);
        __builtin_memcpy(&w, v, 8);
    } else {
        w = uint2{(uint32_t)bf16_bits_rne(x[0]) | (uint32_t)bf16_bits_rne(x[1]) << 16,
                  (uint32_t)bf16_bits_rne(x[2]) | (uint32_t)bf16_bits_rne(x[3]) << 16};
    }
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + off) = w;
}

template <int D, bool PIECES>
__global__ void __launch_bounds__(64 * PF_W) kv4_prefill_kernel(Kv4AttnArgs a) {
    constexpr int NS = D / 32, NF = D / 16, NW = D / 64;     // groups, K fragments, words per thread
    constexpr int TB = kv4_tile_bytes(D), CB = kv4_code_bytes(D);
    constexpr int FB = 32 * D * 2;                           // bytes of a 32-key tile's fragments
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char* const Ks = smem;                          // [2 buffers][2 tiles][NF][64 lanes][16]
    unsigned char* const Vs = smem + 4 * FB;                 // [2][2][NS][2][64][16]
    unsigned long long* const vbad = reinterpret_cast<unsigned long long*>(smem + 8 * FB);   // [4][NS + 1] NaN keys of V, by stage % 4
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, c = lane & 31;
    const int r = a.nq / a.nkv, R = a.rows * r, nkeys = a.ctx_base + a.rows;
    const int nqt = (R + PF_ROWS - 1) / PF_ROWS;
    // this block's part, or its run of units
    const long long total = a.pf_units * a.nkv;
    long long u = PIECES ? blockIdx.x / a.nkv : scalar(total * blockIdx.x / gridDim.x);
    const long long u1 = PIECES ? u + 1 : scalar(total * (blockIdx.x + 1) / gridDim.x);

    // Words of this thread: tile tt of the stage (not in scalar registers: their 64-bit products hold up the stage; 2011
    // queries of 28 heads of 4 behind 14001 tokens 485 us and 513)
    const int wv = tid >> 6, tt = wv >> 2, khi = wv & 1;
    const int ksub = wv >> 1 & 1;                            // K: lane slot khi 64 + lane, words NW ksub ..
    const int vhi = D == 128 ? khi : 0, vsub = D == 128 ? ksub : wv & 3;   // V: lane slot vhi 64 + lane, words NW vsub ..
    const int vdb = D == 128 ? 4 * khi + 2 * ksub : vsub, vg = vdb >> 1;
    const int kkey = 8 * ((lane & 15) >> 2) + 4 * khi + (lane & 3);
    uint32_t kw[NW], vw[NW];
    uint16_t ksc[NW], klo[NW];
    u32x4 vsc, vlo;
    const uint8_t *kb = nullptr, *vb = nullptr;
    // (a tile past the last key's repeats that one: its keys are never seen)
    auto load_k = [&](int st) __attribute__((always_inline)) {
        const uint8_t* kt = kb + (long long)min(2 * st + tt, (nkeys - 1) / KV4_TILE) * TB;
        const uint8_t* kc = kt + khi * 64 * NW * 8 + ksub * NW * 4;
        if constexpr (NW == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(kc + (uint32_t)lane * 16);
            kw[0] = x[0]; kw[1] = x[1];
        } else {
            kw[0] = *reinterpret_cast<const uint32_t*>(kc + (uint32_t)lane * 8);
        }
#pragma unroll
        for (int i = 0; i < NW; i++) {
            const uint8_t* pp = kt + CB + (NW * ksub + i) * 128 + (uint32_t)(2 * kkey);
            ksc[i] = *reinterpret_cast<const uint16_t*>(pp);
            klo[i] = *reinterpret_cast<const uint16_t*>(pp + 64);
        }
    };
    auto load_v = [&](int st) __attribute__((always_inline)) {
        const uint8_t* vt = vb + (long long)min(2 * st + tt, (nkeys - 1) / KV4_TILE) * TB;
        const uint8_t* vc = vt + vhi * 1024 + vsub * NW * 4;
        if constexpr (NW == 2) {
            const u32x2 y = *reinterpret_cast<const u32x2*>(vc + (uint32_t)lane * 16);
            vw[0] = y[0]; vw[1] = y[1];
        } else {
            vw[0] = *reinterpret_cast<const uint32_t*>(vc + (uint32_t)lane * 16);
        }
        const uint8_t* vp = vt + CB + vg * 128;
        vsc = *reinterpret_cast<const u32x4*>(vp + (uint32_t)(lane >> 4) * 16);
        vlo = *reinterpret_cast<const u32x4*>(vp + 64 + (uint32_t)(lane >> 4) * 16);
    };
    const DqConst dq = dq_const();
    const ZeroOff zo = zero_off(0.f);
    auto unpack_k = [&](int buf) __attribute__((always_inline)) {
        unsigned char* const kd = Ks + (buf * 2 + tt) * FB;
        const int kq4 = lane >> 4;
        const int row = key_perm(kkey);                 // of the score tile (its chunks rotated: fewer bank conflicts)
        const int kch = (row & 16) | ((row ^ (row >> 1 & 8)) & 15);
#pragma unroll
        for (int i = 0; i < NW; i++) {
            const f16x8 x = dequant8(kw[i], zo, dq);
            const f16 s = __builtin_bit_cast(f16, ksc[i]), lo = __builtin_bit_cast(f16, klo[i]);
            const f16x8 y = __builtin_elementwise_fma(x, f16x8{s, s, s, s, s, s, s, s}, f16x8{lo, lo, lo, lo, lo, lo, lo, lo});
            const int f = 2 * (NW * ksub + i) + (kq4 >> 1);
            *reinterpret_cast<f16x8*>(kd + (f * 64 + (kq4 & 1) * 32 + kch) * 16) = y;
        }
    };
    auto unpack_v = [&](int st, int buf, int nb) __attribute__((always_inline)) {
        unsigned char* const vd = Vs + (buf * 2 + tt) * FB;
        f16x8 s = __builtin_bit_cast(f16x8, vsc), lo = __builtin_bit_cast(f16x8, vlo);
        const int vn = lane & 15, vq4 = lane >> 4;
        const int key0 = st * PF_KST + tt * 32 + 8 * vq4;    // of the words' eight
        const int left = nkeys - key0;
        if (left < 8) {                                      // what lies behind the last key may be anything
#pragma unroll
            for (int e = 0; e < 8; e++) {
                s[e] = e < left ? s[e] : (f16)0.f;
                lo[e] = e < left ? lo[e] : (f16)0.f;
            }
        }
        // A NaN value would reach the rows that do not see its key as 0 * NaN: it is 0 here, and the rows that do see it
        // get their NaN from the list.
        const f16x2 l0{lo[0], lo[1]}, l1{lo[2], lo[3]}, l2{lo[4], lo[5]}, l3{lo[6], lo[7]};
        const f16x2 any = (l0 * (f16)0.f + l1 * (f16)0.f) + (l2 * (f16)0.f + l3 * (f16)0.f);
        if (!(any[0] + any[1] == (f16)0.f)) {
            uint32_t bits = 0;
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (lo[e] != lo[e]) {
                    bits |= 1u << e;
                    s[e] = lo[e] = (f16)0.f;
                }
            const unsigned long long m = (unsigned long long)bits << (tt * 32 + 8 * vq4);
            if (vn == 0) {
                atomicOr(vbad + nb * (NS + 1) + vg, m);
                atomicOr(vbad + nb * (NS + 1) + NS, m);
            }
        }
#pragma unroll
        for (int i = 0; i < NW; i++) {
            const f16x8 y = __builtin_elementwise_fma(dequant8(vw[i], zo, dq), s, lo);
            const int db = vdb + i;
            *reinterpret_cast<f16x8*>(vd + (((db >> 1) * 2 + (vq4 >> 1)) * 64 + (vq4 & 1) * 32 + (db & 1) * 16 + vn) * 16) = y;
        }
    };
    const int kch = (c & 16) | ((c ^ (c >> 1 & 8)) & 15);    // chunk of score row c
    bool bad = false;

    while (u < u1) {
        const int hk = PIECES ? blockIdx.x % a.nkv : (int)scalar(u / a.pf_units);
        const long long head0 = PIECES ? 0 : (long long)hk * a.pf_units;
        int e;
        long long first;
        pf_find(a, R, r, u - head0, e, first);
        first += head0;
        const int q = pf_tile(a, e, nqt);
        const int nst = pf_stages(q, R, r, a.ctx_base);      // stages of the tile
        int st0, st1;
        if constexpr (PIECES) {
            const long long n = (nst + a.pf_chunk - 1) / a.pf_chunk, j = u - first;
            st0 = (int)(nst * j / n);
            st1 = (int)(nst * (j + 1) / n);
            u = u1;
        } else {
            st0 = (int)(u - first);
            st1 = (int)min((long long)nst, u1 - first);
            u = first + st1;
        }
        kb = a.k + (long long)hk * a.stride_h;
        vb = a.v + (long long)hk * a.stride_h;
        load_k(st0);

        // ---- queries: this lane's row, dims 16 f + 8 h .. + 7 of every fragment f, times 2^qe
        const int row = q * PF_ROWS + wave * 32 + c;
        const int rowc = min(row, R - 1), tok = rowc / r, hd = hk * r + rowc % r;
        const uint16_t* qp = a.q + ((size_t)tok * a.nq + hd) * D + 8 * h;
        u32x4 qw[NF];
        float mx = 0.f;
#pragma unroll
        for (int f = 0; f < NF; f++) {
            qw[f] = *reinterpret_cast<const u32x4*>(qp + 16 * f);
#pragma unroll
            for (int i = 0; i < 4; i++)
                mx = fmaxf(mx, fmaxf(__builtin_fabsf(__uint_as_float(qw[f][i] << 16)),
                                     __builtin_fabsf(__uint_as_float(qw[f][i] & 0xFFFF0000u))));
        }
        mx = max_xor32(mx);
        const int qe = max(-113, min(120, 137 - (int)(__float_as_uint(mx) >> 23)));       // (to 2^10 ..: products stay small)
        const float up = __uint_as_float((uint32_t)(127 + qe) << 23);
        const float sl = a.scale * LOG2E * __uint_as_float((uint32_t)(127 - qe) << 23);
        f16x8 qf[NF];
#pragma unroll
        for (int f = 0; f < NF; f++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                qf[f][2 * i] = (f16)(__uint_as_float(qw[f][i] << 16) * up);
                qf[f][2 * i + 1] = (f16)(__uint_as_float(qw[f][i] & 0xFFFF0000u) * up);
            }
        const int lim = a.ctx_base + tok;                    // this row's last key
        const int row_lo = min(q * PF_ROWS + wave * 32, R - 1), row_hi = min(q * PF_ROWS + wave * 32 + 31, R - 1);
        const int lim_lo = a.ctx_base + row_lo / r, lim_hi = a.ctx_base + row_hi / r;     // of the wave's rows
        const bool active = q * PF_ROWS + wave * 32 < R;

        f32x16 o[NS];
#pragma unroll
        for (int i = 0; i < NS; i++) o[i] = f32x16{};
        float m = -INFINITY, l = 0.f;
        const int n = st1 - st0;
        const int non = active ? min(n, lim_hi / PF_KST + 1 - st0) : 0;      // stages that the wave's rows see keys of

        __syncthreads();                                     // (the last tile's readers are done)
        if (tid < 4 * (NS + 1)) vbad[tid] = 0;
        unpack_k(0);
        if (n > 1) load_k(st0 + 1);
        load_v(st0);
        __syncthreads();
        int next = 0;                                        // K of stage next + 1 and V of stage next are to be unpacked
        auto unpack_next = [&]() __attribute__((always_inline)) {
            if (next + 1 < n) unpack_k(next + 1 & 1);
            if (next < n) unpack_v(st0 + next, next & 1, next & 3);
            if (next + 2 < n) load_k(st0 + next + 2);
            if (next + 1 < n) load_v(st0 + next + 1);
            next++;
        };
        if (wave >= PF_W / 2) {                              // half a stage behind: vector work where the others multiply
            unpack_next();
            __syncthreads();
        }
        f16x8 pf[4];
#pragma clang loop unroll(disable)
        for (int s = 0; s <= n; s++) {
            // ---- matrix half: scores of stage s, output of stage s - 1
            f32x16 sc[2];
            if (s < non) {
                const unsigned char* K = Ks + (s & 1) * 2 * FB;
                sc[0] = f32x16{};
                sc[1] = f32x16{};
#pragma unroll
                for (int f = 0; f < NF; f++)
#pragma unroll
                    for (int t = 0; t < 2; t++) {
                        const f16x8 kf = *reinterpret_cast<const f16x8*>(K + t * FB + (f * 64 + h * 32 + kch) * 16);
                        sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[f], sc[t], 0, 0, 0);
                    }
            }
            if (s > 0 && s <= non) {
                const unsigned char* V = Vs + (s - 1 & 1) * 2 * FB;
#pragma unroll
                for (int ks = 0; ks < 4; ks++)
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        const f16x8 vf = *reinterpret_cast<const f16x8*>(V + (ks >> 1) * FB + ((i * 2 + (ks & 1)) * 64 + lane) * 16);
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[ks], o[i], 0, 0, 0);
                    }
                const unsigned long long* const bl = vbad + (s - 1 & 3) * (NS + 1);
                if (bl[NS] != 0) {                           // NaN for the rows that see one of the keys, in its group
                    const long long left = lim - (st0 + s - 1) * PF_KST;
                    const unsigned long long see = left >= 63 ? ~0ull : left < 0 ? 0ull : (2ull << left) - 1;
#pragma unroll
                    for (int i = 0; i < NS; i++)
                        if (bl[i] & see)
#pragma unroll
                            for (int e = 0; e < 16; e++) o[i][e] = __builtin_nanf("");
                }
            }
            if (s == n) break;
            __syncthreads();
            // ---- vector half: weights of stage s, the next tiles
            if (tid <= NS) vbad[(s + 1 & 3) * (NS + 1) + tid] = 0;       // (the list of stage s - 3)
            if (s < non) {
                const int kbase = (st0 + s) * PF_KST;
                float p[32];
#pragma unroll
                for (int e = 0; e < 32; e++) p[e] = sc[e / 16][e % 16];
                if (kbase + PF_KST - 1 > lim_lo) {
                    const int left = lim - kbase - 8 * h;
#pragma unroll
                    for (int e = 0; e < 32; e++) p[e] = 32 * (e / 16) + 16 * (e % 16 / 8) + e % 8 <= left ? p[e] : -INFINITY;
                }
                float mt = fmaxf(p[0], p[1]);
#pragma unroll
                for (int e = 2; e < 32; e++) mt = fmaxf(mt, p[e]);
                if (__builtin_amdgcn_ballot_w64(mt * sl > m + 8.f) != 0) {
                    const float mn = fmaxf(m, max_xor32(mt) * sl);
                    const float alpha = exp2_hw(m - (mn == -INFINITY ? 0.f : mn));
                    l *= alpha;
#pragma unroll
                    for (int i = 0; i < NS; i++)
#pragma unroll
                        for (int e = 0; e < 16; e++) o[i][e] *= alpha;
                    m = mn;
                }
                const float mb = m == -INFINITY ? 0.f : m;
                float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float x = exp2_hw(__builtin_fmaf(p[e], sl, -mb)), y = exp2_hw(__builtin_fmaf(p[e + 1], sl, -mb));
                    ls[e / 2 % 2] += x;
                    ls[2 + e / 2 % 2] += y;
                    const f16x2 w = __builtin_convertvector(f32x2{x, y}, f16x2);
                    pf[e / 8][e % 8] = w[0];
                    pf[e / 8][e % 8 + 1] = w[1];
                }
                l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
            }
            unpack_next();
            __syncthreads();
        }
        if (wave < PF_W / 2) __syncthreads();
        const bool whole = st0 == 0 && st1 == nst;
        const float lt = l + __shfl_xor(l, 32, 64);
        int row_o = q * PF_ROWS + wave * 32 + c;             // (worked out again: not kept in registers all along)
        asm volatile("" : "+v"(row_o));
        if (whole && row_o < R) {
            const float inv = lt == 0.f ? 0.f : 1.f / lt;
            const size_t orow = ((size_t)(row_o / r) * a.nq + hk * r + row_o % r) * D;
#pragma unroll
            for (int i = 0; i < NS; i++)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float x[4] = {o[i][e] * inv, o[i][e + 1] * inv, o[i][e + 2] * inv, o[i][e + 3] * inv};
                    pf_put<D>(a, orow + i * 32 + 2 * e + 4 * h, x, bad);
                }
        }
        if (!whole && active) {
            // state of this part: the block's slot; in a line slot 0 of two if it does not begin the tile, else 1
            const size_t slot = PIECES ? blockIdx.x : (size_t)blockIdx.x * 2 + (st0 == 0);
            float* pp = a.part + (slot * PF_W + wave) * PF_NREG<D> * 64 + lane;
            pp[0] = m;
            pp[64] = l;
#pragma unroll
            for (int i = 0; i < NS; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) pp[(2 + i * 16 + e) * 64] = o[i][e];
        }
    }
    flag_range(a.err, bad);
}

// Merges the pieces of the row tiles that a cut parts: block (row tile, kv head,
// 32-dim slice), thread (wave, lane) the lane's registers of the slice, piece
// after piece in key order.
template <int D>
__global__ void __launch_bounds__(64 * PF_W) kv4_prefill_merge_kernel(Kv4AttnArgs a, int nblocks) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, c = lane & 31;
    const int q = blockIdx.x, hk = blockIdx.y, i = blockIdx.z;
    const int r = a.nq / a.nkv, R = a.rows * r;
    const int nqt = (R + PF_ROWS - 1) / PF_ROWS, i0 = pf_tile(a, q, nqt);        // (its own inverse)
    long long before = 0;                                    // shares of the head's tiles before this one
    for (int k = 0; k < i0; k += 64) {
        int x = k + lane < i0 ? pf_weight(a, k + lane, nqt, R, r) : 0;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
        before += x;
    }
    const int own = pf_weight(a, i0, nqt, R, r);
    int b0 = 0, b1 = own - 1;                                // its parts; in a line the blocks from its first unit's to its last's
    if (!a.pf_chunk) {
        const long long total = a.pf_units * a.nkv, first = hk * a.pf_units + before;
        // block that has unit x: the largest b with total * b / nblocks <= x
        auto block_of = [&](long long x) { return (int)(((x + 1) * nblocks - 1) / total); };
        b0 = block_of(first);
        b1 = block_of(first + own - 1);
    }
    auto slot_of = [&](int b) { return a.pf_chunk ? (size_t)(before + b) * a.nkv + hk : (size_t)b * 2 + (b == b0); };
    if (b0 == b1 || q * PF_ROWS + wave * 32 >= R) return;
    constexpr int CB = 4;                                    // pieces requested together
    float M = -INFINITY, L = 0.f, acc[16] = {};
    for (int p0 = b0; p0 <= b1; p0 += CB) {
        float mc[CB], lc[CB], v[CB][16];
#pragma unroll
        for (int j = 0; j < CB; j++) {
            const int b = min(p0 + j, b1);
            const float* pp = a.part + (slot_of(b) * PF_W + wave) * PF_NREG<D> * 64 + lane;
            mc[j] = pp[0];
            lc[j] = pp[64];
#pragma unroll
            for (int e = 0; e < 16; e++) v[j][e] = pp[(2 + i * 16 + e) * 64];
        }
        float Mn = M;
#pragma unroll
        for (int j = 0; j < CB; j++)
            if (p0 + j <= b1) Mn = fmaxf(Mn, mc[j]);
        const float Mb = Mn == -INFINITY ? 0.f : Mn, s0 = exp2_hw(M - Mb);
        L *= s0;
#pragma unroll
        for (int e = 0; e < 16; e++) acc[e] *= s0;
#pragma unroll
        for (int j = 0; j < CB; j++) {
            if (p0 + j > b1) break;
            const float s = exp2_hw(mc[j] - Mb);
            L += s * lc[j];
#pragma unroll
            for (int e = 0; e < 16; e++) acc[e] += s * v[j][e];
        }
        M = Mn;
    }
    const int row = q * PF_ROWS + wave * 32 + c;
    const float lt = L + __shfl_xor(L, 32, 64);
    if (row >= R) return;
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    const size_t orow = ((size_t)(row / r) * a.nq + hk * r + row % r) * D;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const float x[4] = {acc[e] * inv, acc[e + 1] * inv, acc[e + 2] * inv, acc[e + 3] * inv};
        pf_put<D>(a, orow + i * 32 + 2 * e + 4 * h, x, bad);
    }
    flag_range(a.err, bad);
}

}  // namespace

// Shares per (row, kv head).  A block costs about 5 us to begin and end and a wave about 1
// us a tile, a second share the merge launch, about 2.5 us: below 32 tiles one block is the
// faster.  Else a tile per wave, as long as the blocks fit the CUs at once (two to a
// CU; one of more than 4 heads of d = 128).  32 heads of 8, d = 128, 1 row of 2048 keys: 1
// share 13.3 us, 2 12.4, 4 10.4, 8 9.7, 16 10.5; 16 rows of up to 32768: 1 192, 2
// 114, 4 105, 8 109; 14 heads of 2, d = 64, 512 keys: 1 5.7, 2 8.2; 28 heads of 4, d = 128, 8 rows
// of up to 8192: 4 26.5, 8 20.1, 16 29.3.
//
// The wide kernel (CT 2) is bound by the vector units, 1.3 us a tile of a SIMD.  Waves of
// four heads each, twice as many, took 8.7 and 8.0 us for 1 row of 500 and 2000 keys of
// 28 heads of 4 instead of 9.2 and 9.4, but 88 instead of 81 for 16 of up to 32000; three blocks
// of four waves to a CU (the queries in shared memory, 168 registers) 79, but 20.9 for 8 of up to 8192 instead
// of 18.4 and 27 for 1 of 30000 instead of 17: more shares to merge.
int kv4_decode_shares(int rows, int nkv, int r, int d, int max_ctx) {
    const long long tiles = ((long long)max_ctx + KV4_TILE) / KV4_TILE, pairs = (long long)rows * nkv;
    const bool wide = d == 128 && r > 4;
    const long long n = tiles < 32 ? 1 : std::min((wide ? 1 : 2) * kCus / pairs, (tiles + DW - 1) / DW);
    return (int)std::max(1ll, std::min({n, tiles, kMaxShares / pairs + 1}));
}

// Share states of any plan up to `rows` and max_ctx (grows with both).
size_t kv4_decode_part_bound(int rows, int nkv, int r, int d, int max_ctx) {
    const long long tiles = ((long long)max_ctx + KV4_TILE) / KV4_TILE, pairs = (long long)rows * nkv;
    return (size_t)std::min(pairs * tiles, pairs + kMaxShares) * r * (d + 2) * 4;
}

template <int D, int CT>
static int launch_decode(const Kv4AttnArgs& a, hipStream_t stream) {
    const size_t lds = (size_t)DW * a.r * D * 4;       // the waves' outputs (at most 32 KB)
    hipLaunchKernelGGL((kv4_decode_kernel<D, CT>), dim3(a.nkv, a.nsplit, a.rows), dim3(64 * DW), lds, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL(kv4_decode_merge_kernel<D>, dim3(a.nkv, a.r, a.rows), dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv4_decode(const Kv4AttnArgs& args, hipStream_t stream) {
    Kv4AttnArgs a = args;
    const int r = a.r = a.nq / a.nkv;
    const int tiles = (int)(((long long)a.max_ctx + KV4_TILE) / KV4_TILE);
    if (r < 1 || r > MAXR || a.nsplit < 1 || a.nsplit > tiles) return -1;
    if (a.nsplit > 1 && !a.part) return -1;
    a.per = (tiles + a.nsplit - 1) / a.nsplit;
    a.nsplit = (tiles + a.per - 1) / a.per;              // (no share beyond the longest context)
    if (a.d == 128) return r <= 4 ? launch_decode<128, 1>(a, stream) : launch_decode<128, 2>(a, stream);
    return a.d == 64 ? launch_decode<64, 1>(a, stream) : -1;
}

constexpr int kMaxParts = 512;       // states of parts in the workspace

// Few queries or keys are left to the decode kernel, a row for each (p.single): it has no fixed cost to speak of, but
// reads the keys once for every query.  The two take the same time at about 2^21 tiles x dims: heads of 128, 8 kv heads,
// 8 / 64 queries of 1000 keys 7.7 / 15.0 us and 12.2 / 19.5 with the prefill kernel, 8 / 12 of 16000 27 / 38 and 28 / 32,
// 24 of 3000 21 and 18; 2 kv heads of 64, 61 of 250 5 and 13.5, 64 of 16000 32 and 48.
// Up to four queries are always the decode kernel's: it reads the keys four times at most, where the prefill kernel
// unpacks and multiplies them for 256 rows.  32 heads of 8 of 128, 131000 keys, 1 / 2 / 4 / 6 queries 33 / 51 / 80 / 123 us
// and 114 with the prefill kernel; 28 of 4, 29 / 42 / 71 / 106 and 86 to 91 (four of 260000
// keys 130 and 124); 8 of 8 of 64, 23 / 33 / 56 / 85 and 109.
//
// For the prefill kernel the way of dealing out the work with the least estimated time, in us.  Pieces waste less on starts
// and on states; the line ends everywhere at once, and takes any number of stages with two states per block.  Measured (pieces, line):
// 128 wide, 32 heads of 8, 1000 tokens from nothing 37 and 51, 64 behind 4000 26.5 and 41, 512 behind 4096 71 and 69,
// 5000 from nothing 265 and 346; 28 heads of 4, 2000 behind 2000 137 and 148, and in parts that fill the chip badly 172.
Kv4PrefillPlan kv4_prefill_plan(int T, int hist, int nkv, int r, int d) {
    const int R = T * r, nqt = (R + PF_ROWS - 1) / PF_ROWS;
    Kv4PrefillPlan p;
    int most = 0;
    for (int q = 0; q < nqt; q++) {
        const int st = pf_stages(q, R, r, hist);
        p.units += st;
        most = std::max(most, st);
    }
    const size_t state = (size_t)PF_W * (2 + 16 * (d / 32)) * 64 * 4;
    const long long total = p.units * nkv;
    // of either kernel (grows with T and hist)
    const int few = std::min(T, 1024);                       // (more see too many keys)
    const long long tiles = ((long long)hist + few + KV4_TILE - 1) / KV4_TILE, pairs = (long long)few * nkv;
    p.part_bytes = std::max((size_t)std::min<long long>(kMaxParts, 2 * total) * state,
                            (size_t)std::min<long long>(2 * kCus, pairs * tiles) * r * (d + 2) * 4);
    p.single = T <= 4 || (T == few && pairs * tiles * d <= 1 << 21);
    if (p.single) return p;
    // a stage of one block alone and with all others (the clock falls), a part's start and end, its state written and read
    // back (of its waves that have rows), the merge launch
    const double t = d == 128 ? 2.2 : 1.9, tf = 1.1 * t, start = 5.0, merge = 3.0;
    const double part = std::min(1.0, (R + 31) / 32 / (double)PF_W) * state * 2 / 5.4e6;
    p.blocks = (int)std::min<long long>(kCus, total);
    const long long run = (total + p.blocks - 1) / p.blocks;
    int starts = 0;                                          // of the block that has the shortest tiles
    for (long long sum = 0; starts < nqt && sum < run; starts++) sum += pf_stages(starts, R, r, hist);
    double best = run * tf + (starts + 0.5) * start + 2 * p.blocks * part + merge;
    for (int c = (int)std::min<long long>(most, std::max<long long>(1, total / kMaxParts));; c += c < 8 ? 1 : c / 5) {
        c = std::min(c, most);
        long long items = 0;
        double longest = 0, work = 0, end = 0;               // us of a part, of all so far; end of one that has to wait
        for (int q = nqt - 1; q >= 0; q--) {
            const int st = pf_stages(q, R, r, hist), n = (st + c - 1) / c, len = (st + n - 1) / n;
            items += (long long)n * nkv;
            work += (double)n * nkv * (len * tf + start);
            longest = std::max(longest, len * t + start);
            if (items > kCus) end = std::max(end, work / kCus + len * t + start);
        }
        const bool split = c < most;
        if (!split || items <= kMaxParts) {
            double us = std::max(longest, std::min(end, (double)((items + kCus - 1) / kCus) * longest));
            if (split) us += items * part + merge;
            if (us < best) {
                best = us;
                p.chunk = c;
                p.blocks = (int)items;
            }
        }
        if (c >= most) break;
    }
    p.merge = p.chunk ? p.chunk < most : p.blocks > 1;
    return p;
}

// (for the host tests)
extern "C" void w4_kv4_prefill_plan(int T, int hist, int nkv, int r, int d, int* single, int* chunk, int* blocks, int* merge) {
    const Kv4PrefillPlan p = kv4_prefill_plan(T, hist, nkv, r, d);
    *single = p.single;
    *chunk = p.chunk;
    *blocks = p.blocks;
    *merge = p.merge;
}

template <int D, bool PIECES>
static int launch_prefill(const Kv4AttnArgs& a, const Kv4PrefillPlan& p, hipStream_t stream) {
    const size_t lds = (size_t)8 * 32 * D * 2 + 4 * (D / 32 + 1) * 8;
    static LdsLimit lim;
    if (ensure_lds_limit(lim, (const void*)kv4_prefill_kernel<D, PIECES>, lds)) return -1;
    hipLaunchKernelGGL((kv4_prefill_kernel<D, PIECES>), dim3(p.blocks), dim3(64 * PF_W), lds, stream, a);
    const int R = a.rows * (a.nq / a.nkv);
    if (p.merge)
        hipLaunchKernelGGL(kv4_prefill_merge_kernel<D>, dim3((R + PF_ROWS - 1) / PF_ROWS, a.nkv, D / 32), dim3(64 * PF_W), 0,
                           stream, a, p.blocks);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv4_prefill(const Kv4AttnArgs& a, hipStream_t stream) {
    if (a.rows < 1 || !a.part) return -1;
    const Kv4PrefillPlan p = kv4_prefill_plan(a.rows, a.ctx_base, a.nkv, a.nq / a.nkv, a.d);
    Kv4AttnArgs b = a;
    if (p.single) {
        b.max_ctx = a.ctx_base + a.rows - 1;
        b.nsplit = kv4_decode_shares(a.rows, a.nkv, a.nq / a.nkv, a.d, b.max_ctx);
        return launch_kv4_decode(b, stream);
    }
    // every block has a part, every state a slot
    if (p.blocks < 1 || (!p.chunk && p.blocks > std::min<long long>(kCus, p.units * a.nkv)) ||
        (p.chunk && p.merge && p.blocks > kMaxParts))
        return -1;
    b.pf_units = p.units;
    b.pf_chunk = p.chunk;
    if (a.d == 128) return p.chunk ? launch_prefill<128, true>(b, p, stream) : launch_prefill<128, false>(b, p, stream);
    if (a.d == 64) return p.chunk ? launch_prefill<64, true>(b, p, stream) : launch_prefill<64, false>(b, p, stream);
    return -1;
}

int load_kv4_attn() { return load_code((const void*)kv4_decode_kernel<128, 1>); }
