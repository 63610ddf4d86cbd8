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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;

// ---------------------------------------------------------------- decode

constexpr int DEC_W = 8;         // waves per block
constexpr int MAXR = 8;          // query heads per kv head

// Eight codes of a word as fp16 multiples of 2^-24: elements 0, 1, 4, 5 are
// c 2^-24, elements 2, 3, 6, 7 are 16 c 2^-24.
__device__ __forceinline__ f16x8 code_frag(uint32_t w) {
    const uint32_t w8 = w >> 8;
    const u32x4 r{w & 0x000F000Fu, w & 0x00F000F0u, w8 & 0x000F000Fu, w8 & 0x00F000F0u};
    return __builtin_bit_cast(f16x8, r);
}

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

// A tile's registers of one lane.
template <int D>
struct KvTile {
    static constexpr int NS = D / 32;
    uint32_t kc[2][NS];          // words of score tiles 0 and 1
    u32x4 vc[NS / 2];            // words of dim blocks 0 .. 3 (4 .. 7)
    f16x8 ks, kl, vs, vl;        // scale and offset of group g, tokens 8 q4 .. + 7
    float mk[8 / NS];            // mask of this lane's scores
};

// One block: a share of the tiles of one (row, kv head), all r query heads of
// the group.  Wave w takes tiles w, w + 8, .. of the share on its own; the next
// tile's loads are in flight while one is computed.  CT column tiles of 16 /
// NS heads.  Softmax: the maximum of a head moves only when a score passes it by
// more than 2 (all lanes of the wave then agree on the new one), so weights stay
// below e^2.  Weights times scales are a pair of fp16 numbers, hi + lo: s c and lo of a
// value near 0 cancel, so P' rounded once would leave 2^-12 of the group's range.
// They are multiplied by ef = 2^10 so that small ones keep their digits; if one
// passes the fp16 range after all (a scale above 8), ef drops to 1 for the rest of
// the share: e^2 times the largest scale (8734) is 64536.
template <int D, int CT>
__global__ void __launch_bounds__(64 * DEC_W) kv4_decode_kernel(Kv4AttnArgs a) {
    constexpr int NS = D / 32, NDB = D / 16, HC = 16 / NS, PS = 8 / NS;
    constexpr int TB = kv4_tile_bytes(D), CB = kv4_code_bytes(D);
    __shared__ __attribute__((aligned(16))) float ored[DEC_W][MAXR][D];
    __shared__ float gst[DEC_W][MAXR][2], glo[DEC_W][MAXR][NS];
    __shared__ unsigned last_flag;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.x / a.nkv, hk = blockIdx.x % a.nkv;
    const int ctx = min(a.ctx_lens ? a.ctx_lens[b] : a.ctx_base + b, a.max_ctx);
    const int ntiles = (ctx + KV4_TILE) / KV4_TILE;             // of ctx + 1 keys
    const int n = max(1, min(a.nsplit, ntiles)), part = blockIdx.y;
    if (part >= n) return;
    const int tile0 = (int)((long long)part * ntiles / n), tile1 = (int)((long long)(part + 1) * ntiles / n);
    const int r = a.nq / a.nkv;
    const int n16 = lane & 15, q4 = lane >> 4, g = n16 % NS;
    const long long base = (long long)b * a.stride_b + (long long)hk * a.stride_h;
    const uint8_t* const kb = a.k + base;
    const uint8_t* const vb = a.v + base;
    const float* const mrow = a.mask ? a.mask + (size_t)b * a.max_seq : nullptr;
    // key of score i (NS 4: tile i; NS 2: tile i / 2) of this lane, of 32
    auto score_key = [&](int i) { return NS == 4 ? 8 * q4 + 4 * i + g : 8 * q4 + 4 * (i >> 1) + 2 * (i & 1) + g; };

    KvTile<D> nx;
    auto load_tile = [&](int tile) __attribute__((always_inline)) {
        const uint8_t* kt = kb + (long long)tile * TB;
        const uint8_t* vt = vb + (long long)tile * TB;
#pragma unroll
        for (int t = 0; t < 2; t++) {
            if constexpr (NS == 4) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(kt + (t * 64 + lane) * 16);
#pragma unroll
                for (int s = 0; s < NS; s++) nx.kc[t][s] = w[s];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2*>(kt + (t * 64 + lane) * 8);
                nx.kc[t][0] = w[0];
                nx.kc[t][1] = w[1];
            }
        }
        const int po = CB + g * 128 + q4 * 16;
        nx.ks = *reinterpret_cast<const f16x8*>(kt + po);
        nx.kl = *reinterpret_cast<const f16x8*>(kt + po + 64);
#pragma unroll
        for (int i = 0; i < NS / 2; i++) nx.vc[i] = *reinterpret_cast<const u32x4*>(vt + (i * 64 + lane) * 16);
        nx.vs = *reinterpret_cast<const f16x8*>(vt + po);
        nx.vl = *reinterpret_cast<const f16x8*>(vt + po + 64);
        if (mrow) {
#pragma unroll
            for (int i = 0; i < PS; i++) nx.mk[i] = mrow[min(tile * KV4_TILE + score_key(i), ctx)];
        }
    };
    int tile = tile0 + wave;
    if (tile < tile1) load_tile(tile);

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
        mx = group_max<NS>(mx);
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
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
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        qs[ct] = sum * 0x1p-24f;
#pragma unroll
        for (int s = 0; s < NS; s++) qf[ct][s] = g == s ? fr : f16x8{};
    }
    const float f1 = a.scale * 0x1p24f;

    f32x4 o[CT][NDB];
    float m[CT], l[CT], olo[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
#pragma unroll
        for (int i = 0; i < NDB; i++) o[ct][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m[ct] = -INFINITY;
        l[ct] = olo[ct] = 0.f;
    }
    float ef = 1024.f;

    for (; tile < tile1; tile += DEC_W) {
        const KvTile<D> c = nx;
        if (tile + DEC_W < tile1) load_tile(tile + DEC_W);
        f32x4 acc[CT][2];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) acc[ct][0] = acc[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; s++)
#pragma unroll
            for (int t = 0; t < 2; t++) {
                const f16x8 kf = code_frag(c.kc[t][s]);
#pragma unroll
                for (int ct = 0; ct < CT; ct++) acc[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[ct][s], acc[ct][t], 0, 0, 0);
            }
        const bool special = mrow || (tile + 1) * KV4_TILE > ctx + 1;
        float p[CT][PS];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) {
            float sc[PS];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; j++)
                    v[j] = __builtin_fmaf((float)c.ks[4 * t + j], acc[ct][t][j], (float)c.kl[4 * t + j] * qs[ct]);
                // sums over the groups (lanes g): lane g keeps the key 4 t + g (NS 2: keys 4 t + g, 4 t + 2 + g)
                const bool b0 = lane & 1;
                const float r0 = (b0 ? v[1] : v[0]) + dpp_mov<0xB1>(b0 ? v[0] : v[1]);
                const float r1 = (b0 ? v[3] : v[2]) + dpp_mov<0xB1>(b0 ? v[2] : v[3]);
                if constexpr (NS == 4) {
                    const bool b1 = lane & 2;
                    sc[t] = (b1 ? r1 : r0) + dpp_mov<0x4E>(b1 ? r0 : r1);
                } else {
                    sc[2 * t] = r0;
                    sc[2 * t + 1] = r1;
                }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < PS; i++) {
                sc[i] = sc[i] * f1 * f2[ct];
                if (special) {
                    bool seen = tile * KV4_TILE + score_key(i) <= ctx;
                    if (mrow) {
                        seen = seen && c.mk[i] != -INFINITY;
                        sc[i] += c.mk[i];
                    }
                    sc[i] = seen ? sc[i] : -INFINITY;
                }
                mx = fmaxf(mx, sc[i]);
            }
            if (__builtin_amdgcn_ballot_w64(mx > m[ct] + 2.f) != 0) {
                mx = group_max<NS>(mx);
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float mn = fmaxf(m[ct], mx);
                const float alpha = exp2_hw((m[ct] - (mn == -INFINITY ? 0.f : mn)) * LOG2E);
                l[ct] *= alpha;
                olo[ct] *= alpha;
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
#pragma unroll
            for (int i = 0; i < PS; i++) {
                p[ct][i] = exp2_hw((sc[i] - mb) * LOG2E);
                l[ct] += p[ct][i];
            }
        }
        // P'_(h,g) of keys 8 q4 + e: weights from the lanes that hold them; offsets summed on the way
        f16x8 pf[CT], pl[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) {
            float w[8];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                if constexpr (NS == 4) {
                    w[4 * t + 0] = dpp_mov<0x00>(p[ct][t]);
                    w[4 * t + 1] = dpp_mov<0x55>(p[ct][t]);
                    w[4 * t + 2] = dpp_mov<0xAA>(p[ct][t]);
                    w[4 * t + 3] = dpp_mov<0xFF>(p[ct][t]);
                } else {
                    w[4 * t + 0] = dpp_mov<0xA0>(p[ct][2 * t]);
                    w[4 * t + 1] = dpp_mov<0xF5>(p[ct][2 * t]);
                    w[4 * t + 2] = dpp_mov<0xA0>(p[ct][2 * t + 1]);
                    w[4 * t + 3] = dpp_mov<0xF5>(p[ct][2 * t + 1]);
                }
            }
            float ps[8], pmax = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                float s = (float)c.vs[e], lo = (float)c.vl[e];
                if (special) {                       // (hidden keys may hold NaN)
                    s = w[e] == 0.f ? 0.f : s;
                    lo = w[e] == 0.f ? 0.f : lo;
                }
                ps[e] = w[e] * s;
                olo[ct] = __builtin_fmaf(w[e], lo, olo[ct]);
                pmax = fmaxf(pmax, ps[e]);
            }
            if (__builtin_amdgcn_ballot_w64(pmax * ef > 65504.f) != 0) {
                const float down = 1.f / ef;
                ef = 1.f;
#pragma unroll
                for (int c2 = 0; c2 < CT; c2++)
#pragma unroll
                    for (int i = 0; i < NDB; i++)
#pragma unroll
                        for (int e = 0; e < 4; e++) o[c2][i][e] *= down;
                if (ct == 1) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        pf[0][e] = (f16)((float)pf[0][e] * down);
                        pl[0][e] = (f16)((float)pl[0][e] * down);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float es = e & 2 ? ef * 0.0625f : ef, x = ps[e] * es, y = ps[e + 1] * es;
                const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(x, y));
                const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(x - (float)hi[0], y - (float)hi[1]));
                pf[ct][e] = hi[0]; pf[ct][e + 1] = hi[1];
                pl[ct][e] = lo[0]; pl[ct][e + 1] = lo[1];
            }
        }
#pragma unroll
        for (int i = 0; i < NDB; i++) {
            const f16x8 vf = code_frag(c.vc[i / 4][i % 4]);
#pragma unroll
            for (int ct = 0; ct < CT; ct++) {
                o[ct][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pf[ct], vf, o[ct][i], 0, 0, 0);
                o[ct][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl[ct], vf, o[ct][i], 0, 0, 0);
            }
        }
    }

    // ---- the waves' states meet in LDS
    const float of = 0x1p24f / ef;
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        l[ct] = group_sum<NS>(l[ct]);
        l[ct] += __shfl_xor(l[ct], 16, 64);
        l[ct] += __shfl_xor(l[ct], 32, 64);
        olo[ct] += __shfl_xor(olo[ct], 16, 64);
        olo[ct] += __shfl_xor(olo[ct], 32, 64);
        const int h = ct * HC + n16 / NS;
        if (q4 == 0 && h < r) {
            glo[wave][h][g] = olo[ct];
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
                if (ho < r) ored[wave][ho][16 * i + n16] = o[ct][i][j] * of;
            }
    }
    __syncthreads();
    // share state: [row, kv head][share][r heads][D] outputs, then [..][r][2] (max, sum)
    const size_t slot = (size_t)blockIdx.x * a.nsplit;
    unsigned long long* const po = reinterpret_cast<unsigned long long*>(a.part) + slot * r * (D / 2);
    unsigned long long* const pst = reinterpret_cast<unsigned long long*>(a.part) +
                                    (size_t)gridDim.x * a.nsplit * r * (D / 2) + slot * r;
    auto pack = [](float x, float y) { return (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x); };
    const size_t orow = ((size_t)b * a.nq + hk * r) * D;
    bool bad = false;
    auto put = [&](int idx, float x, float y, float lt) __attribute__((always_inline)) {     // output pair idx
        const float u = lt == 0.f ? 0.f : x / lt, v = lt == 0.f ? 0.f : y / lt;              // (NaN stays)
        uint32_t w;
        if (a.out_f16) {
            const f16 h0 = act_f16(u, bad), h1 = act_f16(v, bad);
            w = (uint32_t)__builtin_bit_cast(uint16_t, h0) | (uint32_t)__builtin_bit_cast(uint16_t, h1) << 16;
        } else {
            w = (uint32_t)bf16_bits_rne(u) | (uint32_t)bf16_bits_rne(v) << 16;
        }
        reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + orow)[idx] = w;
    };
    for (int idx = tid; idx < r * (D / 2); idx += 64 * DEC_W) {
        const int i = idx / (D / 2), d = 2 * (idx % (D / 2));
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < DEC_W; w++) M = fmaxf(M, gst[w][i][0]);
        float x = 0.f, y = 0.f, lt = 0.f;
#pragma unroll
        for (int w = 0; w < DEC_W; w++) {
            const float sc = gst[w][i][0] == -INFINITY ? 0.f : exp2f((gst[w][i][0] - M) * LOG2E);
            x += sc * (ored[w][i][d] + glo[w][i][d / 32]);
            y += sc * (ored[w][i][d + 1] + glo[w][i][d / 32]);
            lt += sc * gst[w][i][1];
        }
        if (n == 1) {
            put(idx, x, y, lt);
        } else {
            __hip_atomic_store(po + (size_t)part * r * (D / 2) + idx, pack(x, y), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (d == 0)
                __hip_atomic_store(pst + part * r + i, pack(M, lt), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (n > 1) {
        // the last share to arrive merges all of them, in their order
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this thread's stores are complete
        __syncthreads();
        if (tid == 0)
            last_flag = __hip_atomic_fetch_add(a.cnt + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 ==
                        (unsigned)n;
        __syncthreads();
        if (!last_flag) return;
        float2* const st = reinterpret_cast<float2*>(&ored[0][0][0]);     // [share][r] (max, sum)
        for (int i = tid; i < n * r; i += 64 * DEC_W) {
            const unsigned long long u = __hip_atomic_load(pst + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            st[i] = float2{__uint_as_float((unsigned)u), __uint_as_float((unsigned)(u >> 32))};
        }
        __syncthreads();
        constexpr int CBK = 16;              // shares requested together
        for (int idx = tid; idx < r * (D / 2); idx += 64 * DEC_W) {
            const int i = idx / (D / 2);
            float M = -INFINITY;
            for (int c = 0; c < n; c++) M = fmaxf(M, st[c * r + i].x);
            float x = 0.f, y = 0.f, lt = 0.f;
            for (int c0 = 0; c0 < n; c0 += CBK) {
                unsigned long long v[CBK];
#pragma unroll
                for (int c = 0; c < CBK; c++)
                    v[c] = __hip_atomic_load(po + (size_t)(c0 + c < n ? c0 + c : n - 1) * r * (D / 2) + idx,
                                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int c = 0; c < CBK; c++) {
                    if (c0 + c >= n) break;
                    const float2 s = st[(c0 + c) * r + i];
                    if (s.x == -INFINITY && s.y == 0.f) continue;
                    const float w = exp2f((s.x - M) * LOG2E);
                    lt += w * s.y;
                    x += w * __uint_as_float((unsigned)v[c]);
                    y += w * __uint_as_float((unsigned)(v[c] >> 32));
                }
            }
            put(idx, x, y, lt);
        }
    }
    flag_range(a.err, bad);
}

// Clears the arrival counters (a kernel, so that it can be captured).
__global__ void __launch_bounds__(256) kv4_zero_kernel(unsigned* cnt, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) cnt[i] = 0u;
}

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

Kv4DecodePlan kv4_decode_plan(int rows, int nkv, int r, int d, int max_ctx) {
    const long long tiles = ((long long)max_ctx + KV4_TILE) / KV4_TILE, groups = (long long)rows * nkv;
    Kv4DecodePlan p;
    const long long want = (512 + groups - 1) / groups;
    p.nsplit = (int)std::max(1ll, std::min({want, (tiles + 2 * DEC_W - 1) / (2 * DEC_W), 256ll}));
    p.part_bytes = p.nsplit > 1 ? (size_t)groups * p.nsplit * r * (d + 2) * 4 : 0;
    p.cnt_bytes = p.nsplit > 1 ? (size_t)groups * 4 : 0;
    return p;
}

// Share states of any plan up to `rows` and max_ctx (grows with both).
size_t kv4_decode_part_bound(int rows, int nkv, int r, int d, int max_ctx) {
    const long long tiles = ((long long)max_ctx + KV4_TILE) / KV4_TILE, groups = (long long)rows * nkv;
    const long long shares = std::min(groups * ((tiles + 2 * DEC_W - 1) / (2 * DEC_W)), groups + 511);
    return (size_t)shares * r * (d + 2) * 4;
}

int launch_kv4_decode(const Kv4AttnArgs& a, bool zeroed, hipStream_t stream) {
    const int r = a.nq / a.nkv;
    if (r < 1 || r > MAXR || a.nsplit < 1 || (a.nsplit > 1 && (!a.part || !a.cnt))) return -1;
    const int groups = a.rows * a.nkv;
    if (a.nsplit > 1 && !zeroed)
        hipLaunchKernelGGL(kv4_zero_kernel, dim3((groups + 255) / 256), dim3(256), 0, stream, a.cnt, groups);
    const dim3 grid(groups, a.nsplit), block(64 * DEC_W);
    if (a.d == 128 && r <= 4) hipLaunchKernelGGL((kv4_decode_kernel<128, 1>), grid, block, 0, stream, a);
    else if (a.d == 128) hipLaunchKernelGGL((kv4_decode_kernel<128, 2>), grid, block, 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL((kv4_decode_kernel<64, 1>), grid, block, 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv4_attn(const Kv4AttnArgs& a, hipStream_t stream) {
    const dim3 grid(a.rows, a.nq);
    if (a.d == 128) hipLaunchKernelGGL(kv4_attn_kernel<128>, grid, dim3(256), 0, stream, a);
    else if (a.d == 64) hipLaunchKernelGGL(kv4_attn_kernel<64>, grid, dim3(256), 0, stream, a);
    else return -1;
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int load_kv4_attn() { return load_code((const void*)kv4_attn_kernel<128>); }
