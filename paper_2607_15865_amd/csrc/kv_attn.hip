// Grouped-query attention over the bf16 cache with a window, sinks and draft
// trees (kv_attn.h).
//
// The rows of a (sequence, kv head) are its N queries times the r query heads of
// the group, row i r + h.  Every row sees, of the slots before `high`, those from
// `low` on and the sinks, and of a tree's slots those in its mask.  Keys are taken in tiles; tiles
// that no row sees, between the sinks and the window, are never touched, and only tiles
// at a border (of the window, the sinks, the context, in the tree) are masked key by key.  Two kernels:
// kv_attn_few_kernel gives a wave keys of its own (few rows: bound by the
// cache read), kv_attn_many_kernel gives a wave rows of its own and lets
// all waves of a block share the keys (many rows: bound by the matrix units).
//
// A value that is not finite must not reach rows that do not see its slot, as 0
// times it would: where rows differ in what they see, such values are 0 in the
// products, and the rows that do see them are set to NaN.
#include <algorithm>
#include <climits>

#include "kv_attn.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

constexpr float LOG2E = 1.4426950408889634f;
constexpr int kCus = 256;

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
__device__ __forceinline__ float max_halves(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

// A 16-bit half of some word is a bf16 NaN or infinity.
__device__ __forceinline__ bool not_finite(u32x4 w) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; i++) bad |= (w[i] & 0x7F800000u) == 0x7F800000u || (w[i] & 0x7F80u) == 0x7F80u;
    return bad;
}

// ---------------------------------------------------------------- what rows see

// First slot of the window at position p.
__host__ __device__ inline int window_low(int p, int window) {
    return window == INT_MAX ? 0 : p - (window - 1) > 0 ? p - (window - 1) : 0;
}

// The slots that rows of a sequence see, in tiles of KT: tiles 0 .. sink - 1 with
// sinks, then `first` .. last; low: the lowest slot of any row's window, end: the
// last slot of any row.
struct KeyTiles {
    int sink, first, n;
};
template <int KT>
__host__ __device__ inline KeyTiles key_tiles(int low, int end, int sinks) {
    KeyTiles t;
    t.first = low / KT;
    const int s = sinks < end + 1 ? sinks : end + 1;
    t.sink = (s + KT - 1) / KT < t.first ? (s + KT - 1) / KT : t.first;
    t.n = end < 0 ? 0 : t.sink + end / KT - t.first + 1;
    return t;
}
__device__ __forceinline__ int tile_at(const KeyTiles& t, int i) { return i < t.sink ? i : t.first + i - t.sink; }

// The keys kb .. kb + 63 up to x, as bits.
__device__ __forceinline__ u64 up_to(int x, int kb) {
    const int n = x - kb;
    return n < 0 ? 0 : n >= 63 ? ~0ull : (2ull << n) - 1;
}

// What a row sees of a sequence.
struct RowView {
    int low, high;           // context: slots low .. high
    const u64* tree;         // its mask, or null
};
__device__ __forceinline__ RowView row_view(const KvAttnArgs& a, int b, int i, int ctx) {
    const size_t at = (size_t)b * a.N + i;
    RowView v;
    const int p = a.tree ? (a.pos ? a.pos[at] : ctx) : ctx + i;
    v.low = window_low(p, a.window);
    v.high = a.tree ? ctx - 1 : p;
    v.tree = a.tree ? a.tree + at * a.words : nullptr;
    return v;
}
// Of keys kb .. kb + 63, as bits.
__device__ __forceinline__ u64 seen_bits(const KvAttnArgs& a, const RowView& v, int ctx, int kb) {
    u64 x = up_to(v.high, kb) & (~up_to(v.low - 1, kb) | up_to(a.sinks - 1, kb));
    const int n = kb - ctx;                                  // (node of the first key)
    if (v.tree && n > -64 && n < a.N) {
        const int w = n >> 6, sh = n & 63;
        u64 t = w >= 0 ? v.tree[w] >> sh : 0;
        if (sh && w + 1 < a.words) t |= v.tree[w + 1] << (64 - sh);
        x |= t & up_to(a.N - 1, n);
    }
    return x;
}

// ---------------------------------------------------------------- few rows

constexpr int FW = 8;            // waves per block
constexpr int FKT = 32;          // keys per tile

// One block: up to 16 CT rows of a (sequence, kv head) and a share of its key
// tiles; wave w takes tiles w, w + 8, .. of the share on its own, so there is no
// barrier in the loop.  K goes from memory straight into the A operand of the
// 16x16x32 MFMA, V through a swizzled LDS tile of the wave, out of which the
// transposing read takes V^T; both are requested a tile ahead.  Scores are
// formed transposed, S^T = K Q^T, with the key rows in the order that leaves the weights
// in the operand layout of P^T.  A maximum moves only when a score passes it by more
// than 5 (weights below e^5); the weights are multiplied as bf16 pairs hi + lo: the matrix units
// have the time, and the weights of short contexts keep 16 bits.
template <int D, int CT>
__global__ void __launch_bounds__(64 * FW) kv_attn_few_kernel(KvAttnArgs a) {
    constexpr int NCK = D / 8, KROWS = 64 / NCK, NV = FKT / KROWS, NS = D / 32, NDB = D / 16, RT = 16 * CT;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ float gst[FW][RT][2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hk = blockIdx.x % a.nkv, row0 = blockIdx.x / a.nkv * RT, part = blockIdx.y, b = blockIdx.z;
    const int r = a.nq / a.nkv, R = a.N * r, nr = min(RT, R - row0);
    const int n16 = lane & 15, q4 = lane >> 4;
    int ctx = a.ctx_lens ? a.ctx_lens[b] : a.ctx_base;

    // ---- queries: column n16 of column tile ct is row row0 + 16 ct + n16, dims 32 s + 8 q4 .. + 7
    u32x4 qw[CT][NS];
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        const int row = min(row0 + 16 * ct + n16, R - 1);
        const uint16_t* qp = a.q + (((size_t)b * a.N + row / r) * a.nq + hk * r + row % r) * D + 8 * q4;
#pragma unroll
        for (int s = 0; s < NS; s++) qw[ct][s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
    }
    ctx = min(ctx, a.max_ctx);

    // ---- this block's tiles
    const int i0 = row0 / r, i1 = (row0 + nr - 1) / r;       // (of a chain)
    const int end = ctx < 0 ? -1 : a.tree ? ctx + a.N - 1 : ctx + i1;
    const KeyTiles kt = key_tiles<FKT>(window_low(a.tree ? ctx : ctx + i0, a.window), end, a.sinks);
    const int high_min = a.tree ? ctx - 1 : ctx + i0, low_max = window_low(a.tree ? ctx + a.N - 1 : ctx + i1, a.window);
    const int t0 = (int)((long long)kt.n * part / a.nsplit), t1 = (int)((long long)kt.n * (part + 1) / a.nsplit);
    const long long base = b * a.stride_b + hk * a.stride_h;
    const uint16_t* const kc = a.k + base;
    const uint16_t* const vc = a.v + base;
    const float* const mrow = a.mask ? a.mask + (size_t)b * a.max_seq : nullptr;
    const uint32_t ss = (uint32_t)a.stride_s;
    unsigned char* const Vst = smem + wave * FKT * D * 2;    // [32 keys][D], 16-byte chunks swizzled by key
    auto vswz = [](int k) { return 2 * ((k >> 3) & 3); };

    // A row n16 of score tile t is key 8 (n16 / 4) + 4 t + n16 % 4 of the tile, so register j of lane (n16, q4) is key
    // 8 q4 + 4 t + j; keys past the last one read that one
    u32x4 kr[2][NS], vr[NV];
    float mk[8];                                             // mask of keys 8 q4 .. + 7
    auto load_k = [&](int kb) __attribute__((always_inline)) {
        const uint16_t* kt0 = kc + kb * a.stride_s;
        const int lim = end - kb;
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const uint32_t off = (uint32_t)min(8 * (n16 >> 2) + 4 * t + (n16 & 3), lim) * ss + 8 * q4;
#pragma unroll
            for (int s = 0; s < NS; s++) kr[t][s] = *reinterpret_cast<const u32x4*>(kt0 + off + 32 * s);
        }
        if (mrow) {
#pragma unroll
            for (int e = 0; e < 8; e++) mk[e] = mrow[kb + min(8 * q4 + e, lim)];
        }
    };
    auto load_v = [&](int kb) __attribute__((always_inline)) {
        const uint16_t* vt0 = vc + kb * a.stride_s;
        const int lim = end - kb;
#pragma unroll
        for (int i = 0; i < NV; i++)
            vr[i] = *reinterpret_cast<const u32x4*>(vt0 + (uint32_t)min(i * KROWS + lane / NCK, lim) * ss + lane % NCK * 8);
    };
    int t = t0 + wave;
    if (t < t1) {
        load_k(tile_at(kt, t) * FKT);
        load_v(tile_at(kt, t) * FKT);
    }
    bf16x8 qf[CT][NS];
#pragma unroll
    for (int ct = 0; ct < CT; ct++)
#pragma unroll
        for (int s = 0; s < NS; s++) qf[ct][s] = __builtin_bit_cast(bf16x8, qw[ct][s]);

    f32x4 o[CT][NDB];
    float m[CT], l[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
#pragma unroll
        for (int i = 0; i < NDB; i++) o[ct][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m[ct] = -INFINITY;
        l[ct] = 0.f;
    }
    for (; t < t1; t += FW) {
        const int kb = tile_at(kt, t) * FKT, next = t + FW < t1 ? tile_at(kt, t + FW) * FKT : -1;
        f32x4 acc[CT][2];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) acc[ct][0] = acc[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; s++)
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int ct = 0; ct < CT; ct++)
                    acc[ct][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[h][s]), qf[ct][s], acc[ct][h], 0, 0, 0);
        float p[CT][8];
#pragma unroll
        for (int ct = 0; ct < CT; ct++)
#pragma unroll
            for (int e = 0; e < 8; e++) p[ct][e] = acc[ct][e / 4][e % 4] * a.scale;
        uint32_t bad = 0, seen[CT];                          // keys whose values are not finite, keys that the rows see
        if (mrow || kb + FKT - 1 > high_min || (kb < low_max && kb + FKT > a.sinks)) {
            int col = n16;
            asm volatile("" : "+v"(col));                    // (worked out here: not kept in registers all along)
#pragma unroll
            for (int ct = 0; ct < CT; ct++)
                seen[ct] = (uint32_t)seen_bits(a, row_view(a, b, min(row0 + 16 * ct + col, R - 1) / r, ctx), ctx, kb);
            if (a.N == 1) {                                  // all rows see the same: what they do not see is 0
                uint32_t mine = seen[0] >> (8 * q4) & 0xFF;
                if (mrow) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        mine &= ~((uint32_t)(mk[e] == -INFINITY) << e);
#pragma unroll
                        for (int ct = 0; ct < CT; ct++) p[ct][e] += mk[e];
                    }
                }
#pragma unroll
                for (int ct = 0; ct < CT; ct++)
#pragma unroll
                    for (int e = 0; e < 8; e++) p[ct][e] = mine >> e & 1 ? p[ct][e] : -INFINITY;
#pragma unroll
                for (int i = 0; i < NV; i++) {
                    const int k = i * KROWS + lane / NCK;    // (lane 16 (k / 8) has its bit)
                    if (!(__shfl(mine, 16 * (k >> 3), 64) >> (k & 7) & 1)) vr[i] = u32x4{0u, 0u, 0u, 0u};
                }
            } else {
#pragma unroll
                for (int ct = 0; ct < CT; ct++)
#pragma unroll
                    for (int e = 0; e < 8; e++) p[ct][e] = seen[ct] >> (8 * q4 + e) & 1 ? p[ct][e] : -INFINITY;
#pragma unroll
                for (int i = 0; i < NV; i++) {
                    const u64 x = __builtin_amdgcn_ballot_w64(not_finite(vr[i]));
                    if (x) {
                        for (int k = 0; k < KROWS; k++)
                            if (x >> (k * NCK) & ((1ull << NCK) - 1)) bad |= 1u << (i * KROWS + k);
                        if (bad >> (i * KROWS + lane / NCK) & 1) vr[i] = u32x4{0u, 0u, 0u, 0u};
                    }
                }
            }
        }
        // V to LDS (its readers below are this wave alone, so no barrier; a wave's LDS operations are served in order)
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int k = i * KROWS + lane / NCK;
            *reinterpret_cast<u32x4*>(Vst + k * D * 2 + ((lane % NCK ^ vswz(k)) << 4)) = vr[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (next >= 0) {
            load_k(next);
            load_v(next);
        }
        bf16x8 phi[CT], plo[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ct++) {
            float mx = p[ct][0];
#pragma unroll
            for (int e = 1; e < 8; e++) mx = fmaxf(mx, p[ct][e]);
            if (__builtin_amdgcn_ballot_w64(mx > m[ct] + 5.f) != 0) {
                const float mn = fmaxf(m[ct], max_quarters(mx));
                const float alpha = exp2_hw((m[ct] - (mn == -INFINITY ? 0.f : mn)) * LOG2E);
                l[ct] *= alpha;
                m[ct] = mn;
#pragma unroll
                for (int i = 0; i < NDB; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) o[ct][i][e] *= alpha;
            }
            const float mb = m[ct] == -INFINITY ? 0.f : m[ct];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {                 // (the difference first: a mask may be the lowest float)
                const float x = exp2_hw((p[ct][e] - mb) * LOG2E), y = exp2_hw((p[ct][e + 1] - mb) * LOG2E);
                l[ct] += x + y;
                const bf16x2 hi = __builtin_convertvector(f32x2{x, y}, bf16x2);
                const bf16x2 lo = __builtin_convertvector(f32x2{x - (float)hi[0], y - (float)hi[1]}, bf16x2);
                phi[ct][e] = hi[0]; phi[ct][e + 1] = hi[1];
                plo[ct][e] = lo[0]; plo[ct][e + 1] = lo[1];
            }
        }
        // O^T += V^T P^T per 16-dim block db: lane (n16, q4) takes V of keys 8 q4 .. + 7, dim 16 db + n16 (two transposing
        // reads: lane n16 of its group points at key 8 q4 + n16 / 4 (+ 4), dims 16 db + 4 (n16 % 4) .. + 3)
        const uint16_t* Vw = reinterpret_cast<const uint16_t*>(Vst + (8 * q4 + (n16 >> 2)) * D * 2);
#pragma unroll
        for (int db = 0; db < NDB; db++) {
            const int off = (((2 * db + ((n16 & 3) >> 1)) ^ (2 * q4)) << 3) | (4 * (n16 & 1));
            const i16x4 v0 = lds_read_tr16(Vw + off), v1 = lds_read_tr16(Vw + 4 * D + off);
            const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int ct = 0; ct < CT; ct++) {
                o[ct][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, phi[ct], o[ct][db], 0, 0, 0);
                o[ct][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, plo[ct], o[ct][db], 0, 0, 0);
            }
        }
        if (bad) {
#pragma unroll
            for (int ct = 0; ct < CT; ct++)
                if (seen[ct] & bad)
#pragma unroll
                    for (int i = 0; i < NDB; i++)
#pragma unroll
                        for (int e = 0; e < 4; e++) o[ct][i][e] = __builtin_nanf("");
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    // ---- the waves' states meet in LDS, over the V tiles
    __syncthreads();
    float* const ored = reinterpret_cast<float*>(smem);      // [FW][nr][D]
#pragma unroll
    for (int ct = 0; ct < CT; ct++) {
        const int lr = 16 * ct + n16;
        l[ct] = sum_quarters(l[ct]);
        if (lr >= nr) continue;
#pragma unroll
        for (int db = 0; db < NDB; db++) *reinterpret_cast<f32x4*>(ored + (wave * nr + lr) * D + 16 * db + 4 * q4) = o[ct][db];
        if (q4 == 0) {
            gst[wave][lr][0] = m[ct];
            gst[wave][lr][1] = l[ct];
        }
    }
    __syncthreads();
    // one share: the output; more: its state, [(sequence, kv head)][share][R rows][D] outputs, then [..][R] (max, sum)
    const size_t slot = (((size_t)b * a.nkv + hk) * a.nsplit + part) * R + row0;
    float* const po = a.part + slot * D;
    float2* const pst = reinterpret_cast<float2*>(a.part + (size_t)a.B * a.nkv * a.nsplit * R * D) + slot;
    for (int idx = tid; idx < nr * (D / 2); idx += 64 * FW) {
        const int lr = idx / (D / 2), d = 2 * (idx % (D / 2));
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < FW; w++) M = fmaxf(M, gst[w][lr][0]);
        const float Mb = M == -INFINITY ? 0.f : M;
        float x = 0.f, y = 0.f, lt = 0.f;
#pragma unroll
        for (int w = 0; w < FW; w++) {
            const float sc = exp2_hw((gst[w][lr][0] - Mb) * LOG2E), lw = gst[w][lr][1];
            const float2 v = *reinterpret_cast<const float2*>(ored + (w * nr + lr) * D + d);
            // (a wave whose scores were NaN alone has the maximum -inf and a NaN sum)
            const bool on = sc != 0.f || lw != lw;
            x += on ? (lw != lw ? lw : sc * v.x) : 0.f;
            y += on ? (lw != lw ? lw : sc * v.y) : 0.f;
            lt += on ? (lw != lw ? lw : sc * lw) : 0.f;
        }
        if (a.nsplit == 1) {
            const int row = row0 + lr;
            const float u = lt == 0.f ? 0.f : x / lt, v = lt == 0.f ? 0.f : y / lt;
            *reinterpret_cast<uint32_t*>(a.out + (((size_t)b * a.N + row / r) * a.nq + hk * r + row % r) * D + d) =
                (uint32_t)bf16_bits_rne(u) | (uint32_t)bf16_bits_rne(v) << 16;
        } else {
            *reinterpret_cast<float2*>(po + 2 * idx) = float2{x, y};
            if (d == 0) pst[lr] = float2{M, lt};
        }
    }
}

// Merges the shares of a row: one block each, wave w takes shares w, w + 4, ..;
// their order does not depend on timing.
template <int D>
__global__ void __launch_bounds__(256) kv_attn_few_merge_kernel(KvAttnArgs a) {
    constexpr int CB = 4, E = D / 64;        // shares of a wave requested together, dims of a lane
    __shared__ float sm[4][2 + E][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hk = blockIdx.x, row = blockIdx.y, b = blockIdx.z, n = a.nsplit, r = a.nq / a.nkv, R = a.N * r;
    const size_t slot = ((size_t)b * a.nkv + hk) * n * R + row;
    const float* const po = a.part + slot * D + E * lane;
    const float2* const pst = reinterpret_cast<const float2*>(a.part + (size_t)a.B * a.nkv * n * R * D) + slot;
    float M = -INFINITY, L = 0.f, acc[E] = {};
    auto join = [&](float m2, float l2, const float (&v)[E]) __attribute__((always_inline)) {
        const float Mn = fmaxf(M, m2), Mb = Mn == -INFINITY ? 0.f : Mn;
        const float keep = exp2_hw((M - Mb) * LOG2E), w = l2 != l2 ? 1.f : exp2_hw((m2 - Mb) * LOG2E);   // (NaN stays)
        L = L * keep + w * l2;
#pragma unroll
        for (int e = 0; e < E; e++) acc[e] = acc[e] * keep + (w == 0.f ? 0.f : w * v[e]);
        M = Mn;
    };
    for (int c0 = wave; c0 < n; c0 += 4 * CB) {
        float2 s[CB];
        float v[CB][E];
#pragma unroll
        for (int c = 0; c < CB; c++) {
            const size_t o = (size_t)min(c0 + 4 * c, n - 1) * R;
            s[c] = pst[o];
#pragma unroll
            for (int e = 0; e < E; e++) v[c][e] = po[o * D + e];
        }
#pragma unroll
        for (int c = 0; c < CB; c++)
            if (c0 + 4 * c < n) join(s[c].x, s[c].y, v[c]);
    }
    sm[wave][0][lane] = M;
    sm[wave][1][lane] = L;
#pragma unroll
    for (int e = 0; e < E; e++) sm[wave][2 + e][lane] = acc[e];
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < 4; w++) {
        float v[E];
#pragma unroll
        for (int e = 0; e < E; e++) v[e] = sm[w][2 + e][lane];
        join(sm[w][0][lane], sm[w][1][lane], v);
    }
    uint16_t* const out = a.out + (((size_t)b * a.N + row / r) * a.nq + hk * r + row % r) * D + E * lane;
    if constexpr (E == 2) {
        const float x = L == 0.f ? 0.f : acc[0] / L, y = L == 0.f ? 0.f : acc[1] / L;
        *reinterpret_cast<uint32_t*>(out) = (uint32_t)bf16_bits_rne(x) | (uint32_t)bf16_bits_rne(y) << 16;
    } else {
        *out = bf16_bits_rne(L == 0.f ? 0.f : acc[0] / L);
    }
}

// ---------------------------------------------------------------- many rows

constexpr int MW = 8;            // waves per block
constexpr int MROWS = 32 * MW;   // rows per block
constexpr int MKT = 64;          // keys per stage

// One block: 256 rows of a (sequence, kv head), 32 to a wave, and a part of the
// stages of 64 keys that they see.  Every thread takes 16-byte pieces of the next stage's K and V through
// registers into LDS, in rows whose pieces are swizzled so that the operand reads of K, and the transposing reads
// that take V^T, meet no bank twice.  Scores are formed transposed, S^T =
// K Q^T on the 32x32x16 MFMA, with the keys of a tile in an order (bits 2 and 3 of the row index
// swapped) that leaves the weights in the operand layout of P^T.  A lane owns one row: the
// online softmax needs a lane exchange only when a maximum moves, which it does when a
// score passes it by more than 8 (log2 units).  The two halves of the block's waves run half
// a stage apart: one multiplies while the other does its softmax.
template <int D>
constexpr int M_NREG = 2 + 16 * (D / 32);    // floats of a lane's state: maximum, sum, output

__device__ __forceinline__ int key_perm(int x) { return (x & ~12) | (x & 4) << 1 | (x & 8) >> 1; }   // swap bits 2 and 3

// What is common to the rows of a block (and a merge).
struct ManyTile {
    int b, hk, q, ctx;       // sequence, kv head, row tile, context
    KeyTiles kt;
    int end, high_min, low_max, n;   // n: parts of the tile
};
__device__ __forceinline__ ManyTile many_tile(const KvAttnArgs& a, int unit, int q) {
    ManyTile t;
    t.b = unit / a.nkv;
    t.hk = unit % a.nkv;
    t.q = q;
    t.ctx = min(a.ctx_lens ? a.ctx_lens[t.b] : a.ctx_base, a.max_ctx);
    const int r = a.nq / a.nkv, R = a.N * r;
    const int i0 = q * MROWS / r, i1 = (min((q + 1) * MROWS, R) - 1) / r;
    t.end = t.ctx < 0 ? -1 : a.tree ? t.ctx + a.N - 1 : t.ctx + i1;
    t.high_min = a.tree ? t.ctx - 1 : t.ctx + i0;
    t.low_max = window_low(a.tree ? t.ctx + a.N - 1 : t.ctx + i1, a.window);
    t.kt = key_tiles<MKT>(window_low(a.tree ? t.ctx : t.ctx + i0, a.window), t.end, a.sinks);
    t.n = max(1, min(a.nsplit, t.kt.n));
    return t;
}

template <int D>
__global__ void __launch_bounds__(64 * MW) kv_attn_many_kernel(KvAttnArgs a) {
    constexpr int NS = D / 32, NF = D / 16, NCH = D / 8, NL = MKT * NCH / (64 * MW);     // pieces per thread of K (of V)
    constexpr int STB = MKT * D * 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char* const Ks = smem;                          // [2 stages][64 keys][D]
    unsigned char* const Vs = smem + 2 * STB;
    u64* const vbad = reinterpret_cast<u64*>(smem + 4 * STB);   // [4] keys of V that are not finite, by stage % 4
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, c = lane & 31;
    const int units = a.B * a.nkv, unit = blockIdx.x % units, rest = blockIdx.x / units;
    const int r = a.nq / a.nkv, R = a.N * r, nqt = (R + MROWS - 1) / MROWS;
    const int part = rest % a.nsplit;
    const ManyTile mt = many_tile(a, unit, nqt - 1 - rest / a.nsplit);       // (the last, longest ones first)
    if (part >= mt.n) return;
    const int st0 = (int)((long long)mt.kt.n * part / mt.n), st1 = (int)((long long)mt.kt.n * (part + 1) / mt.n);
    const long long base = mt.b * a.stride_b + mt.hk * a.stride_h;
    const uint16_t* const kc = a.k + base;
    const uint16_t* const vc = a.v + base;
    const uint32_t ss = (uint32_t)a.stride_s;

    // piece j of this thread: row j 64 MW / NCH + tid / NCH, chunk tid % NCH
    constexpr int LROWS = 64 * MW / NCH;
    const int lrow = tid / NCH, lch = tid % NCH;
    auto kswz = [](int row) { return D == 128 ? row & 15 : row >> 1 & 7; };
    auto vswz = [](int row) { return D == 128 ? 4 * (row & 3) : 4 * (row >> 1 & 1); };
    u32x4 kr[NL], vr[NL];
    auto load = [&](u32x4 (&x)[NL], const uint16_t* src, int st) __attribute__((always_inline)) {
        const int kb = tile_at(mt.kt, st) * MKT, lim = mt.end - kb;      // (keys past the last one read that one)
        const uint16_t* p = src + kb * a.stride_s;
#pragma unroll
        for (int j = 0; j < NL; j++) x[j] = *reinterpret_cast<const u32x4*>(p + (uint32_t)min(j * LROWS + lrow, lim) * ss + lch * 8);
    };
    // some row of the block does not see some key of the stage
    auto mixed = [&](int st) {
        const int kb = tile_at(mt.kt, st) * MKT;
        return kb + MKT - 1 > mt.high_min || (kb < mt.low_max && kb + MKT > a.sinks);
    };
    auto store_k = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NL; j++) {
            const int row = j * LROWS + lrow;
            *reinterpret_cast<u32x4*>(Ks + (s & 1) * STB + row * 2 * D + ((lch ^ kswz(row)) << 4)) = kr[j];
        }
    };
    auto store_v = [&](int s) __attribute__((always_inline)) {
        if (mixed(st0 + s)) {
#pragma unroll
            for (int j = 0; j < NL; j++)
                if (not_finite(vr[j])) {
                    atomicOr(vbad + (s & 3), 1ull << (j * LROWS + lrow));
                    vr[j] = u32x4{0u, 0u, 0u, 0u};
                }
        }
#pragma unroll
        for (int j = 0; j < NL; j++) {
            const int row = j * LROWS + lrow;
            *reinterpret_cast<u32x4*>(Vs + (s & 1) * STB + row * 2 * D + ((lch ^ vswz(row)) << 4)) = vr[j];
        }
    };

    const int n = st1 - st0;
    if (n > 0) load(kr, kc, st0);
    // ---- queries: this lane's row, dims 16 f + 8 h .. + 7 of every fragment f
    const int row = mt.q * MROWS + wave * 32 + c, rowc = min(row, R - 1);
    const uint16_t* qp = a.q + (((size_t)mt.b * a.N + rowc / r) * a.nq + mt.hk * r + rowc % r) * D + 8 * h;
    bf16x8 qf[NF];
#pragma unroll
    for (int f = 0; f < NF; f++) qf[f] = *reinterpret_cast<const bf16x8*>(qp + 16 * f);
    const RowView view = row_view(a, mt.b, rowc / r, mt.ctx);
    const bool active = mt.q * MROWS + wave * 32 < R;
    const float sl = a.scale * LOG2E;
    // stages that none of the wave's rows sees (of a chain: their first and last positions)
    const int wi0 = min(mt.q * MROWS + wave * 32, R - 1) / r, wi1 = min(mt.q * MROWS + wave * 32 + 31, R - 1) / r;
    const int w_low = window_low(a.tree ? mt.ctx : mt.ctx + wi0, a.window), w_high = a.tree ? mt.end : mt.ctx + wi1;
    const int w_low_max = window_low(a.tree ? mt.ctx + a.N - 1 : mt.ctx + wi1, a.window), w_high_min = a.tree ? mt.ctx - 1 : mt.ctx + wi0;
    auto on = [&](int st) {
        const int kb = tile_at(mt.kt, st) * MKT;
        return active && kb <= w_high && (kb + MKT > w_low || kb < a.sinks);
    };

    f32x16 o[NS];
#pragma unroll
    for (int i = 0; i < NS; i++) o[i] = f32x16{};
    float m = -INFINITY, l = 0.f;

    if (n > 0) {
        if (tid < 4) vbad[tid] = 0;
        store_k(0);
        if (n > 1) load(kr, kc, st0 + 1);
        load(vr, vc, st0);
        __syncthreads();
        int next = 0;                                        // K of stage next + 1 and V of stage next go to LDS
        auto store_next = [&]() __attribute__((always_inline)) {
            if (next + 1 < n) store_k(next + 1);
            if (next < n) store_v(next);
            if (next + 2 < n) load(kr, kc, st0 + next + 2);
            if (next + 1 < n) load(vr, vc, st0 + next + 1);
            next++;
        };
        if (wave >= MW / 2) {                                // half a stage behind: vector work where the others multiply
            store_next();
            __syncthreads();
        }
        const int krow = key_perm(c);
        bf16x8 pf[4];
#pragma clang loop unroll(disable)
        for (int s = 0; s <= n; s++) {
            // ---- matrix half: scores of stage s, output of stage s - 1
            f32x16 sc[2];
            const bool now = s < n && on(st0 + s);
            if (now) {
                const unsigned char* K = Ks + (s & 1) * STB;
                sc[0] = f32x16{};
                sc[1] = f32x16{};
#pragma unroll
                for (int f = 0; f < NF; f++)
#pragma unroll
                    for (int t = 0; t < 2; t++) {
                        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(K + (32 * t + krow) * 2 * D + (((2 * f + h) ^ kswz(krow)) << 4));
                        sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[f], sc[t], 0, 0, 0);
                    }
            }
            if (s > 0 && on(st0 + s - 1)) {
                const __bf16* V = reinterpret_cast<const __bf16*>(Vs + (s - 1 & 1) * STB);
                // this lane's 8 keys 16 ks + 8 h .. + 7, dim 32 i + c, by two transposing reads: lane x of a 16-lane group
                // points at key 16 ks + 8 h + x / 4 (+ 4), dims 32 i + 16 (c / 16) + 4 (x % 4) .. + 3
                const int vrow = 8 * h + ((lane & 15) >> 2), vch = 2 * (c >> 4) + ((lane & 3) >> 1);
#pragma unroll
                for (int ks = 0; ks < 4; ks++)
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        const __bf16* p0 = V + (16 * ks + vrow) * D + (((4 * i + vch) ^ vswz(vrow)) << 3) + 4 * (lane & 1);
                        const __bf16* p1 = V + (16 * ks + vrow + 4) * D + (((4 * i + vch) ^ vswz(vrow + 4)) << 3) + 4 * (lane & 1);
                        const i16x4 v0 = lds_read_tr16(p0), v1 = lds_read_tr16(p1);
                        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[ks], o[i], 0, 0, 0);
                    }
                const u64 bad = vbad[s - 1 & 3];
                if (bad != 0 && (seen_bits(a, view, mt.ctx, tile_at(mt.kt, st0 + s - 1) * MKT) & bad) != 0) {
#pragma unroll
                    for (int i = 0; i < NS; i++)
#pragma unroll
                        for (int e = 0; e < 16; e++) o[i][e] = __builtin_nanf("");
                }
            }
            if (s == n) break;
            __syncthreads();
            // ---- vector half: weights of stage s, the next tiles
            if (tid == 0) vbad[s + 1 & 3] = 0;               // (the list of stage s - 3)
            if (now) {
                const int kb = tile_at(mt.kt, st0 + s) * MKT;
                float p[32];
#pragma unroll
                for (int e = 0; e < 32; e++) p[e] = sc[e / 16][e % 16];
                if (kb + MKT - 1 > w_high_min || (kb < w_low_max && kb + MKT > a.sinks)) {
                    const u64 seen = seen_bits(a, view, mt.ctx, kb) >> (8 * h);
                    const uint32_t lo = (uint32_t)seen, hi = (uint32_t)(seen >> 32);
#pragma unroll
                    for (int e = 0; e < 32; e++)
                        p[e] = (e < 16 ? lo : hi) >> (16 * (e % 16 / 8) + e % 8) & 1 ? p[e] : -INFINITY;
                }
                float mt2 = fmaxf(p[0], p[1]);
#pragma unroll
                for (int e = 2; e < 32; e++) mt2 = fmaxf(mt2, p[e]);
                if (__builtin_amdgcn_ballot_w64(mt2 * sl > m + 8.f) != 0) {
                    const float mn = fmaxf(m, max_halves(mt2) * sl);
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
                    const bf16x2 w = __builtin_convertvector(f32x2{x, y}, bf16x2);
                    pf[e / 8][e % 8] = w[0];
                    pf[e / 8][e % 8 + 1] = w[1];
                }
                l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
            }
            store_next();
            __syncthreads();
        }
        if (wave < MW / 2) __syncthreads();
    }
    const float lt = l + __shfl_xor(l, 32, 64);
    if (mt.n == 1) {
        if (row >= R) return;
        const float inv = lt == 0.f ? 0.f : 1.f / lt;
        uint16_t* const out = a.out + (((size_t)mt.b * a.N + row / r) * a.nq + mt.hk * r + row % r) * D + 4 * h;
#pragma unroll
        for (int i = 0; i < NS; i++)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<uint2*>(out + i * 32 + 2 * e) =
                    uint2{(uint32_t)bf16_bits_rne(o[i][e] * inv) | (uint32_t)bf16_bits_rne(o[i][e + 1] * inv) << 16,
                          (uint32_t)bf16_bits_rne(o[i][e + 2] * inv) | (uint32_t)bf16_bits_rne(o[i][e + 3] * inv) << 16};
        return;
    }
    if (!active) return;
    float* pp = a.part + ((size_t)blockIdx.x * MW + wave) * M_NREG<D> * 64 + lane;       // state of this part
    pp[0] = m;
    pp[64] = l;
#pragma unroll
    for (int i = 0; i < NS; i++)
#pragma unroll
        for (int e = 0; e < 16; e++) pp[(2 + i * 16 + e) * 64] = o[i][e];
}

// Merges the parts of the row tiles that have more than one: block (row tile and unit, 32-dim slice), thread
// (wave, lane) the lane's registers of the slice, part after part in key order.
template <int D>
__global__ void __launch_bounds__(64 * MW) kv_attn_many_merge_kernel(KvAttnArgs a) {
    constexpr int CB = 4;                                    // parts requested together
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, c = lane & 31, i = blockIdx.y;
    const int units = a.B * a.nkv, unit = blockIdx.x % units, back = blockIdx.x / units;
    const int r = a.nq / a.nkv, R = a.N * r, nqt = (R + MROWS - 1) / MROWS;
    const ManyTile mt = many_tile(a, unit, nqt - 1 - back);
    const int row = mt.q * MROWS + wave * 32 + c;
    if (mt.n == 1 || mt.q * MROWS + wave * 32 >= R) return;
    float M = -INFINITY, L = 0.f, acc[16] = {};
    for (int p0 = 0; p0 < mt.n; p0 += CB) {
        float mc[CB], lc[CB], v[CB][16];
#pragma unroll
        for (int j = 0; j < CB; j++) {
            const size_t block = (size_t)(back * a.nsplit + min(p0 + j, mt.n - 1)) * units + unit;
            const float* pp = a.part + (block * MW + wave) * M_NREG<D> * 64 + lane;
            mc[j] = pp[0];
            lc[j] = pp[64];
#pragma unroll
            for (int e = 0; e < 16; e++) v[j][e] = pp[(2 + i * 16 + e) * 64];
        }
        float Mn = M;
#pragma unroll
        for (int j = 0; j < CB; j++)
            if (p0 + j < mt.n) Mn = fmaxf(Mn, mc[j]);
        const float Mb = Mn == -INFINITY ? 0.f : Mn, s0 = exp2_hw(M - Mb);
        L *= s0;
#pragma unroll
        for (int e = 0; e < 16; e++) acc[e] *= s0;
#pragma unroll
        for (int j = 0; j < CB; j++) {
            if (p0 + j >= mt.n) break;
            const float s = lc[j] != lc[j] ? 1.f : exp2_hw(mc[j] - Mb);      // (NaN stays)
            L += s * lc[j];
#pragma unroll
            for (int e = 0; e < 16; e++) acc[e] += s * v[j][e];
        }
        M = Mn;
    }
    const float lt = L + __shfl_xor(L, 32, 64);
    if (row >= R) return;
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    uint16_t* const out = a.out + (((size_t)mt.b * a.N + row / r) * a.nq + mt.hk * r + row % r) * D + i * 32 + 4 * h;
#pragma unroll
    for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<uint2*>(out + 2 * e) =
            uint2{(uint32_t)bf16_bits_rne(acc[e] * inv) | (uint32_t)bf16_bits_rne(acc[e + 1] * inv) << 16,
                  (uint32_t)bf16_bits_rne(acc[e + 2] * inv) | (uint32_t)bf16_bits_rne(acc[e + 3] * inv) << 16};
}

}  // namespace

constexpr int kFewRows = 64;             // at most, for the kernel of few rows
constexpr int kFewBlocks = 512, kManyParts = 512;   // of a call that has more than one share (part) per tile

// Slots from the lowest that a row may see to the last, of the longest sequence.
static KeyTiles longest(const KvAttnShape& s, int kt) {
    const int end = s.max_ctx + s.N - 1, low = window_low(s.max_ctx, s.window);
    return kt == FKT ? key_tiles<FKT>(low, end, s.sinks) : key_tiles<MKT>(low, end, s.sinks);
}

KvAttnPlan kv_attn_plan(const KvAttnShape& s) {
    KvAttnPlan p;
    const long long R = (long long)s.N * s.r, pairs = (long long)s.B * s.nkv;
    p.few = R <= kFewRows;
    if (p.few) {
        p.ct = R <= 16 ? 1 : 2;
        const long long tiles = longest(s, FKT).n, blocks = pairs * ((R + 16 * p.ct - 1) / (16 * p.ct));
        const long long n = tiles < 32 ? 1 : std::min((p.ct == 1 ? 2 : 1) * kCus / blocks, (tiles + FW - 1) / FW);
        p.nsplit = (int)std::max(1ll, n);
        return p;
    }
    const long long stages = longest(s, MKT).n, blocks = pairs * ((R + MROWS - 1) / MROWS);
    const long long n = std::min(2 * kCus / blocks, stages / 4);
    p.nsplit = (int)std::max(1ll, n);
    return p;
}

size_t kv_attn_part_bytes(const KvAttnShape& s, const KvAttnPlan& p) {
    const size_t R = (size_t)s.N * s.r, pairs = (size_t)s.B * s.nkv;
    if (p.nsplit == 1) return 0;
    if (p.few) return pairs * p.nsplit * R * (s.d + 2) * 4;
    return pairs * p.nsplit * ((R + MROWS - 1) / MROWS) * MROWS * (s.d + 4) * 4;
}

// (either kernel's; a product of what grows, and a constant)
size_t kv_attn_part_bound(const KvAttnShape& s) {
    const size_t R = (size_t)s.N * s.r, pairs = (size_t)s.B * s.nkv, slots = (size_t)s.max_ctx + s.N;
    const size_t few = std::min<size_t>(pairs * R * (slots / FKT + 2), (size_t)kFewBlocks * 32);
    const size_t many = std::min<size_t>(pairs * ((R + MROWS - 1) / MROWS) * (slots / MKT + 2), kManyParts) * MROWS;
    return std::max<size_t>(256, std::max(few, many) * (s.d + 4) * 4);
}

template <int D, int CT>
static int launch_few(const KvAttnArgs& a, hipStream_t stream) {
    const int R = a.N * (a.nq / a.nkv), tiles = (R + 16 * CT - 1) / (16 * CT);
    const size_t lds = (size_t)FW * std::max(FKT * D * 2, std::min(R, 16 * CT) * D * 4);
    static LdsLimit lim;
    if (ensure_lds_limit(lim, (const void*)kv_attn_few_kernel<D, CT>, lds)) return -1;
    hipLaunchKernelGGL((kv_attn_few_kernel<D, CT>), dim3(a.nkv * tiles, a.nsplit, a.B), dim3(64 * FW), lds, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL(kv_attn_few_merge_kernel<D>, dim3(a.nkv, R, a.B), dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D>
static int launch_many(const KvAttnArgs& a, hipStream_t stream) {
    const int R = a.N * (a.nq / a.nkv);
    const long long tiles = (long long)a.B * a.nkv * ((R + MROWS - 1) / MROWS);
    if (tiles * a.nsplit > INT_MAX) return -1;
    const size_t lds = (size_t)4 * MKT * D * 2 + 4 * 8;
    static LdsLimit lim;
    if (ensure_lds_limit(lim, (const void*)kv_attn_many_kernel<D>, lds)) return -1;
    hipLaunchKernelGGL(kv_attn_many_kernel<D>, dim3((unsigned)(tiles * a.nsplit)), dim3(64 * MW), lds, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL(kv_attn_many_merge_kernel<D>, dim3((unsigned)tiles, D / 32), dim3(64 * MW), 0, stream, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_attn(const KvAttnArgs& args, size_t part_bytes, hipStream_t stream) {
    KvAttnArgs a = args;
    const KvAttnShape s{a.B, a.N, a.nkv, a.nq / a.nkv, a.d, a.max_ctx, a.window, a.sinks};
    const KvAttnPlan p = kv_attn_plan(s);
    if (kv_attn_part_bytes(s, p) > part_bytes || (a.mask && a.N != 1)) return -1;
    a.nsplit = p.nsplit;
    if (p.few) {
        if (p.ct == 1) return a.d == 128 ? launch_few<128, 1>(a, stream) : launch_few<64, 1>(a, stream);
        return a.d == 128 ? launch_few<128, 2>(a, stream) : launch_few<64, 2>(a, stream);
    }
    if (a.mask) return -1;
    return a.d == 128 ? launch_many<128>(a, stream) : launch_many<64>(a, stream);
}

int load_kv_attn() { return load_code((const void*)kv_attn_few_kernel<128, 1>); }
