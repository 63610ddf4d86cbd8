// Attention over the bf16 cache with a window, sinks and draft trees
// (kv_attn.hip), and the draft trees' own steps (tree.hip).
#pragma once
#include "common.h"

// One launch: B sequences of N queries each.  Query i of sequence b stands at
// position ctx + i (a chain: slots 0 .. ctx + i, its own among them), or, with
// `tree`, at pos[b][i], where it sees slots 0 .. ctx - 1 and those slots ctx + a
// whose bit its mask has.
struct KvAttnArgs {
    const uint16_t* q;       // bf16 [B][N][nq][d]
    const uint16_t* k;       // caches (strides in elements)
    const uint16_t* v;
    long long stride_b, stride_h, stride_s;
    const int32_t* ctx_lens; // [B] device (below 0: zero rows), or null: ctx_base
    int ctx_base;
    int max_ctx;             // the largest
    int window, sinks;       // window INT_MAX: none
    const float* mask;       // fp32 [B][max_seq], added to the scores, or null (chains of one query)
    int max_seq;
    const unsigned long long* tree;   // [B][N][words], or null
    const int32_t* pos;      // [B][N]; null: no window
    int words;
    uint16_t* out;           // [B][N][nq][d]: bf16, or (out_f16) bf16 values held as fp16
    int out_f16;
    int* err;                // raised with W4_FLAG_F16_RANGE (out_f16), or null
    int B, N, nq, nkv, d;
    float scale;             // of the scores
    int nsplit;              // set by the launcher: shares of a row tile's keys,
    int whole, rest;         // many rows: of the tiles behind the first `whole`, `rest` in number
    float* part;             // their states
};
// What a plan depends on (r: query heads per kv head).
struct KvAttnShape {
    int B, N, nkv, r, d, max_ctx, window, sinks;
    bool tree, mask;
};
struct KvAttnPlan {
    bool few = false;        // the kernel of few rows
    bool halves = false;     // many rows: tiles of 128, two waves for the keys of each
    int nsplit = 1;          // shares of a row tile's keys,
    int whole = 0;           // many rows: except for so many tiles
};
KvAttnPlan kv_attn_plan(const KvAttnShape& s);
size_t kv_attn_part_bytes(const KvAttnShape& s, const KvAttnPlan& p);
size_t kv_attn_part_bound(const KvAttnShape& s);     // of any plan, window and sinks; grows with B, N and max_ctx
int launch_kv_attn(const KvAttnArgs& a, size_t part_bytes, hipStream_t stream);

struct KvSlotArgs {
    long long stride_b, stride_h, stride_s;
    const int32_t* ctx_lens; // [B]
    int max_seq, B, T, nkv, d;
};
// T new rows per sequence, bf16 [B][T][nkv][d], into slots ctx_lens[b] + t.
int launch_kv_append_step(const KvSlotArgs& a, uint16_t* k, uint16_t* v, const uint16_t* k_new, const uint16_t* v_new,
                          hipStream_t stream);
// The rows of a path (T = N) moved together, in up to KEEP_CACHES pairs of caches.
constexpr int KEEP_CACHES = 64;
struct KeepCaches {
    uint16_t* p[2 * KEEP_CACHES];
};
int launch_kv_keep(const KvSlotArgs& a, const KeepCaches& c, int ncaches, const int32_t* path, const int32_t* n_path,
                   hipStream_t stream);

struct TreePlanArgs {
    const int32_t* parents;
    const int32_t* ctx_lens;
    int B, N, window, sinks; // window INT_MAX: none
    unsigned long long* mask;
    int32_t* pos;
};
int launch_tree_plan(const TreePlanArgs& a, hipStream_t stream);

struct TreeAcceptArgs {
    const int32_t* parents;
    const int32_t* tokens;
    const int32_t* picks;
    int B, N;
    int32_t* path;
    int32_t* n_path;
    int32_t* next;
};
int launch_tree_accept(const TreeAcceptArgs& a, hipStream_t stream);

int load_kv_attn();
int load_tree();
