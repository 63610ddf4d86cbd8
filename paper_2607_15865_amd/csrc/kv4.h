// The 4-bit key/value cache: its device layout and the launchers of its kernels
// (kv4.hip: write and read back; kv4_attn.hip: attention).
//
// Per token and kv head the head's D dims (64 or 128) are cut into NS = D / 32
// groups of 32.  A group holds
//     lo = min x,  s = fp16((max x - lo) / 15),  c = min(15, floor((x - lo) / s + 1/2))
// of its values x (taken as fp16), c = 0 where s = 0, and stands for lo + s c.
// A group with a value that has no fp16 value (NaN, an infinity, beyond 65504)
// holds s = lo = NaN.
//
// K and V are separate buffers, [batch][kv head][tile] of tiles of 32 tokens
// (tokens past max_seq in the last tile are padding).  A tile is 32 D / 2
// bytes of codes, then NS * 128 bytes of parameters: per group 32 fp16 scales
// (one per token), then 32 fp16 offsets lo.  The codes lie in the order in which
// the attention's 16x16x32 MFMAs take them, so that a wave reads a tile in
// whole 1 KB lines, lane by lane, and unpacks in registers:
//   K: word s of lane (n16, q4) of score tile t at word (t 64 + q4 16 + n16) NS + s:
//      dims 32 s + 8 q4 .. + 7 of token 8 (n16 / 4) + 4 t + n16 % 4;
//   V: word i of lane (n16, q4) of half hf at word (hf 64 + q4 16 + n16) 4 + i:
//      dim 16 (4 hf + i) + n16 of tokens 8 q4 .. + 7 (a word spans tokens, so
//      writing a single one replaces nibbles).
// Element e of a word's eight sits at bits 4 (e / 2) + 16 (e % 2), as in the
// weights' words.
#pragma once
#include "common.h"

constexpr int KV4_TILE = 32;             // tokens per tile

__host__ __device__ constexpr int kv4_code_bytes(int d) { return KV4_TILE * d / 2; }
__host__ __device__ constexpr int kv4_tile_bytes(int d) { return kv4_code_bytes(d) + d / 32 * 128; }

// First slots of the rows of one launch, by value.
constexpr int KV4_ROWS = 64;
struct Kv4Slots {
    int32_t v[KV4_ROWS];
};

struct Kv4StoreArgs {
    uint8_t* k;              // caches (byte strides)
    uint8_t* v;
    long long stride_b, stride_h;
    uint16_t* k_x;           // bf16 rows: written into the cache, or read out of it
    uint16_t* v_x;
    long long x_b, x_t, x_h; // strides of the bf16 rows, in elements
    const int32_t* slots_dev;   // first slots on the device, or null: in slots
    Kv4Slots slots;
    int max_seq, B, T, nkv, d;
    int* err;                // raised with W4_FLAG_F16_RANGE by a group without fp16 values, or null
};
int launch_kv4_append(const Kv4StoreArgs& a, hipStream_t stream);
int launch_kv4_read(const Kv4StoreArgs& a, hipStream_t stream);

struct Kv4AttnArgs {
    const uint16_t* q;       // bf16 [rows][nq][d]
    const uint8_t* k;
    const uint8_t* v;
    long long stride_b, stride_h;   // bytes; stride_b 0: the rows are tokens of one sequence
    const int32_t* ctx_lens; // [rows] device: row b sees slots 0 .. ctx_lens[b]; null: 0 .. ctx_base + b
    int ctx_base;
    int max_ctx;             // the longest context
    const float* mask;       // fp32 [rows][max_seq] or null
    int max_seq;
    void* out;               // [rows][nq][d]: bf16, or (out_f16) bf16 values held as fp16
    int out_f16;
    int rows, nq, nkv, d;
    float scale;             // of the scores
    int nsplit;              // decode: shares of a (row, kv head)'s tiles
    float* part;             // decode: share states (nsplit > 1), [rows nkv][nsplit] of r (d + 2) floats; prefill:
                             // plan.part_bytes
    long long pf_units;      // prefill, set by the launcher: stages of one kv head's row tiles
    int pf_chunk;            // and most stages of a part (0: equal runs)
    int r, per;              // set by the launcher: nq / nkv; decode: tiles per share
    int* err;                // raised with W4_FLAG_F16_RANGE (out_f16), or null
};
int kv4_decode_shares(int rows, int nkv, int r, int d, int max_ctx);      // nsplit
size_t kv4_decode_part_bound(int rows, int nkv, int r, int d, int max_ctx);
int launch_kv4_decode(const Kv4AttnArgs& a, hipStream_t stream);
// Prefill: rows queries of one sequence after ctx_base tokens (part: part_bytes).
struct Kv4PrefillPlan {
    long long units = 0;     // stages of one kv head's row tiles
    int blocks = 0, chunk = 0;   // chunk: parts of so many stages at most, a block each; 0: equal runs
    bool merge = false;
    bool single = false;     // the queries are rows of the decode kernel (then nothing above)
    size_t part_bytes = 0;   // grows with T and hist
};
Kv4PrefillPlan kv4_prefill_plan(int T, int hist, int nkv, int r, int d);
int launch_kv4_prefill(const Kv4AttnArgs& a, hipStream_t stream);

int load_kv4();
int load_kv4_attn();
