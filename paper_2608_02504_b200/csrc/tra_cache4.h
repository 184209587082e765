// The cache of 4 bits: where a row's codes lie, and the launches that write, read and attend over it.
//
// A row is one (key/value head, token): d / 2 bytes of codes and, per group of 32 channels, a step and a lowest value.  Rows of a head
// follow one another, so that a tile of keys is one run of bytes.  Inside a row the codes lie as the products of tra_cache4_rows.cuh
// take them, so that eight codes of a 32-bit word become four operand registers by one mask each.  G = d / 32 groups:
//   keys  : word G t + j, t = 0 .. 3, holds of group j the channels 32 j + 8 (n % 4) + 2 t + n / 4 in nibbles n = 0 .. 7 (a product's
//           thread t of four holds channels 2 t and 2 t + 1 of every eight);
//   values: word (G / 2) g + w, g = 0 .. 7, holds the channels 64 w + 8 n + g (thread g of eight holds channel g of every eight).
// Steps and lowest values: [G] steps, then [G] lowest values, in the tensors' type.
#pragma once
#include "tra_packed.h"

constexpr int kCacheGroup = 32;

struct tra_cache4_launch {
  tra_packed_launch a;         // (its K and V are not used: the maps stay empty)
  const uint8_t *k, *v;        // [kv_heads][tokens][d / 2]
  const void *k_step, *v_step; // [kv_heads][tokens][2][d / 32]
  int row_tiles;               // tiles of 16 rows per (sequence, key/value head)
};

int tra_cache4_rows(const tra_packed_ctx& c, const tra_cache4_launch& a, int chunk, bool clustered);

// Joins the parts of a split launch (tra_packed.cu).
int tra_packed_join(const tra_packed_ctx& c, const tra_packed_launch& p);
// Checks what every attention call shares and fills the launch; a->k and a->v are looked at when `keys`.
int tra_packed_begin(const tra_packed_t* h, const tra_packed_args_t* a, bool keys, tra_packed_launch* p);
// tra_packed_attn over keys and values that were read back, at more than 16 rows per key/value head (see FwdCfg).  fp16 tensors: K and V of twice
// the heads, rounded elements, then what rounding took from them.  bf16: Q, K and V are fp16, with their multiples' q_mul and kv_top.
int tra_packed_attn_read_back(const tra_packed_t* h, const tra_packed_args_t* a, const float* q_mul, const uint32_t* kv_top, void* workspace,
                              size_t workspace_bytes, void* stream);
// Keys that `tokens` queries walk at most.
int tra_packed_longest_axis(const tra_packed_t* h, int max_k, int tokens);
