// Paged KV cache in DialectFP4: storage, index arithmetic and the views that the kernels take.
//
// The pool is [pages][kv_heads][page_tokens / 32] records of 35 * head_dim bytes.  A record holds one chunk of 32
// tokens of one KV head: its keys as nb = head_dim / 32 tiles of 32 rows (tokens) x 32 dimensions, its values as nb
// tiles of 32 rows (channels) x 32 tokens.  A row of a tile is one block of the format (scale, dialect id, 32 codes),
// so both operands of attention have the block along their multiplication dimension (appendix "Quantization
// Dimension").  Parts in order: key codes, value codes (16 d bytes each), key scales, value scales (d each), key ids,
// value ids (d / 2 each): everything a warp needs of 32 tokens is one contiguous, 16-byte aligned bulk copy.
//
// Inside a tile row r = 8 j + g.  Word t (elements 8 t .. 8 t + 7) of row r of tile b sits at word
// ((8 b + g) * 4 + t) * 4 + j: lane 4 g + t of a warp reads the words of its four rows as one 16-byte load, and the
// 32 lanes read 512 consecutive bytes.  Scale bytes and id nibbles sit at index (4 g + j) * nb + b, so a lane reads
// the scales of all its rows and tiles with one load too.  A token's scales and ids share no byte with another
// token's: tokens of one chunk arrive in different calls.
// Row of token 8 x + 2 y + z of a chunk in the key tiles: 8 y + 2 x + z.  With this order the probabilities that the
// score fragments hold become, after an 8 x 8 transpose, the fragments of the second product in the value words' order.
// Elements 0 .. 7 of a word sit in its nibbles 0, 2, 1, 3, 4, 6, 5, 7 as sign << 3 | index: the two elements of a
// 16-bit pair then take their signs from the same masked copy of the word (see expand_f16).
//
// The values of an unfinished chunk wait in high precision: row token % 64 of the sequence's tail
// [slots][kv_heads][64][head_dim].  64 rows keep the chunk before the newest one as well, so a step of up to 32 tokens
// can be repeated or taken back (rejected drafts).
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define BD_HD __host__ __device__ __forceinline__
#else
#define BD_HD static inline
#endif

namespace bd {
namespace pg {

constexpr int kChunk = 32;            // tokens per record
constexpr int kTailRows = 64;

struct Pool {
    uint8_t *base;
    void *tail;
    int pages, slots, kv_heads, chunks_per_page, head_dim;
    int tail_esz;                     // bytes per element of the tail
};
struct Batch {
    const int32_t *table;             // [n][ld_table] page numbers
    const int32_t *slot;              // [n]
    const int32_t *kv_len;            // [n] tokens in the cache, this step's included
    const int32_t *q_start;           // [n + 1] first row of each sequence
    int64_t ld_table;
    int n, rows, max_q, max_kv;
};
// One sequence, checked: rows [q0, q0 + t) are its tokens kv - t .. kv - 1.
struct Sequence {
    int q0, t, kv;
    bool ok;
};

BD_HD int64_t record_bytes(int d) { return 35 * (int64_t)d; }
BD_HD int64_t value_codes(int d) { return 16 * (int64_t)d; }
BD_HD int64_t key_scales(int d) { return 32 * (int64_t)d; }
BD_HD int64_t value_scales(int d) { return 33 * (int64_t)d; }
BD_HD int64_t key_ids(int d) { return 34 * (int64_t)d; }
BD_HD int64_t value_ids(int d) { return 34 * (int64_t)d + d / 2; }

// Byte of word t of row r, tile b; index of its scale byte / id nibble.
BD_HD int word_byte(int b, int r, int t) { return 4 * (((8 * b + r % 8) * 4 + t) * 4 + r / 8); }
BD_HD int entry_of(int nb, int b, int r) { return (4 * (r % 8) + r / 8) * nb + b; }
BD_HD int key_row(int token) { return 8 * (token / 2 % 4) + 2 * (token / 8) + token % 2; }
BD_HD int key_token(int row) { return 8 * (row % 8 / 2) + 2 * (row / 8) + row % 2; }

// Reads a sequence's numbers and checks them: rows inside [0, rows), at most max_q of them, 0 <= kv <= max_kv.
BD_HD Sequence sequence_of(const Batch &s, int i) {
    Sequence q;
    const int64_t a = s.q_start[i], b = s.q_start[i + 1];
    const int64_t kv = s.kv_len[i];
    q.ok = a >= 0 && b >= a && b <= s.rows && b - a <= s.max_q && kv >= 0 && kv <= s.max_kv;
    q.q0 = q.ok ? (int)a : 0;
    q.t = q.ok ? (int)(b - a) : 0;
    q.kv = q.ok ? (int)kv : 0;
    return q;
}
// Offset of the record of chunk c of sequence i, head h; -1 for a page number outside the pool.
BD_HD int64_t record_offset(const Pool &p, const Batch &s, int i, int h, int c) {
    const int page = s.table[(int64_t)i * s.ld_table + c / p.chunks_per_page];
    if (page < 0 || page >= p.pages) return -1;
    return (((int64_t)page * p.kv_heads + h) * p.chunks_per_page + c % p.chunks_per_page) * record_bytes(p.head_dim);
}
// Element offset of the tail row of `token` (slot already checked).
BD_HD int64_t tail_offset(const Pool &p, int slot, int h, int token) {
    return (((int64_t)slot * p.kv_heads + h) * kTailRows + token % kTailRows) * p.head_dim;
}

}  // namespace pg
}  // namespace bd
