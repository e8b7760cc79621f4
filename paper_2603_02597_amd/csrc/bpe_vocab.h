// What a vocabulary handle holds (made in bpe_vocab.hip), for the kernels that walk through its tokens.
#pragma once
#include "bpe_common.h"

typedef uint32_t Record __attribute__((ext_vector_type(4)));

struct bpe_vocab {
    bpe_vocab_info_t info;
    void *device_mem;      // one allocation: tok | tok_out | out_of | int_of | pool
    const Record *tok;      // [n_ids] by internal id: see kInlineBytes
    const Record *tok_out;  // [n_out] by output id, or nullptr
    const int32_t *out_of, *int_of;
    int64_t token_bytes;    // of all expansions
    const uint8_t *pool;
    int32_t n_out;
    int device;
};

namespace bpe {

// What a token stands for, as one 16-byte word: x = length in bytes (0 = id not in use); the bytes
// themselves in y, z, w if they are at most kInlineBytes, else y = their offset in the pool (a
// multiple of 4).  Word-like tokens (up to 12 bytes) are one gather instead of an {offset, length}
// and, after it, one of the pool per four bytes: a gather of 64 unrelated lines costs the texture
// path 64 line look-ups whatever its width.  2.1 M tokens (13.5 MB): 24.0 us with the two gathers,
// 22.5 with the records (and the assembly moved in front of the look-back).
constexpr uint32_t kInlineBytes = 12;

}  // namespace bpe
