// Grammars over the vocabulary: a deterministic automaton over bytes, and which tokens' bytes it can take from a state.
#include <algorithm>
#include <cstring>
#include <new>
#include <unordered_map>
#include <string>

#include "bpe_lookback.h"
#include "bpe_numeric.h"
#include "bpe_vocab.h"

struct bpe_grammar {
    bpe_grammar_info_t info;
    void *device_mem;          // one allocation: next | class_of | accepting
    const uint16_t *next;      // [n_states + 1][n_classes]: the state behind a byte of the class; state n_states is the end of the walk
    const uint8_t *class_of;   // [256]
    const uint8_t *accepting;  // [n_states]
    int device;
};

namespace bpe {

constexpr int64_t kMaxGrammarStates = 65534;

struct GrammarView {
    const uint16_t *next;
    const uint8_t *class_of, *accepting;
    int32_t n_states, n_classes;
};

struct TokenView {
    const Record *tok;
    const uint8_t *pool;
    int32_t n_tok;
};

__device__ __forceinline__ uint32_t token_byte(const Record &rec, const uint8_t *pool, uint32_t j) {
    if (rec.x > kInlineBytes) return pool[rec.y + j];
    const uint32_t w = j < 4 ? rec.y : j < 8 ? rec.z : rec.w;
    return (w >> (8 * (j & 3))) & 255u;
}

// The state behind all bytes of a token; n_states where the walk ends.
__device__ __forceinline__ uint32_t walk(const GrammarView &g, const Record &rec, const uint8_t *pool, uint32_t s) {
    for (uint32_t j = 0; j < rec.x && s < (uint32_t)g.n_states; ++j)
        s = g.next[s * (uint32_t)g.n_classes + g.class_of[token_byte(rec, pool, j)]];
    return s;
}

struct MaskParams {
    GrammarView g;
    TokenView t;
    const int32_t *states;
    int32_t n, n_vocab, end_id;
    uint32_t *masks;
    int64_t mask_stride;
};

// Few states: one lane per token, up to four states at a time, whose chains of reads are under way together.  Bound by those chains,
// a read per byte of a token, from caches (the tables and the tokens' bytes together are a few MB): 12 states of 50,257 tokens 5.5
// us, which is the call's time on the host, 64 states 12.3.
constexpr int kMaskChains = 4;
__global__ void __launch_bounds__(kGroupThreads) grammar_masks_kernel(MaskParams p) {
    const int v = blockIdx.x * kGroupThreads + threadIdx.x, n_classes = p.g.n_classes;
    const uint32_t dead = (uint32_t)p.g.n_states;
    Record rec = {0, 0, 0, 0};
    if (v < p.n_vocab && v < p.t.n_tok) rec = p.t.tok[v];
    for (int i0 = blockIdx.y * kMaskChains; i0 < p.n; i0 += gridDim.y * kMaskChains) {
        uint32_t s[kMaskChains], e[kMaskChains];
#pragma unroll
        for (int q = 0; q < kMaskChains; ++q) {
            s[q] = i0 + q < p.n ? (uint32_t)p.states[i0 + q] : dead;
            if (s[q] > dead) s[q] = dead;
            e[q] = rec.x ? s[q] : dead;
        }
        for (uint32_t j = 0; j < rec.x; ++j) {
            bool on = false;
#pragma unroll
            for (int q = 0; q < kMaskChains; ++q) on |= e[q] != dead;
            if (!on) break;
            const uint32_t c = p.g.class_of[token_byte(rec, p.t.pool, j)];
#pragma unroll
            for (int q = 0; q < kMaskChains; ++q) e[q] = p.g.next[e[q] * (uint32_t)n_classes + c];     // (the end of the walk leads to itself)
        }
#pragma unroll
        for (int q = 0; q < kMaskChains; ++q) {
            if (i0 + q >= p.n) break;
            bool on = e[q] != dead;
            if (v == p.end_id) on = s[q] != dead && p.g.accepting[s[q]] != 0;
            const uint64_t bits = __ballot(on);
            if ((v & 31) == 0 && v < p.n_vocab) p.masks[(i0 + q) * p.mask_stride + (v >> 5)] = (uint32_t)(bits >> (v & 32));
        }
    }
}

// Many states.  A workgroup takes a tile of 2,048 tokens, as strings of classes in LDS, and a share of the states; a wavefront takes
// one state after the other.  Most states let few bytes pass: one look at the transitions per class says which, and only the
// tokens behind those are walked, which the tile holds in order of their first class.  Where many tokens pass, all are walked
// in order of their ids, four per lane at a time, so that four chains of reads are under way together.  1,500 states of 50,257 tokens:
// 45 us, of which 17 lay out the tiles; bound by instructions (the bytes are 9.4 MB of masks, 2 us), with transitions in LDS.  Long tokens
// are walked by a lane each while the others wait: 1,500 states of 100,256 tokens, of up to 2,049 bytes, 2.8 ms.
constexpr int kMaskTile = 2048, kMaskThreads = 1024, kMaskWaves = kMaskThreads / kWave;
static_assert(kMaskTile == 32 * kWave, "a word of bits per lane");
constexpr int kMaskTable = 48 * 1024;            // transitions that are kept in LDS
constexpr int kMaskStates = 2048;                // states of a workgroup that are at hand at a time
// Behind up to so many classes tokens are walked class by class.  1,500 states of 50,257 tokens, as many letters lead on from each: 1 letter 17 us
// class by class and 97 all tokens, 3 letters 24 and 96, 5 letters 33 and 100, 8 letters 47 and 112, 12 letters 70 and 138, all 26 the
// same 116; a grammar of words and free text 42, with all of it class by class 74.  (So 5 is on the safe side for letters, more so for bytes
// that few tokens begin with; what counts is how many tokens those are, not how many classes.)
constexpr int kMaskFew = 5;
template <bool IN_LDS>
__global__ void __launch_bounds__(kMaskThreads) grammar_tile_masks_kernel(MaskParams p) {
    __shared__ uint32_t start[257], filled[256];
    __shared__ uint16_t order[kMaskTile];
    __shared__ __attribute__((aligned(16))) Record text[kMaskTile];       // like a token's record, with classes for bytes
    __shared__ uint32_t found[kMaskWaves][kMaskTile / 32];
    __shared__ uint8_t class_of[256];
    __shared__ uint16_t state[kMaskStates];                              // of the states at hand; `dead` for one that is not the grammar's
    __shared__ int taken;
    __shared__ __attribute__((aligned(16))) uint16_t table[IN_LDS ? kMaskTable : 1];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int first = blockIdx.x * kMaskTile, n_classes = p.g.n_classes, dead = p.g.n_states;
    const int per = (p.n + gridDim.y - 1) / gridDim.y, begin = blockIdx.y * per, end = min(begin + per, p.n);
    constexpr int kMine = kMaskTile / kMaskThreads;
    Record rec[kMine];
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
        const int v = first + q * kMaskThreads + tid;
        rec[q] = Record{0, 0, 0, 0};
        if (v < p.n_vocab && v < p.t.n_tok) rec[q] = p.t.tok[v];
    }
    if (tid < 256) {
        class_of[tid] = p.g.class_of[tid];
        filled[tid] = 0;
    }
    if constexpr (IN_LDS) {
        const int groups = ((dead + 1) * n_classes + 7) / 8;             // (the table is padded to 256 bytes)
        for (int i = tid; i < groups; i += kMaskThreads) ((uint4 *)table)[i] = ((const uint4 *)p.g.next)[i];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
        if (rec[q].x > kInlineBytes) {
            const uint32_t *w = (const uint32_t *)(p.t.pool + rec[q].y);
            rec[q].y = w[0]; rec[q].z = w[1]; rec[q].w = w[2];
        }
#pragma unroll
        for (int k = 1; k < 4; ++k) {                                    // (what lies behind a token's end is not looked at)
            const uint32_t w = rec[q][k];
            rec[q][k] = class_of[w & 255u] | (uint32_t)class_of[w >> 8 & 255u] << 8 | (uint32_t)class_of[w >> 16 & 255u] << 16 | (uint32_t)class_of[w >> 24] << 24;
        }
        if (rec[q].x) atomicAdd(&filled[rec[q].y & 255u], 1u);
        text[q * kMaskThreads + tid] = rec[q];
    }
    __syncthreads();
    if (wv == 0) {
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) { c[q] = filled[4 * lane + q]; sum += c[q]; }
        uint32_t at = (uint32_t)wave_scan_inclusive((int)sum) - sum;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            start[4 * lane + q] = filled[4 * lane + q] = at;
            at += c[q];
        }
        if (lane == 63) start[256] = at;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kMine; ++q)
        if (rec[q].x) order[atomicAdd(&filled[rec[q].y & 255u], 1u)] = (uint16_t)(q * kMaskThreads + tid);
    __syncthreads();
    const uint16_t *next = IN_LDS ? table : p.g.next;
    // class j of a token's string; beyond kInlineBytes it comes from memory
    auto class_at = [&](const Record &r, int t, uint32_t j) -> uint32_t {
        if (j < kInlineBytes) return ((j < 4 ? r.y : j < 8 ? r.z : r.w) >> (8 * (j & 3))) & 255u;
        return class_of[p.t.pool[p.t.tok[first + t].y + j]];
    };
    for (int chunk = begin; chunk < end; chunk += kMaskStates) {
        const int in_chunk = min(end - chunk, kMaskStates);
        __syncthreads();
        for (int k = tid; k < in_chunk; k += kMaskThreads) {
            const uint32_t s = (uint32_t)p.states[chunk + k];
            state[k] = (uint16_t)min(s, (uint32_t)dead);
        }
        if (tid == 0) taken = 0;
        __syncthreads();
        for (;;) {
            int i = 0;
            if (lane == 0) i = atomicAdd(&taken, 1);
            i = __builtin_amdgcn_readfirstlane(i);
            if (i >= in_chunk) break;
            const int s = __builtin_amdgcn_readfirstlane((int)state[i]);
            const bool known = s < dead;
            i += chunk;
            uint32_t bits = 0;                                               // lane w: word w of the tile's bits
            if (known) {
                int passing = 0;                                             // classes that go on and that a token begins with
                for (int c0 = 0; c0 < n_classes; c0 += kWave)
                    passing += __builtin_popcountll(__ballot(c0 + lane < n_classes && next[s * n_classes + c0 + lane] != dead && start[c0 + lane + 1] > start[c0 + lane]));
                if (passing > kMaskFew) {
                    for (int t0 = 0; t0 < kMaskTile; t0 += 4 * kWave) {
                        Record r[4];
                        int e[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            r[q] = text[t0 + q * kWave + lane];
                            e[q] = r[q].x ? s : dead;
                        }
                        auto on = [&](uint32_t j) {
                            return __ballot((j < r[0].x && e[0] != dead) || (j < r[1].x && e[1] != dead) || (j < r[2].x && e[2] != dead) || (j < r[3].x && e[3] != dead));
                        };
#pragma unroll
                        for (int k = 0; k < 3; ++k) {                        // four steps at a time
                            if (!on(4 * k)) break;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    const int to = next[e[q] * n_classes + (int)(r[q][1 + k] >> (8 * j) & 255u)];       // (the end of the walk leads to itself)
                                    e[q] = (uint32_t)(4 * k + j) < r[q].x ? to : e[q];
                                }
                        }
                        for (uint32_t j = kInlineBytes; on(j); ++j)
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                if (j < r[q].x && e[q] != dead) e[q] = next[e[q] * n_classes + (int)class_at(r[q], t0 + q * kWave + lane, j)];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint64_t m = __ballot(e[q] != dead);
                            const int w = (t0 + q * kWave) / 32;
                            if (lane == w) bits = (uint32_t)m;
                            if (lane == w + 1) bits = (uint32_t)(m >> 32);
                        }
                    }
                } else if (passing > 0) {
                    found[wv][lane] = 0;
                    wave_sync();
                    for (int c0 = 0; c0 < n_classes; c0 += kWave) {
                        int to = dead;
                        if (c0 + lane < n_classes && start[c0 + lane + 1] > start[c0 + lane]) to = next[s * n_classes + c0 + lane];
                        for (uint64_t on = __ballot(to != dead); on; on &= on - 1) {
                            const int c = __builtin_ctzll(on), s1 = __builtin_amdgcn_readlane(to, c);
                            const int stop = (int)start[c0 + c + 1];
                            for (int at = (int)start[c0 + c] + lane; at < stop; at += kWave) {
                                const int t = order[at];
                                const Record r = text[t];
                                int e = s1;
                                for (uint32_t j = 1; j < r.x && e != dead; ++j) e = next[e * n_classes + (int)class_at(r, t, j)];
                                if (e != dead) atomicOr(&found[wv][t >> 5], 1u << (t & 31));
                            }
                        }
                    }
                    wave_sync();
                    bits = found[wv][lane];
                    wave_sync();
                }
            }
            const int v0 = first + 32 * lane;
            if (v0 < p.n_vocab) {
                if (known && p.end_id >= v0 && p.end_id < v0 + 32) {
                    const uint32_t bit = 1u << (p.end_id & 31);
                    bits = p.g.accepting[s] ? bits | bit : bits & ~bit;
                }
                p.masks[i * p.mask_stride + (v0 >> 5)] = bits;
            }
        }
    }
}

struct AdvanceParams {
    GrammarView g;
    TokenView t;
    const int32_t *states, *ids;
    int32_t n, end_id;
    int32_t *out;
};

// A lane per state: the chain of reads along one token's bytes; bound by the launch (5 us).
__global__ void __launch_bounds__(kGroupThreads) grammar_advance_kernel(AdvanceParams p) {
    const int i = blockIdx.x * kGroupThreads + threadIdx.x;
    if (i >= p.n) return;
    const int s = p.states[i], id = p.ids[i];
    int to = -1;
    if (s >= 0 && s < p.g.n_states) {
        if (p.end_id >= 0 && id == p.end_id) {
            to = p.g.accepting[s] ? s : -1;
        } else if (id >= 0 && id < p.t.n_tok) {
            const Record rec = p.t.tok[id];
            const uint32_t e = rec.x ? walk(p.g, rec, p.t.pool, (uint32_t)s) : (uint32_t)p.g.n_states;
            to = e < (uint32_t)p.g.n_states ? (int)e : -1;
        }
    }
    p.out[i] = to;
}

static int64_t align256g(int64_t v) { return (v + 255) & ~255ll; }

static GrammarView view_of(const bpe_grammar *g) {
    return {g->next, g->class_of, g->accepting, (int32_t)g->info.n_states, g->info.n_classes};
}

// Checks shared by the calls that walk tokens.
static int check_walk(const bpe_vocab *v, const bpe_grammar *g, int64_t n, int ids_are_output_ids, TokenView &t) {
    if (!v || !g) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (n < 0 || n >= (1 << 30)) { set_error("n out of range (%lld)", (long long)n); return BPE_ERR_SIZE; }
    if (ids_are_output_ids && !v->int_of) { set_error("the vocabulary was built without output ids"); return BPE_ERR_OPTION; }
    int rc = check_device(v->device, "the vocabulary");
    if (rc == BPE_OK) rc = check_device(g->device, "the grammar");
    t = {ids_are_output_ids ? v->tok_out : v->tok, v->pool, ids_are_output_ids ? v->n_out : (int32_t)v->info.n_ids};
    return rc;
}

}  // namespace bpe

using namespace bpe;

extern "C" int bpe_grammar_build(const int32_t *transitions, const uint8_t *accepting, int64_t n_states, bpe_grammar **out_grammar) {
    if (!out_grammar) { set_error("out_grammar is NULL"); return BPE_ERR_NULL; }
    *out_grammar = nullptr;
    if (!transitions) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (n_states < 1 || n_states > kMaxGrammarStates) { set_error("n_states %lld out of range", (long long)n_states); return BPE_ERR_SIZE; }
    for (int64_t i = 0; i < 256 * n_states; ++i)
        if (transitions[i] >= n_states) {
            set_error("byte %lld of state %lld leads to state %d of %lld", (long long)(i & 255), (long long)(i >> 8), transitions[i], (long long)n_states);
            return BPE_ERR_ID_RANGE;
        }
    try {
        // columns that are equal in every state are one class: refined state by state
        uint8_t class_of[256] = {0};
        int n_classes = 1;
        for (int64_t s = 0; s < n_states && n_classes < 256; ++s) {
            std::unordered_map<int64_t, int> seen;            // (class so far, state behind the byte) -> new class
            uint8_t refined[256];
            for (int b = 0; b < 256; ++b) {
                const int64_t to = std::max(transitions[256 * s + b], -1);
                refined[b] = (uint8_t)seen.emplace(((int64_t)class_of[b] << 32) + to + 1, (int)seen.size()).first->second;
            }
            n_classes = (int)seen.size();
            memcpy(class_of, refined, 256);
        }
        const int64_t b_next = 0, b_class = align256g(2 * (n_states + 1) * n_classes), b_accept = b_class + 256,
                      b_total = b_accept + align256g(n_states);
        std::vector<char> blob((size_t)b_total, 0);
        uint16_t *next = (uint16_t *)(blob.data() + b_next);
        for (int64_t s = 0; s < n_states; ++s)
            for (int b = 0; b < 256; ++b) {
                const int32_t to = transitions[256 * s + b];
                next[s * n_classes + class_of[b]] = (uint16_t)(to < 0 ? n_states : to);
            }
        for (int c = 0; c < n_classes; ++c) next[n_states * n_classes + c] = (uint16_t)n_states;
        memcpy(blob.data() + b_class, class_of, 256);
        for (int64_t s = 0; accepting && s < n_states; ++s) blob[b_accept + s] = accepting[s] != 0;

        bpe_grammar *g = new (std::nothrow) bpe_grammar();
        if (!g) { set_error("out of host memory"); return BPE_ERR_SIZE; }
        hipError_t e = hipGetDevice(&g->device);
        if (e != hipSuccess) { delete g; return hip_fail(e, "hipGetDevice"); }
        e = hipMalloc(&g->device_mem, blob.size());
        if (e != hipSuccess) { delete g; return hip_fail(e, "hipMalloc(grammar)"); }
        e = hipMemcpy(g->device_mem, blob.data(), blob.size(), hipMemcpyHostToDevice);
        if (e != hipSuccess) { (void)hipFree(g->device_mem); delete g; return hip_fail(e, "hipMemcpy(grammar)"); }
        char *d = (char *)g->device_mem;
        g->next = (const uint16_t *)(d + b_next);
        g->class_of = (const uint8_t *)(d + b_class);
        g->accepting = (const uint8_t *)(d + b_accept);
        g->info.n_states = n_states;
        g->info.n_classes = n_classes;
        g->info.device_bytes = b_total;
        *out_grammar = g;
        return BPE_OK;
    } catch (const std::exception &) {
        set_error("out of host memory");
        return BPE_ERR_SIZE;
    }
}

extern "C" int bpe_grammar_free(bpe_grammar *g) {
    if (!g) return BPE_OK;
    const hipError_t e = hipFree(g->device_mem);
    delete g;
    return e == hipSuccess ? BPE_OK : hip_fail(e, "hipFree(grammar)");
}

extern "C" int bpe_grammar_info(const bpe_grammar *g, bpe_grammar_info_t *info) {
    if (!g || !info) { set_error("null pointer"); return BPE_ERR_NULL; }
    *info = g->info;
    return BPE_OK;
}

extern "C" int bpe_grammar_masks(const bpe_vocab *v, const bpe_grammar *g, const int32_t *states, int64_t n, int ids_are_output_ids,
                                 int64_t n_vocab, int64_t end_id, uint32_t *masks, int64_t mask_stride, void *stream) {
    MaskParams p = {};
    const int rc = check_walk(v, g, n, ids_are_output_ids, p.t);
    if (rc != BPE_OK) return rc;
    if (n_vocab < 1 || n_vocab >= (1 << 30)) { set_error("n_vocab out of range (%lld)", (long long)n_vocab); return BPE_ERR_SIZE; }
    if (end_id < -1 || end_id >= n_vocab) { set_error("end_id %lld is outside [-1, n_vocab)", (long long)end_id); return BPE_ERR_ID_RANGE; }
    if (n == 0) return BPE_OK;
    if (!states || !masks) { set_error("null pointer"); return BPE_ERR_NULL; }
    if (n > 1 && mask_stride < (n_vocab + 31) / 32) { set_error("mask_stride is shorter than a row"); return BPE_ERR_SIZE; }
    p.g = view_of(g);
    p.states = states;
    p.n = (int32_t)n;
    p.n_vocab = (int32_t)n_vocab;
    p.end_id = (int32_t)end_id;
    p.masks = masks;
    p.mask_stride = mask_stride;
    const char *what = "bpe_grammar_masks launch";
    // A tile costs some 17 us before its first state is done.  Of 50,257 tokens: 64 states 12.3 us and in tiles 23, 128 states 20.3 and
    // 24.1, 300 states 39.5 and 25.8, 1,500 states 170 and 44.5; of 1,257 tokens 3,000 states 13.2 and 19.2.
    if (n * n_vocab <= 8000000) {
        const dim3 grid((unsigned)((n_vocab + kGroupThreads - 1) / kGroupThreads), (unsigned)std::min<int64_t>((n + kMaskChains - 1) / kMaskChains, 32768));
        return launch(grammar_masks_kernel, grid, kGroupThreads, p, stream, what);
    }
    const int64_t tiles = (n_vocab + kMaskTile - 1) / kMaskTile;
    const int64_t groups = std::max<int64_t>(std::min<int64_t>((n + kMaskWaves - 1) / kMaskWaves, std::max<int64_t>(256 / tiles, 1)), 1);
    const dim3 grid((unsigned)tiles, (unsigned)groups);
    const bool in_lds = (g->info.n_states + 1) * g->info.n_classes <= kMaskTable;
    return launch(in_lds ? grammar_tile_masks_kernel<true> : grammar_tile_masks_kernel<false>, grid, kMaskThreads, p, stream, what);
}

extern "C" int bpe_grammar_advance(const bpe_vocab *v, const bpe_grammar *g, const int32_t *states, const int32_t *ids, int64_t n,
                                   int ids_are_output_ids, int64_t end_id, int32_t *out_states, void *stream) {
    AdvanceParams p = {};
    const int rc = check_walk(v, g, n, ids_are_output_ids, p.t);
    if (rc != BPE_OK) return rc;
    if (end_id < -1 || end_id > 0x7FFFFFFFll) { set_error("end_id %lld out of range", (long long)end_id); return BPE_ERR_ID_RANGE; }
    if (n == 0) return BPE_OK;
    if (!states || !ids || !out_states) { set_error("null pointer"); return BPE_ERR_NULL; }
    p.g = view_of(g);
    p.states = states;
    p.ids = ids;
    p.n = (int32_t)n;
    p.end_id = (int32_t)end_id;
    p.out = out_states;
    return launch(grammar_advance_kernel, dim3((unsigned)((n + kGroupThreads - 1) / kGroupThreads)), kGroupThreads, p, stream,
                  "bpe_grammar_advance launch");
}
