// Grammars over the vocabulary: a deterministic automaton over bytes, and which tokens' bytes it can take from a state.
#include <algorithm>
#include <cstring>
#include <new>
#include <unordered_map>
#include <string>

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

// One lane per token, one row of the grid per state.
__global__ void __launch_bounds__(kGroupThreads) grammar_masks_kernel(MaskParams p) {
    const int v = blockIdx.x * kGroupThreads + threadIdx.x;
    for (int i = blockIdx.y; i < p.n; i += gridDim.y) {
        const int s = p.states[i];
        bool on = false;
        if (s >= 0 && s < p.g.n_states && v < p.n_vocab) {
            Record rec = {0, 0, 0, 0};
            if (v < p.t.n_tok) rec = p.t.tok[v];
            on = rec.x != 0 && walk(p.g, rec, p.t.pool, (uint32_t)s) < (uint32_t)p.g.n_states;
            if (v == p.end_id) on = p.g.accepting[s] != 0;
        }
        const uint64_t bits = __ballot(on);
        if ((v & 31) == 0 && v < p.n_vocab) p.masks[i * p.mask_stride + (v >> 5)] = (uint32_t)(bits >> (v & 32));
    }
}

struct AdvanceParams {
    GrammarView g;
    TokenView t;
    const int32_t *states, *ids;
    int32_t n, end_id;
    int32_t *out;
};

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
    if (n < 0 || n >= 0x7FFFFFFFll) { set_error("n out of range (%lld)", (long long)n); return BPE_ERR_SIZE; }
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
    const dim3 grid((unsigned)((n_vocab + kGroupThreads - 1) / kGroupThreads), (unsigned)std::min<int64_t>(n, 32768));
    return launch(grammar_masks_kernel, grid, kGroupThreads, p, stream, "bpe_grammar_masks launch");
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
