// Entry points of the calls on histories (gm_seq_*): checks of arguments, workspace, launches, and what the device found.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gm_context.h"

static Arena arena_of(gm_ctx* c) {
    Arena ar;
    ar.base = c->ws;
    ar.cap = c->ws_bytes;
    ar.off = c->persistent;
    return ar;
}

// What the kernels wrote into the pinned words, once the stream has drained; the words are clear afterwards.
static int found(gm_ctx* c) {
    u32 w[SEQ_WORDS];
    for (int i = 0; i < SEQ_WORDS; ++i) {
        w[i] = *(volatile u32*)(c->seq_status + i);
        *(volatile u32*)(c->seq_status + i) = 0;
    }
    if (w[SEQ_BAD_TOKEN]) return fail(c, GM_ERR_INDEX, "a token is neither a row of the table nor -1");
    if (w[SEQ_BAD_OFFSETS])
        return fail(c, GM_ERR_INDEX, "offsets are not monotone from 0 to the number of rows, or a length exceeds `longest` or the rows behind its start");
    if (w[SEQ_CAPACITY]) return fail(c, GM_ERR_CAPACITY, "emb_rows_capacity is smaller than the number of distinct tokens");
    return GM_OK;
}
static int drain(gm_ctx* c) {
    HIPCHK(c, hipStreamSynchronize(c->stream));
    HIPCHK(c, hipGetLastError());
    prof_drain(c);
    return found(c);
}
// the end of every call
static int leave(gm_ctx* c) {
    if (c->wait) return drain(c);
    HIPCHK(c, hipGetLastError());
    return GM_OK;
}
// No exception passes the C boundary.
template <typename F>
static int guarded(gm_ctx* c, F&& body) {
    if (!c) return GM_ERR_ARG;
    try {
        if (!c->seq_status) return fail(c, GM_ERR_ARG, "the context was not created");
        HIPCHK(c, hipSetDevice(c->device));
        return body();
    } catch (...) {
        return GM_ERR_HIP;
    }
}

extern "C" int gm_wait(gm_ctx* c) {
    return guarded(c, [&]() -> int { return drain(c); });
}

// ------------------------------------------------------------------------------------------------ embedding rows
static int check_embed(gm_ctx* c, int64_t n, const int32_t* tokens, int64_t n_rows, int32_t dim, int32_t dtype, int64_t ld, float scale) {
    if (n < 0 || (n > 0 && !tokens)) return fail(c, GM_ERR_ARG, "bad tokens");
    if (n_rows < 1 || n_rows >= ((int64_t)1 << 31) - 1) return fail(c, GM_ERR_ARG, "n_rows must be in [1, 2^31 - 2]");
    if (dim < 1 || dim > 65536) return fail(c, GM_ERR_ARG, "dim must be in [1, 65536]");
    if (dtype != 0 && dtype != 1) return fail(c, GM_ERR_ARG, "dtype must be 0 (fp32) or 1 (bf16)");
    if (ld < dim) return fail(c, GM_ERR_ARG, "a row stride is smaller than dim");
    if (n >= (int64_t)1 << 31) return fail(c, GM_ERR_CAPACITY, "2^31 tokens or more in one call");
    if (!std::isfinite(scale)) return fail(c, GM_ERR_ARG, "scale must be finite");
    return GM_OK;
}

extern "C" int gm_seq_embed(gm_ctx* c, int64_t n_tokens, const int32_t* tokens, int64_t n_rows, int32_t dim, const float* table, float scale,
                            int32_t dtype, void* out, int64_t ld_out) {
    return guarded(c, [&]() -> int {
        const int rc = check_embed(c, n_tokens, tokens, n_rows, dim, dtype, ld_out, scale);
        if (rc != GM_OK) return rc;
        if (!table || (n_tokens > 0 && !out)) return fail(c, GM_ERR_ARG, "null table / out");
        {
            Prof p(c, "seq_embed", 4.0 * n_tokens + (double)n_tokens * dim * (4 + (dtype ? 2 : 4)), (double)n_tokens * dim);
            launch_seq_embed(c->stream, SeqEmbedArgs{n_tokens, tokens, n_rows, dim, scale, c->seq_status}, table, dtype, out, ld_out);
        }
        return leave(c);
    });
}

// keys and positions twice, the passes' counts, the rows of every chunk, the chunks' pieces
static SeqEmbedGradBufs embed_grad_bufs(Arena& ar, int64_t n, int32_t dim) {
    SeqEmbedGradBufs b;
    for (int i = 0; i < 2; ++i) {
        b.keys[i] = ar.get<u32>(n + 4);
        b.vals[i] = ar.get<u32>(n + 4);
    }
    const int64_t chunks = seq_chunks(n);
    b.hist = ar.get<u32>(std::max(radix_hist_words(n, 0), radix_wide_words(n)));
    b.counts = ar.get<u32>(chunks + 1);
    b.scan_tmp = ar.get<u32>(scan_tmp_words(chunks));
    b.partial = ar.get<float>(2 * chunks * dim);
    return b;
}
extern "C" size_t gm_seq_embed_grad_bytes(int64_t n_tokens, int32_t dim) {
    if (n_tokens < 0 || dim < 1 || n_tokens >= (int64_t)1 << 31 || dim > 65536) return 0;
    // (a call may need less than one of fewer tokens, where chunks are longer, the sort's tiles larger or its passes narrower: the most of any up to n_tokens)
    size_t most = 0;
    for (int64_t n : {n_tokens, SEQ_SHORT_LIST, RS_LONG - 1, RS_WIDE}) {
        Arena ar;
        ar.cap = ~(size_t)0 >> 1;
        embed_grad_bufs(ar, std::min(n, n_tokens), dim);
        most = std::max(most, ar.off);
    }
    return most;
}

extern "C" int gm_seq_embed_grad(gm_ctx* c, int64_t n_tokens, const int32_t* tokens, int64_t n_rows, int32_t dim, int32_t dtype, const void* grad,
                                 int64_t ld_grad, float scale, int64_t* emb_rows, float* emb_grad, int64_t* n_emb_rows, int64_t emb_rows_capacity,
                                 float* table) {
    return guarded(c, [&]() -> int {
        const int rc = check_embed(c, n_tokens, tokens, n_rows, dim, dtype, ld_grad, scale);
        if (rc != GM_OK) return rc;
        if (n_tokens > 0 && !grad) return fail(c, GM_ERR_ARG, "null grad");
        if (!table && (!n_emb_rows || emb_rows_capacity < 0 || (emb_rows_capacity > 0 && (!emb_rows || !emb_grad))))
            return fail(c, GM_ERR_ARG, "null outputs: a table, or emb_rows, emb_grad and n_emb_rows");
        Arena ar = arena_of(c);
        const SeqEmbedGradBufs b = embed_grad_bufs(ar, n_tokens, dim);
        if (ar.overflow) return fail(c, GM_ERR_WORKSPACE, "workspace too small: gm_seq_embed_grad needs %zu bytes", ar.off);
        {
            Prof p(c, "seq_embed_grad", 4.0 * n_tokens + (double)n_tokens * dim * (dtype ? 2 : 4), (double)n_tokens * dim);
            launch_seq_embed_grad(c->stream, SeqEmbedArgs{n_tokens, tokens, n_rows, dim, scale, c->seq_status}, dtype, grad, ld_grad, b, emb_rows, emb_grad,
                                  table ? nullptr : n_emb_rows, emb_rows_capacity, table);
        }
        return leave(c);
    });
}

// ------------------------------------------------------------------------------------------------ recurrence
// Rows, none of which a sequence may hold: nothing would be launched that could find it out.
static int check_longest(gm_ctx* c, const gm_seq* s) {
    if (s->longest == 0 && s->n_rows > 0 && !s->lengths) return fail(c, GM_ERR_INDEX, "`longest` is 0 and there are %lld rows", (long long)s->n_rows);
    return GM_OK;
}
static int check_scan(gm_ctx* c, const gm_seq* s, int32_t channels, int32_t dtype) {
    if (!s) return fail(c, GM_ERR_ARG, "null sequences");
    if (s->n_seqs < 0 || s->n_rows < 0 || s->longest < 0 || (s->n_seqs == 0 && s->n_rows > 0) || (s->n_seqs > 0 && !s->offsets))
        return fail(c, GM_ERR_ARG, "bad sequences");
    if (channels < 1 || channels > 65536) return fail(c, GM_ERR_ARG, "channels must be in [1, 65536]");
    if (dtype != 0 && dtype != 1) return fail(c, GM_ERR_ARG, "dtype must be 0 (fp32) or 1 (bf16)");
    if (s->longest >= (int64_t)1 << 31 || s->n_seqs >= (int64_t)1 << 31 || s->n_seqs * ((channels + 31) / 32) >= (int64_t)1 << 31)
        return fail(c, GM_ERR_CAPACITY, "a sequence of 2^31 rows or more, or too many sequences times channels");
    return check_longest(c, s);
}
// The pieces of the time axis, as many as what is left of the arena holds the maps of.
static SeqSplit scan_split(Arena& ar, int64_t n_seqs, int64_t longest, int32_t channels, int32_t dtype, int grad, float** agg) {
    const int64_t room = ar.off < ar.cap ? (int64_t)((ar.cap - ar.off) / 256 * 256 / sizeof(float)) : 0;
    const SeqSplit sp = seq_scan_split(n_seqs, longest, channels, dtype, grad, room);
    *agg = sp.chunks > 1 ? ar.get<float>(2 * n_seqs * sp.chunks * channels) : nullptr;
    return sp;
}
extern "C" size_t gm_seq_scan_bytes(int64_t n_seqs, int64_t longest, int32_t channels, int32_t dtype) {
    if (n_seqs < 0 || longest < 0 || n_seqs >= (int64_t)1 << 31 || longest >= (int64_t)1 << 31 || channels < 1 || channels > 65536 || (dtype != 0 && dtype != 1)) return 0;
    Arena ar;
    ar.cap = ~(size_t)0 >> 1;
    float* agg;
    scan_split(ar, n_seqs, longest, channels, dtype, 1, &agg);   // (the gradient is split wherever the forward pass is, into as many chunks)
    return ar.off;
}
static int run_scan(gm_ctx* c, SeqScanArgs& a, const gm_seq* s, int32_t channels, int32_t dtype, int grad) {
    a.v = SeqView{s->n_seqs, s->n_rows, s->longest, s->offsets, c->seq_status};
    a.channels = channels;
    Arena ar = arena_of(c);
    const SeqSplit sp = scan_split(ar, s->n_seqs, s->longest, channels, dtype, grad, &a.agg);
    a.chunks = sp.chunks;
    a.chunk = sp.chunk;
    {
        const double n = (double)s->n_rows * channels * (dtype ? 2 : 4);
        Prof p(c, grad ? "seq_scan_grad" : "seq_scan", (grad ? 6 : 3) * n, 0);
        launch_seq_scan(c->stream, a, dtype, grad);
    }
    return leave(c);
}

extern "C" int gm_seq_scan(gm_ctx* c, const gm_seq* seqs, int32_t channels, int32_t dtype, const void* x, int64_t ldx, const void* gate, int64_t ldg,
                           const float* h0, void* h, int64_t ldh, float* last) {
    return guarded(c, [&]() -> int {
        const int rc = check_scan(c, seqs, channels, dtype);
        if (rc != GM_OK) return rc;
        if (seqs->n_rows > 0 && (!x || !gate || !h)) return fail(c, GM_ERR_ARG, "null x / gate / h");
        if (std::min({ldx, ldg, ldh}) < channels) return fail(c, GM_ERR_ARG, "a row stride is smaller than the number of channels");
        SeqScanArgs a{};
        a.x = x; a.ldx = ldx; a.gate = gate; a.ldg = ldg; a.start = h0; a.out = h; a.ldo = ldh; a.end = last;
        return run_scan(c, a, seqs, channels, dtype, 0);
    });
}

extern "C" int gm_seq_scan_grad(gm_ctx* c, const gm_seq* seqs, int32_t channels, int32_t dtype, const void* x, int64_t ldx, const void* gate,
                                int64_t ldg, const void* h, int64_t ldh, const float* h0, const void* dh, int64_t lddh, const float* dlast, void* dx,
                                int64_t lddx, void* dgate, int64_t lddg, float* dh0) {
    return guarded(c, [&]() -> int {
        const int rc = check_scan(c, seqs, channels, dtype);
        if (rc != GM_OK) return rc;
        if (seqs->n_rows > 0 && (!x || !gate || !h || !dh || !dx || !dgate)) return fail(c, GM_ERR_ARG, "null x / gate / h / dh / dx / dgate");
        if (std::min({ldx, ldg, ldh, lddh, lddx, lddg}) < channels) return fail(c, GM_ERR_ARG, "a row stride is smaller than the number of channels");
        SeqScanArgs a{};
        a.x = x; a.ldx = ldx; a.gate = gate; a.ldg = ldg; a.h = h; a.ldh = ldh; a.dh = dh; a.lddh = lddh;
        a.start = h0; a.tail = dlast; a.out = dx; a.ldo = lddx; a.out2 = dgate; a.ldo2 = lddg; a.end = dh0;
        return run_scan(c, a, seqs, channels, dtype, 1);
    });
}

extern "C" int gm_seq_scan_step(gm_ctx* c, int64_t n_seqs, int32_t channels, int32_t dtype, const void* x, int64_t ldx, const void* gate, int64_t ldg,
                                float* state, void* h, int64_t ldh) {
    return guarded(c, [&]() -> int {
        if (n_seqs < 0) return fail(c, GM_ERR_ARG, "bad n_seqs");
        const gm_seq one{0, 0, 1, nullptr, nullptr};
        const int rc = check_scan(c, &one, channels, dtype);
        if (rc != GM_OK) return rc;
        if (n_seqs > 0 && (!x || !gate || !state)) return fail(c, GM_ERR_ARG, "null x / gate / state");
        if (std::min(ldx, ldg) < channels || (h && ldh < channels)) return fail(c, GM_ERR_ARG, "a row stride is smaller than the number of channels");
        if (n_seqs >= ((int64_t)1 << 38) / channels) return fail(c, GM_ERR_CAPACITY, "too many sequences times channels");
        {
            Prof p(c, "seq_scan_step", (double)n_seqs * channels * (8 + 3 * (dtype ? 2 : 4)), 0);
            launch_seq_scan_step(c->stream, n_seqs, channels, dtype, x, ldx, gate, ldg, state, h, ldh);
        }
        return leave(c);
    });
}

// ------------------------------------------------------------------------------------------------ attention
// what a size query needs, too
static int check_attend_sizes(gm_ctx* c, const gm_seq* q, const gm_seq* k, const gm_seq_heads* hd) {
    if (hd->dtype != 0 && hd->dtype != 1) return fail(c, GM_ERR_ARG, "dtype must be 0 (fp32) or 1 (bf16)");
    const int unit = hd->dtype ? 8 : 4;
    if (hd->head_dim < unit || hd->head_dim > 128 || hd->head_dim % unit)
        return fail(c, GM_ERR_ARG, "head_dim must be a multiple of %d (16 bytes), at most 128", unit);
    if (hd->n_kv_heads < 1 || hd->n_heads < 1 || hd->n_heads % hd->n_kv_heads || hd->n_heads > 1024)
        return fail(c, GM_ERR_ARG, "n_heads must be a multiple of n_kv_heads, at most 1024");
    const int64_t most = (int64_t)1 << 31, group = hd->n_heads / hd->n_kv_heads;
    const int64_t place = most - 256;   // (the kernels' places inside a sequence are int; a tile may go that far beyond its end)
    if (q->n_seqs >= most || q->n_rows >= most || q->longest >= place || k->longest >= place || q->longest * group >= place || q->n_rows * hd->n_heads >= most ||
        q->n_seqs * hd->n_kv_heads >= most / (std::max(q->longest * group, k->longest) / 32 + 1))   // (workgroups; as a product it may pass 64 bits)
        return fail(c, GM_ERR_CAPACITY, "too many rows, heads or sequences for one call");
    return GM_OK;
}
static int check_attend(gm_ctx* c, const gm_seq* q, const gm_seq* k, const gm_seq_heads* hd, bool grad) {
    if (!q || !k || !hd) return fail(c, GM_ERR_ARG, "null sequences / heads");
    if (q->n_seqs < 0 || q->n_seqs != k->n_seqs) return fail(c, GM_ERR_ARG, "queries and keys must have the same number of sequences");
    for (const gm_seq* s : {q, k})
        if (s->n_rows < 0 || s->longest < 0 || (s->n_seqs == 0 && s->n_rows > 0) || (s->n_seqs > 0 && !s->offsets)) return fail(c, GM_ERR_ARG, "bad sequences");
    if (q->lengths || (grad && k->lengths)) return fail(c, GM_ERR_ARG, "lengths: only for the keys of gm_seq_attend");
    if (!(hd->scale > 0.f) || !std::isfinite(hd->scale)) return fail(c, GM_ERR_ARG, "scale must be positive and finite");
    int rc = check_attend_sizes(c, q, k, hd);
    if (rc != GM_OK || (rc = check_longest(c, q)) != GM_OK) return rc;
    return check_longest(c, k);
}
static int check_rows(gm_ctx* c, const gm_seq_heads* hd, int heads, int64_t n, const void* p, int64_t ld, const char* name) {
    if (n > 0 && !p) return fail(c, GM_ERR_ARG, "null %s", name);
    const int64_t elem = hd->dtype ? 2 : 4;
    if (ld < (int64_t)heads * hd->head_dim) return fail(c, GM_ERR_ARG, "the row stride of %s is smaller than its heads", name);
    if (ld >= MAX_WIDTH) return fail(c, GM_ERR_ARG, "the row stride of %s must be below %d elements", name, (int)MAX_WIDTH);
    if ((uintptr_t)p % 16 || (ld * elem) % 16) return fail(c, GM_ERR_ARG, "%s must be 16-byte aligned, its row stride too", name);
    return GM_OK;
}
static SeqAttendArgs attend_args(gm_ctx* c, const gm_seq* q, const gm_seq* k, const gm_seq_heads* hd) {
    SeqAttendArgs a{};
    a.n_seqs = q->n_seqs; a.n_queries = q->n_rows; a.n_keys = k->n_rows;
    a.longest_q = q->longest; a.longest_k = k->longest;
    a.q_offsets = q->offsets; a.k_offsets = k->offsets; a.k_lengths = k->lengths;
    a.kv_heads = hd->n_kv_heads; a.group = hd->n_heads / hd->n_kv_heads; a.dim = hd->head_dim; a.scale = hd->scale;
    a.splits = 1;
    a.status = c->seq_status;
    return a;
}
static void attend_bufs(Arena& ar, SeqAttendArgs& a, int n_cus, int dtype, bool grad) {
    const int64_t n = a.n_queries * a.kv_heads * a.group;
    seq_attend_shape(a, n_cus, dtype, grad);
    a.order = ar.get<int32_t>(2 * 256);
    if (grad) {
        a.stat = ar.get<float2>(n + 1);
        return;
    }
    if (a.splits > 1) {
        a.part_o = ar.get<float>(a.splits * n * a.dim);
        a.part_ml = ar.get<float>(a.splits * n * 2);
    }
}
extern "C" size_t gm_seq_attend_bytes(const gm_ctx* c, const gm_seq* queries, const gm_seq* keys, const gm_seq_heads* heads, int32_t grad) {
    if (!c || !queries || !keys || !heads || queries->n_seqs < 0 || queries->n_rows < 0 || queries->longest < 0 || keys->longest < 0) return 0;
    if (check_attend_sizes(nullptr, queries, keys, heads) != GM_OK) return 0;
    SeqAttendArgs a = attend_args(const_cast<gm_ctx*>(c), queries, keys, heads);
    Arena ar, most;
    ar.cap = most.cap = ~(size_t)0 >> 1;
    attend_bufs(ar, a, c->n_cus, heads->dtype, grad != 0);
    if (grad) return ar.off;
    // (fewer rows are cut into more pieces: the most of any call of no more of anything)
    const int64_t n = seq_attend_pieces(a, c->n_cus, heads->dtype);
    most.get<int32_t>(2 * 256);
    most.get<float>(n * a.dim);
    most.get<float>(n * 2);
    return std::max(ar.off, most.off);
}

extern "C" int gm_seq_attend(gm_ctx* c, const gm_seq* queries, const gm_seq* keys, const gm_seq_heads* heads, const void* q, int64_t ldq, const void* k,
                             int64_t ldk, const void* v, int64_t ldv, const uint8_t* key_mask, void* o, int64_t ldo, float* lse) {
    return guarded(c, [&]() -> int {
        int rc = check_attend(c, queries, keys, heads, false);
        if (rc != GM_OK) return rc;
        const int H = heads->n_heads, G = heads->n_kv_heads;
        if ((rc = check_rows(c, heads, H, queries->n_rows, q, ldq, "q")) != GM_OK || (rc = check_rows(c, heads, G, keys->n_rows, k, ldk, "k")) != GM_OK ||
            (rc = check_rows(c, heads, G, keys->n_rows, v, ldv, "v")) != GM_OK || (rc = check_rows(c, heads, H, queries->n_rows, o, ldo, "o")) != GM_OK)
            return rc;
        if (queries->n_rows > 0 && !lse) return fail(c, GM_ERR_ARG, "null lse");
        SeqAttendArgs a = attend_args(c, queries, keys, heads);
        a.q = q; a.ldq = ldq; a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.key_mask = key_mask; a.out = o; a.ldout = ldo; a.lse = lse;
        Arena ar = arena_of(c);
        attend_bufs(ar, a, c->n_cus, heads->dtype, false);
        if (ar.overflow) return fail(c, GM_ERR_WORKSPACE, "workspace too small: gm_seq_attend needs %zu bytes", ar.off);
        {
            Prof p(c, "seq_attend", 0, 0);
            launch_seq_attend(c->stream, a, heads->dtype);
        }
        return leave(c);
    });
}

extern "C" int gm_seq_attend_grad(gm_ctx* c, const gm_seq* queries, const gm_seq* keys, const gm_seq_heads* heads, const void* dout, int64_t lddo,
                                  const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* o, int64_t ldo,
                                  const float* lse, const uint8_t* key_mask, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv, int64_t lddv) {
    return guarded(c, [&]() -> int {
        int rc = check_attend(c, queries, keys, heads, true);
        if (rc != GM_OK) return rc;
        const int H = heads->n_heads, G = heads->n_kv_heads;
        const int64_t nq = queries->n_rows, nk = keys->n_rows;
        const struct { const void* p; int64_t ld; int heads; int64_t n; const char* name; } rows[] = {
            {dout, lddo, H, nq, "dout"}, {q, ldq, H, nq, "q"}, {k, ldk, G, nk, "k"}, {v, ldv, G, nk, "v"}, {o, ldo, H, nq, "o"},
            {dq, lddq, H, nq, "dq"}, {dk, lddk, G, nk, "dk"}, {dv, lddv, G, nk, "dv"}};
        for (const auto& r : rows)
            if ((rc = check_rows(c, heads, r.heads, r.n, r.p, r.ld, r.name)) != GM_OK) return rc;
        if (nq > 0 && !lse) return fail(c, GM_ERR_ARG, "null lse");
        SeqAttendArgs a = attend_args(c, queries, keys, heads);
        a.q = q; a.ldq = ldq; a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.o = o; a.ldo = ldo; a.dout = dout; a.lddo = lddo;
        a.key_mask = key_mask; a.lse = const_cast<float*>(lse);
        a.dq = dq; a.lddq = lddq; a.dk = dk; a.lddk = lddk; a.dv = dv; a.lddv = lddv;
        Arena ar = arena_of(c);
        attend_bufs(ar, a, c->n_cus, heads->dtype, true);
        if (ar.overflow) return fail(c, GM_ERR_WORKSPACE, "workspace too small: gm_seq_attend_grad needs %zu bytes", ar.off);
        {
            Prof p(c, "seq_attend_grad", 0, 0);
            launch_seq_attend_grad(c->stream, a, heads->dtype);
        }
        return leave(c);
    });
}
