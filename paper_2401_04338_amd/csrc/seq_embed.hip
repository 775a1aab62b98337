// Rows of an embedding table, one per token of a history: the scaled lookup and its gradient by sorted tokens.
//   lookup    out[i, :] = scale * table[token_i, :]                       (padding, token -1: zeros)
//   gradient  sum[r, :] = scale * sum over {i : token_i = r} of grad[i, :]
// The gradient's order is fixed: tokens are sorted with their positions (stable), a chunk of 16 or 64 positions is summed in that
// order by one group of lanes, and the pieces of a row that spans chunks are added in the order of the chunks.
#include <algorithm>

#include "gm_internal.h"

// Most vectors of a row that the layout allows: 8, 4 or 1 elements a lane.
static int row_vector(int dim, int64_t ld, const void* p, int elem, const void* fp32_rows) {
    for (int v : {8, 4}) {
        const int bytes = std::min(v * elem, 16);
        if (dim % v == 0 && (ld * elem) % bytes == 0 && (uintptr_t)p % bytes == 0 && (uintptr_t)fp32_rows % 16 == 0) return v;
    }
    return 1;
}
static int lanes_of_row(int dim, int v) {   // log2
    int l = 2;
    while (l < 6 && (v << l) < dim) ++l;
    return l;
}

// A group of 2^lg lanes per row, several rows a lane in flight.  Bound: memory, the rows read once and the output written once: a million tokens of 128
// columns, 1.05 Zipf over a million rows, bf16: 72 to 88 us, 3.9 to 4.9 TB/s (100 with the output through the caches).
template <typename T, int V>
__global__ __launch_bounds__(256) void seq_embed_kernel(SeqEmbedArgs a, const float* __restrict__ table, T* __restrict__ out, int64_t ld, int lg) {
    constexpr int ROWS = 4;
    const int rows = 256 >> lg, c0 = (threadIdx.x & ((1 << lg) - 1)) * V;
    const int64_t first = (int64_t)workgroup() * rows * ROWS + (threadIdx.x >> lg);
    int tok[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int64_t i = first + (int64_t)j * rows;
        tok[j] = i < a.n ? a.tokens[i] : -1;
        if ((u32)tok[j] >= (u32)a.n_rows) {
            if (tok[j] != -1) seq_flag(a.status, SEQ_BAD_TOKEN);
            tok[j] = -1;
        }
    }
    for (int c = c0; c < a.dim; c += V << lg) {
        Pack<float, V> x[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            x[j] = tok[j] >= 0 ? *reinterpret_cast<const Pack<float, V>*>(table + (int64_t)tok[j] * a.dim + c) : Pack<float, V>{};
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const int64_t i = first + (int64_t)j * rows;
            if (i >= a.n) break;
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = tok[j] >= 0 ? a.scale * x[j].get(e) : 0.f;   // (not 0 * scale: that may be negative zero, or NaN)
            Pack<T, V> p;
            p.put(y);
            stream_out(out + i * ld + c, p);
        }
    }
}

void launch_seq_embed(hipStream_t st, const SeqEmbedArgs& a, const float* table, int out_bf16, void* out, int64_t ld) {
    if (a.n <= 0) return;
    const int v = row_vector(a.dim, ld, out, out_bf16 ? 2 : 4, table), lg = lanes_of_row(a.dim, v);
    const dim3 grid = workgroups((a.n + (256 >> lg) * 4 - 1) / ((256 >> lg) * 4));
#define EMBED(T_, V_) hipLaunchKernelGGL((seq_embed_kernel<T_, V_>), grid, dim3(256), 0, st, a, table, (T_*)out, ld, lg)
    if (out_bf16) { if (v == 8) EMBED(bf16_t, 8); else if (v == 4) EMBED(bf16_t, 4); else EMBED(bf16_t, 1); }
    else { if (v == 8) EMBED(float, 8); else if (v == 4) EMBED(float, 4); else EMBED(float, 1); }
#undef EMBED
}

// ------------------------------------------------------------------------------------------------ gradient
// Sorted positions a group of lanes sums.  us with 16 / 32 / 64: 30,000 tokens 49 / 57 / 74, 200,000 81 / 84 / 103, 400,000 118 / 116 / 118, a million 186 / 186 / 184,
// where 64 leave a quarter of the pieces and of their workspace.
static int seq_chunk(int64_t n) { return n <= SEQ_SHORT_LIST ? 16 : 64; }
int64_t seq_chunks(int64_t n) { return (n + seq_chunk(n) - 1) / seq_chunk(n); }

// Padding and bad tokens get the key n_rows: they sort behind every row.
__global__ __launch_bounds__(256) void seq_keys_kernel(SeqEmbedArgs a, u32* keys, u32* vals) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.n) return;
    const int tok = a.tokens[i];
    const bool ok = (u32)tok < (u32)a.n_rows;
    if (!ok && tok != -1) seq_flag(a.status, SEQ_BAD_TOKEN);
    keys[i] = ok ? (u32)tok : (u32)a.n_rows;
    vals[i] = (u32)i;
}

// rows that begin in every chunk
__global__ __launch_bounds__(256) void seq_heads_kernel(const u32* __restrict__ keys, int64_t n, int ch, u32 pad, u32* counts) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool head = i < n && keys[i] != pad && (i == 0 || keys[i - 1] != keys[i]);
    const u64 heads = __ballot(head);
    const int lane = threadIdx.x & 63;
    if (i < n && i % ch == 0) counts[i / ch] = (u32)__popcll((heads >> lane) & (~0ull >> (64 - ch)));
}

// The shortest lists: keys, sort and the rows in front of every chunk by one workgroup.  A pass sorts by eight bits, stable: every wave ranks its share of the positions
// 64 at a time by ballots, the counts of the waves are summed a digit a thread, and the pairs move through LDS.  Bound: latency of the passes.  us a call with the
// launches for long lists / with this: 100 tokens 26 / 19, 1,000 of a million rows 37 / 24, 4,096 48 / 36, 8,000 55 / 47.
#define SEQ_SORT 8192
__global__ __launch_bounds__(1024) void seq_sort_one_kernel(SeqEmbedArgs a, int bits, int ch, u32* keys, u32* vals, u32* before, u32* total) {
    constexpr int R = SEQ_SORT / 1024, W = 16;
    __shared__ u32 sk[SEQ_SORT];
    __shared__ uint16_t sv[SEQ_SORT];
    __shared__ __attribute__((aligned(16))) uint16_t cnt[W][256];
    __shared__ u32 start[256], sums[W];
    const int n = (int)a.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rounds = (n + 1023) / 1024;
    const u64 below = (1ull << lane) - 1ull;
    u32 key[R], val[R], rank[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (wave * rounds + r) * 64 + lane;
        key[r] = val[r] = 0;
        if (r < rounds && i < n) {
            const int tok = a.tokens[i];
            const bool ok = (u32)tok < (u32)a.n_rows;
            if (!ok && tok != -1) seq_flag(a.status, SEQ_BAD_TOKEN);
            key[r] = ok ? (u32)tok : (u32)a.n_rows;
            val[r] = (u32)i;
        }
    }
    for (int shift = 0; shift < bits; shift += 8) {
        for (int i = threadIdx.x; i < W * 128; i += 1024) reinterpret_cast<u32*>(&cnt[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= rounds) break;
            const bool valid = (wave * rounds + r) * 64 + lane < n;
            const u32 d = key[r] >> shift & 255u;
            u64 peers = __ballot(valid);
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const bool bit = (d >> b) & 1u;
                const u64 m = __ballot(bit);
                peers &= bit ? m : ~m;
            }
            const int leader = valid ? __ffsll((unsigned long long)peers) - 1 : lane;
            u32 old = 0;
            if (valid && lane == leader) {
                old = cnt[wave][d];
                cnt[wave][d] = (uint16_t)(old + (u32)__popcll(peers));
            }
            rank[r] = __shfl(old, leader) + (u32)__popcll(peers & below);
        }
        __syncthreads();
        u32 of_digit = 0, incl = 0;
        if (threadIdx.x < 256) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const u32 c = cnt[w][threadIdx.x];
                cnt[w][threadIdx.x] = (uint16_t)of_digit;
                of_digit += c;
            }
            incl = of_digit;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const u32 o = __shfl_up(incl, d);
                if (lane >= d) incl += o;
            }
            if (lane == 63) sums[wave] = incl;
        }
        __syncthreads();
        if (threadIdx.x < 256) {
            u32 front = 0;
#pragma unroll
            for (int w = 0; w < 3; ++w) front += w < wave ? sums[w] : 0u;
            start[threadIdx.x] = front + incl - of_digit;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < rounds && (wave * rounds + r) * 64 + lane < n) {
                const u32 d = key[r] >> shift & 255u, at = start[d] + cnt[wave][d] + rank[r];
                sk[at] = key[r];
                sv[at] = (uint16_t)val[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = (wave * rounds + r) * 64 + lane;
            if (r < rounds && i < n) {
                key[r] = sk[i];
                val[r] = sv[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (wave * rounds + r) * 64 + lane;
        if (r < rounds && i < n) {
            keys[i] = key[r];
            vals[i] = val[r];
        }
    }
    if (!before) return;
    const int i0 = threadIdx.x * 8;   // (a chunk is a multiple of 8 positions)
    u32 c = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i0 + j < n) c += sk[i0 + j] != (u32)a.n_rows && (i0 + j == 0 || sk[i0 + j - 1] != sk[i0 + j]) ? 1u : 0u;
    u32 incl = c;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const u32 o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    __syncthreads();   // (the passes' sums)
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    u32 front = 0, whole = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (w < wave) front += sums[w];
        whole += sums[w];
    }
    if (i0 < n && i0 % ch == 0) before[i0 / ch] = front + incl - c;
    if (threadIdx.x == 0) *total = whole;
}

__global__ void seq_none_kernel(int64_t* n_emb_rows) { *n_emb_rows = 0; }

struct SeqSumArgs {
    const u32 *keys, *vals, *seg;   // seg: rows that begin in front of every chunk (list form)
    int64_t n, capacity;
    u32 pad;
    int dim, ch;
    float scale;
    float *partial;                 // [chunks][2][dim]: a chunk's piece of the row that began before it, of the row that goes on behind it
    int64_t* emb_rows;
    float *emb_grad, *table;
    const u32* total;               // rows of the list
    int64_t* n_emb_rows;
    u32* status;
};
template <int V>
__device__ __forceinline__ Pack<float, V> seq_old(const SeqSumArgs& a, u32 key, int c) {
    return *reinterpret_cast<const Pack<float, V>*>(a.table + (int64_t)key * a.dim + c);
}
template <int V, bool TABLE>   // old: the table's row (table form)
__device__ __forceinline__ void seq_emit(const SeqSumArgs& a, u32 key, int64_t seg, int c, const Pack<float, V>& old, const float (&acc)[V]) {
    float y[V];
    float* p;
    if (TABLE) {
        p = a.table + (int64_t)key * a.dim + c;
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = fmaf(a.scale, acc[e], old.get(e));
    } else {
        if (seg >= a.capacity) return;
        if (c == 0) a.emb_rows[seg] = (int64_t)key;
        p = a.emb_grad + seg * a.dim + c;
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = a.scale * acc[e];
    }
    Pack<float, V> o;
    o.put(y);
    stream_out(p, o);
}

// One group of 2^lg lanes per chunk and slab of columns (blockIdx.y): gradient rows in sorted order, eight in flight.
// Bound: memory -- the gradient rows, read once in runs of dim elements: a million of 128 columns, bf16, 82 us of the call's 162 (the sort 60, the pieces 12).
// The table's rows that a chunk adds to are asked for with the gradient rows that end them (one after the other they took 23 us for 61,000 tokens).
template <typename T, int V, bool TABLE>
__global__ __launch_bounds__(256) void seq_sum_kernel(SeqSumArgs a, const T* __restrict__ grad, int64_t ld, int lg) {
    if (!TABLE && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        *a.n_emb_rows = (int64_t)*a.total;
        if ((int64_t)*a.total > a.capacity) seq_flag(a.status, SEQ_CAPACITY);
    }
    extern __shared__ u32 sh[];   // per group the chunk's keys and values, and the keys on either side
    const int ch = a.ch, per = 2 * ch + 2, grp = threadIdx.x >> lg, l = threadIdx.x & ((1 << lg) - 1), lanes = 1 << lg;
    const int64_t chunk = (int64_t)blockIdx.x * (256 >> lg) + grp, cb = chunk * ch;
    u32* k = sh + grp * per + 1;
    u32* v = k + ch + 1;
    if (cb < a.n)
        for (int p = l - 1; p <= ch; p += lanes) {
            const int64_t i = cb + p;
            k[p] = i >= 0 && i < a.n ? a.keys[i] : ~0u;   // (no row's key, nor the padding's)
            if (p >= 0 && p < ch) v[p] = i < a.n ? a.vals[i] : 0u;
        }
    __syncthreads();
    const int c = (int)blockIdx.y * (V << lg) + l * V;
    // a workgroup inside one row (the keys in front of it and behind it are the same) leaves one piece, under its first chunk
    const int64_t b0 = (int64_t)blockIdx.x * (256 >> lg) * ch, b1 = b0 + (int64_t)(256 >> lg) * ch;
    const bool inside = b0 > 0 && b1 < a.n && a.keys[b0 - 1] == a.keys[b1] && a.keys[b1] != a.pad;
    if (inside) {
        __shared__ float stage[256 * V];
        float acc[V] = {};
        if (c < a.dim)
            for (int p0 = 0; p0 < ch; p0 += 8) {
                Pack<T, V> x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = stream_in<Pack<T, V>>(grad + (int64_t)v[p0 + j] * ld + c);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] += x[j].get(e);
            }
#pragma unroll
        for (int e = 0; e < V; ++e) stage[e * 256 + threadIdx.x] = acc[e];
        __syncthreads();
        if (grp == 0 && c < a.dim) {
            for (int g = 1; g < 256 >> lg; ++g)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += stage[e * 256 + (g << lg) + l];
            Pack<float, V> o;
            o.put(acc);
            *reinterpret_cast<Pack<float, V>*>(a.partial + chunk * 2 * a.dim + c) = o;
        }
        return;
    }
    if (cb >= a.n || c >= a.dim) return;
    const int cnt = (int)min((int64_t)ch, a.n - cb);
    int64_t seg = TABLE ? 0 : (int64_t)a.seg[chunk] - 1;
    bool before = cb > 0 && k[-1] == k[0];
    float acc[V] = {};
    for (int p0 = 0; p0 < cnt; p0 += 8) {
        Pack<T, V> x[8];
        Pack<float, V> old[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int p = min(p0 + j, cnt - 1);
            x[j] = k[p] != a.pad ? stream_in<Pack<T, V>>(grad + (int64_t)v[p] * ld + c) : Pack<T, V>{};
            if (TABLE) old[j] = k[p] != a.pad && k[p + 1] != k[p] ? seq_old<V>(a, k[p], c) : Pack<float, V>{};
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int p = p0 + j;
            if (p >= cnt || k[p] == a.pad) break;
            if (k[p] != k[p - 1]) {
                ++seg;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += x[j].get(e);
            if (p + 1 < cnt && k[p + 1] == k[p]) continue;
            // the row's last position in this chunk
            const bool on = p + 1 == cnt && k[p + 1] == k[p];
            if (before || on) {
                Pack<float, V> o;
                o.put(acc);
                *reinterpret_cast<Pack<float, V>*>(a.partial + (chunk * 2 + (before ? 0 : 1)) * a.dim + c) = o;
            } else {
                seq_emit<V, TABLE>(a, k[p], seg, c, old[j], acc);
            }
            before = false;
        }
    }
}

// Rows that span chunks: the group of the chunk in which the row begins adds the pieces in order -- single chunks up to a workgroup's border,
// whole workgroups of the kernel above, single chunks again -- eight reads in flight; a row of more than SEQ_LONG chunks is left to the whole
// workgroup, whose groups take every (256 >> lg)th piece each and are added in the order of the groups.  A frequent row is a serial chain otherwise: a
// million tokens, the most frequent one in 13 (2,400 pieces of 32), took 1,796 us by one group.
#define SEQ_LONG 24
template <int V, bool TABLE>
__global__ __launch_bounds__(256) void seq_join_kernel(SeqSumArgs a, int lg) {
    __shared__ int n_long, far;
    __shared__ int64_t longs[64];
    __shared__ float stage[256 * V];
    const int ch_ = a.ch, grp = threadIdx.x >> lg, groups = 256 >> lg, l = threadIdx.x & ((1 << lg) - 1);
    const int64_t chunk = (int64_t)blockIdx.x * groups + grp, end = (chunk + 1) * ch_;
    const int c = (int)blockIdx.y * (V << lg) + l * V;
    if (threadIdx.x == 0) n_long = 0;
    __syncthreads();
    auto piece = [&](int64_t ch, int which) { return *reinterpret_cast<const Pack<float, V>*>(a.partial + (ch * 2 + which) * a.dim + c); };
    auto add = [&](float (&acc)[V], const Pack<float, V>& y) {
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += y.get(e);
    };
    // the pieces of chunks first, first + step, .. below last
    auto sum = [&](float (&acc)[V], int64_t first, int64_t last, int64_t step) {
        int64_t ch = first;
        for (; ch + 7 * step < last; ch += 8 * step) {
            Pack<float, V> y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = piece(ch + j * step, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) add(acc, y[j]);
        }
        for (; ch < last; ch += step) add(acc, piece(ch, 0));
    };
    // member `which` of `of` takes its share of the pieces of a row that begins in chunk `first` and whose last chunk is `last`
    auto row = [&](float (&acc)[V], int64_t first, int64_t last, int which, int of) {
        const int64_t up = (first + groups) / groups * groups, from = min(up, last + 1);      // the first border behind `first`
        const int64_t whole = last >= from ? (last - from) / groups : 0, to = from + whole * groups;   // (a workgroup is whole if the next begins with the row)
        if (which == 0) add(acc, piece(first, 1));
        sum(acc, first + 1 + which, from, of);
        sum(acc, from + (int64_t)which * groups, to, (int64_t)of * groups);
        sum(acc, to + which, last + 1, of);
    };
    u32 key = 0;
    if (end < a.n && (key = a.keys[end - 1]) != a.pad && a.keys[end] == key && (chunk == 0 || a.keys[chunk * ch_ - 1] != key)) {
        if ((chunk + 1 + SEQ_LONG) * ch_ < a.n && a.keys[(chunk + 1 + SEQ_LONG) * ch_] == key) {
            if (l == 0) longs[atomicAdd(&n_long, 1)] = chunk;   // (in any order: each is summed by itself)
        } else if (c < a.dim) {
            int64_t last = chunk + 1;
            while ((last + 1) * ch_ < a.n && a.keys[(last + 1) * ch_] == key) ++last;
            float acc[V] = {};
            row(acc, chunk, last, 0, 1);
            seq_emit<V, TABLE>(a, key, TABLE ? 0 : (int64_t)a.seg[chunk + 1] - 1, c, TABLE ? seq_old<V>(a, key, c) : Pack<float, V>{}, acc);
        }
    }
    __syncthreads();
    for (int i = 0; i < n_long; ++i) {
        const int64_t first = longs[i];
        const u32 k = a.keys[(first + 1) * ch_];
        // its last chunk, by a probe a thread at a time: every `step`th chunk behind `lo`, which is the row's
        int64_t lo = first + 1, step = ((a.n - 1) / ch_ - lo + 256) / 256;
        for (;;) {
            if (threadIdx.x == 0) far = 0;
            __syncthreads();
            const int64_t ch = lo + (threadIdx.x + 1) * step;
            if (ch * ch_ < a.n && a.keys[ch * ch_] == k) atomicMax(&far, (int)threadIdx.x + 1);
            __syncthreads();
            lo += far * step;
            __syncthreads();
            if (step == 1) break;
            step = (step + 255) / 256;
        }
        float acc[V] = {};
        if (c < a.dim) row(acc, first, lo, grp, groups);
#pragma unroll
        for (int e = 0; e < V; ++e) stage[e * 256 + threadIdx.x] = acc[e];
        __syncthreads();
        if (grp == 0 && c < a.dim) {
            for (int g = 1; g < groups; ++g)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += stage[e * 256 + (g << lg) + l];
            seq_emit<V, TABLE>(a, k, TABLE ? 0 : (int64_t)a.seg[first + 1] - 1, c, TABLE ? seq_old<V>(a, k, c) : Pack<float, V>{}, acc);
        }
        __syncthreads();
    }
}

void launch_seq_embed_grad(hipStream_t st, const SeqEmbedArgs& a, int bf16, const void* grad, int64_t ld, const SeqEmbedGradBufs& b,
                           int64_t* emb_rows, float* emb_grad, int64_t* n_emb_rows, int64_t capacity, float* table) {
    if (a.n <= 0) {
        if (n_emb_rows) hipLaunchKernelGGL(seq_none_kernel, dim3(1), dim3(1), 0, st, n_emb_rows);
        return;
    }
    const unsigned nb = (unsigned)((a.n + 255) / 256);
    const int64_t chunks = seq_chunks(a.n);
    const int ch = seq_chunk(a.n);
    const bool one = a.n <= SEQ_SORT;
    int at = 0;
    int bits = 1;
    while (bits < 32 && (1ll << bits) <= a.n_rows) ++bits;   // (the padding's key too)
    if (one) {
        hipLaunchKernelGGL(seq_sort_one_kernel, dim3(1), dim3(1024), 0, st, a, bits, ch, b.keys[0], b.vals[0], table ? nullptr : b.counts, b.counts + chunks);
    } else {
        hipLaunchKernelGGL(seq_keys_kernel, dim3(nb), dim3(256), 0, st, a, b.keys[0], b.vals[0]);
        at = launch_radix_sort(st, b.keys[0], b.vals[0], b.keys[1], b.vals[1], a.n, bits, b.hist, nullptr, true) & 1;
    }
    if (!one && !table) {
        hipLaunchKernelGGL(seq_heads_kernel, dim3(nb), dim3(256), 0, st, b.keys[at], a.n, ch, (u32)a.n_rows, b.counts);
        launch_scan_u32(st, b.counts, b.counts, chunks, b.scan_tmp, b.counts + chunks);
    }
    const int v = row_vector(a.dim, ld, grad, bf16 ? 2 : 4, table ? table : emb_grad), lg = lanes_of_row(a.dim, v);
    const SeqSumArgs s{b.keys[at], b.vals[at], b.counts, a.n, capacity, (u32)a.n_rows, a.dim, ch, a.scale, b.partial, emb_rows, emb_grad, table, b.counts + chunks, n_emb_rows, a.status};
    const dim3 grid((unsigned)((chunks + (256 >> lg) - 1) / (256 >> lg)), (unsigned)((a.dim + (v << lg) - 1) / (v << lg)));
    const dim3 join((unsigned)((chunks + (256 >> lg) - 1) / (256 >> lg)), grid.y);
    const size_t lds = (size_t)(256 >> lg) * (2 * ch + 2) * sizeof(u32);
#define SUM(T_, V_)                                                                                                                     \
    do {                                                                                                                                \
        if (table) {                                                                                                                    \
            hipLaunchKernelGGL((seq_sum_kernel<T_, V_, true>), grid, dim3(256), lds, st, s, (const T_*)grad, ld, lg);                   \
            hipLaunchKernelGGL((seq_join_kernel<V_, true>), join, dim3(256), 0, st, s, lg);                                         \
        } else {                                                                                                                        \
            hipLaunchKernelGGL((seq_sum_kernel<T_, V_, false>), grid, dim3(256), lds, st, s, (const T_*)grad, ld, lg);                  \
            hipLaunchKernelGGL((seq_join_kernel<V_, false>), join, dim3(256), 0, st, s, lg);                                        \
        }                                                                                                                               \
    } while (0)
    if (bf16) { if (v == 8) SUM(bf16_t, 8); else if (v == 4) SUM(bf16_t, 4); else SUM(bf16_t, 1); }
    else { if (v == 8) SUM(float, 8); else if (v == 4) SUM(float, 4); else SUM(float, 1); }
#undef SUM
}
