// Cross attention of a user's queries to the states of the user's history, both packed, of any lengths:
//   s_ij = scale q_i . k_j over the keys that count,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
// and its gradients, from lse and delta_i = do_i . o_i:
//   p = exp(s - lse),  ds = p (do . v - delta),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i.
// A key head is shared by `group` query heads: (query, head of the group) pairs are the rows of one product, so that keys and
// values are read once for all of them and the sums of dk and dv run over the group by themselves.
//
// Orientation.  A 32 x 32 block on the matrix cores leaves a lane one column and 16 rows: 8 (i / 4) + 4 (lane / 32) + i % 4.  The
// blocks are formed so that their columns are what the kernel owns (queries in the forward pass and for dq, keys for dk and dv) and
// their rows are what it walks over and sums: the softmax statistics are a lane's own, and the 16 values of a lane are, packed
// four by four, the operand of the next product over these rows without leaving the registers.  The other operand of that product is
// then needed with its contraction index slowest, which a transposing LDS read delivers (bf16) or a plain one (fp32, one value a lane).
// Sums, maxima, exponentials and accumulators are fp32; with bf16 tensors p and ds are rounded to bf16 as operands of their products.
//
// Causal order (CAUSAL): the walks end with the last key that a workgroup's last row sees, or begin with the first row that sees its first key, and the blocks at the diagonal
// compare places; workgroups with the longest walks begin.  Bound: as without it, and what the diagonal's blocks do for nothing (a workgroup's 128 rows or keys).  32 ragged histories of up to
// 2,048, 8 heads over 2 of 128, bf16: 154 to 156 us, 680 TFLOP/s of the products that are seen (without order, twice as many: 266); gradient of 64 of up to 1,024, 8 heads over 4 of 64, a
// mask: 223 us, 265 TFLOP/s (303).
//
// Keys that do not count are taken out twice: their scores never enter a maximum or a sum, and their rows are zero in LDS, whatever
// they hold in memory (0 * NaN would be NaN).  A row without any key has o = 0, lse = -infinity and no gradient.
#include <algorithm>
#include <type_traits>

#include "gm_internal.h"

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define LOG2E 1.44269504088896340736f
#define LN2 0.69314718055994530942f

template <typename T> struct Elem;
template <> struct Elem<bf16_t> {
    enum { E = 8, KC = 16 };          // elements of 16 bytes; contraction length of a fragment (both halves of the wave)
    typedef bf16x8 frag;
    static __device__ __forceinline__ void mma(f32x16& c, frag a, frag b) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Elem<float> {
    enum { E = 4, KC = 8 };
    typedef float4 frag;
    static __device__ __forceinline__ void mma(f32x16& c, frag a, frag b) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, b.x, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, b.y, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, b.z, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, b.w, c, 0, 0, 0);
    }
};

// fp32: whether fragment q holds any of a head's elements (the others are zeros; a fragment of bf16 takes less time than the question).
template <typename T> __device__ __forceinline__ bool used(int q, int dim) { return sizeof(T) == 2 || q * Elem<T>::KC < dim; }

// acc[32 columns of the tile x 32] += (rows 0..31, columns col0.. of the tile)^T * P, P a block as the matrix cores leave it
__device__ __forceinline__ void pack_block(const float (&p)[16], bf16x8 (&f)[2]) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const uint4 u = make_uint4(f2bf2(p[8 * s], p[8 * s + 1]), f2bf2(p[8 * s + 2], p[8 * s + 3]), f2bf2(p[8 * s + 4], p[8 * s + 5]), f2bf2(p[8 * s + 6], p[8 * s + 7]));
        f[s] = __builtin_bit_cast(bf16x8, u);
    }
}
// Columns 32 b .. of a 32-row tile, rows 16 s .. of it in the order in which a lane holds a block's values.  (16 lanes at a time: lane i points at
// four consecutive columns of row i / 4 and receives column i of the four rows.)
__device__ __forceinline__ bf16x8 transposed(const bf16_t* tile, int ld, int b, int s, int lane) {
    typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
    const bf16_t* base = tile + (4 * (lane >> 5) + ((lane & 15) >> 2)) * ld + (lane & 16) + (lane & 3) * 4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(base + (16 * s) * ld + 32 * b));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(base + (16 * s + 8) * ld + 32 * b));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <int NB>
__device__ __forceinline__ void mma_packed_t(f32x16 (&acc)[NB], const bf16_t* tile, int ld, const bf16x8 (&f)[2], int lane) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int s = 0; s < 2; ++s) Elem<bf16_t>::mma(acc[b], transposed(tile, ld, b, s, lane), f[s]);
}
template <int NB>
__device__ __forceinline__ void mma_tile_t(f32x16 (&acc)[NB], const bf16_t* tile, int ld, const float (&p)[16], int lane) {
    bf16x8 f[2];
    pack_block(p, f);
    mma_packed_t<NB>(acc, tile, ld, f, lane);
}
template <int NB>
__device__ __forceinline__ void mma_tile_t(f32x16 (&acc)[NB], const float* tile, int ld, const float (&p)[16], int lane) {
    const float* base = tile + 4 * (lane >> 5) * ld + (lane & 31);
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(base[(8 * (i / 4) + i % 4) * ld + 32 * b], p[i], acc[b], 0, 0, 0);
}
// LDS rows.  bf16: 32 bytes beyond the tile's width, so that the four rows of a transposing read lie 8 banks apart (with 16 bytes two of them
// meet in every bank) and eight consecutive rows of a 16-byte read in eight groups of banks; fp32: an odd number of 16-byte units.
template <typename T, int DP> struct Ld { enum { V = DP + (sizeof(T) == 2 ? 16 : 4) }; };

// What a workgroup works on.
struct Span {
    int64_t q0, nq, k0, nk;
    bool ok;
};
__device__ __forceinline__ Span span_of(const SeqAttendArgs& a, int64_t s) {
    Span p;
    const int64_t q0 = a.q_offsets[s], q1 = a.q_offsets[s + 1], k0 = a.k_offsets[s];
    int64_t k1;
    if (a.k_lengths) {
        const int64_t n = a.k_lengths[s];
        k1 = k0 >= 0 && k0 <= a.n_keys && n <= a.n_keys - k0 ? k0 + n : -1;   // (a length below 0 ends in front of k0)
    } else k1 = a.k_offsets[s + 1];
    p.ok = seq_inside(q0, q1, a.n_queries, a.longest_q) && seq_inside(k0, k1, a.n_keys, a.longest_k) &&
           (s > 0 || (q0 == 0 && (a.k_lengths || k0 == 0))) && (s + 1 < a.n_seqs || (q1 == a.n_queries && (a.k_lengths || k1 == a.n_keys)));
    p.q0 = q0; p.nq = p.ok ? q1 - q0 : 0; p.k0 = k0; p.nk = p.ok ? k1 - k0 : 0;
    if (!p.ok) seq_flag(a.status, SEQ_BAD_OFFSETS);
    return p;
}
// Causal: the last query of a sequence stands at its last key, so query i of nq sees the keys up to i + nk - nq: the new rows of a cache that holds them already,
// or, with queries = keys, every row itself and what comes before it.
__device__ __forceinline__ int64_t seen_by(const Span& sp, int64_t query) { return min(max(query + 1 + sp.nk - sp.nq, (int64_t)0), sp.nk); }   // how many keys
// Whether the i-th of a lane's 16 rows of a block is among the block's first n, for n as in_block makes it.
__device__ __forceinline__ int in_block(int n, int h) { return n - 4 * h; }
__device__ __forceinline__ bool among(int n, int i) { return 8 * (i / 4) + i % 4 < n; }
// The span as the keys from c0 on are seen: the rows in front see none of them, and neither do those that see no key that counts (whose queries may hold
// anything).  Returns by how much a key's number exceeds that of the first of these queries that sees it.
__device__ __forceinline__ int64_t seeing_span(const SeqAttendArgs& a, Span& sp, int64_t c0) {
    int64_t key = c0;
    if (a.key_mask) {
        int64_t first = sp.nk;
        for (int64_t i = 0; i < sp.nk; i += 64) {
            const int64_t k = i + (threadIdx.x & 63);
            const u64 on = __ballot(k < sp.nk && a.key_mask[sp.k0 + min(k, sp.nk - 1)] != 0);
            if (on) {
                first = i + __builtin_ctzll(on);
                break;
            }
        }
        key = max(key, first);
    }
    const int64_t shift = sp.nk - sp.nq, skip = __builtin_amdgcn_readfirstlane((int)min(max(key - shift, (int64_t)0), sp.nq));
    sp.q0 += skip;
    sp.nq -= skip;
    return shift + skip;
}
// What a workgroup is: one of `per` of a (history, key head) pair.  Workgroups are dealt to the eight XCDs in turn: a pair's go to one of
// them, whose cache holds its keys, and the pairs to all in turn; from 32 pairs on, with fewer the XCDs would hold unlike numbers of them.  (64 users of
// 256 queries and 1,024 keys, 8 heads over 2 of 64, bf16, dealt out in order and like this: gradient 173 / 165 us, forward 61 / 59.)
struct Work { int64_t seq; int kvh; int64_t block; };
static int64_t work_grid(const SeqAttendArgs& a, int64_t per) {
    const int64_t pairs = a.n_seqs * a.kv_heads;
    return (pairs < 32 ? pairs : (pairs + 7) / 8 * 8) * per;
}
// id: of the launch's workgroups of this kind; order: the sequences in the order in which they are to begin, or null
__device__ __forceinline__ Work work_of(const SeqAttendArgs& a, u32 id, u32 per, const int32_t* order = nullptr) {
    const u32 pairs = (u32)(a.n_seqs * a.kv_heads);
    const u32 pair = pairs < 32 ? id / per : id / (8 * per) * 8 + (id & 7);
    const u32 block = pairs < 32 ? id % per : (id >> 3) % per;
    const int64_t place = pair < pairs ? (int64_t)(pair / (u32)a.kv_heads) : -1;
    return Work{place >= 0 && order ? (int64_t)order[place] : place, (int)(pair % (u32)a.kv_heads), (int64_t)block};
}
// (tiles on their way in registers need not be waited for, as __syncthreads would)
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00020000);
}
#define NOWHERE (1u << 31)   // an offset behind every tile: reads zeros
// A tile of rows on its way to LDS: each thread's 16-byte pieces, through a buffer that ends with the tile's last row (what lies
// behind it reads as zero).  Row strides are below 2^22 elements: a tile's offsets stay below 2^31.
template <typename T, int DP, int ROWS> struct Stage {
    enum { E = Elem<T>::E, PR = DP / E, N = (ROWS * PR + 255) / 256 };
    u32x4 x[N];
    static __device__ __forceinline__ int row(int i) { return (int)(threadIdx.x + 256 * i) / PR; }
    static __device__ __forceinline__ int col(int i) { return (int)(threadIdx.x + 256 * i) % PR * E; }
    static __device__ __forceinline__ void places(u32 (&at)[N], int64_t ld, int dim) {   // rows that follow each other at a stride
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = row(i) < ROWS && col(i) < dim ? ((u32)row(i) * (u32)ld + (u32)col(i)) * (u32)sizeof(T) : NOWHERE;
    }
    __device__ __forceinline__ void request(__amdgpu_buffer_rsrc_t rs, const u32 (&at)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)at[i], 0, 0);
    }
    template <int LD = Ld<T, DP>::V, typename Keep>
    __device__ __forceinline__ void put(T* tile, Keep&& keep) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (ROWS * PR % 256 == 0 || row(i) < ROWS)
                *reinterpret_cast<u32x4*>(tile + row(i) * LD + col(i)) = keep(i) ? x[i] : u32x4{0u, 0u, 0u, 0u};
    }
};
// Tiles of keys and values on their way, and which of their keys count: with a mask as a float per key, 0 or -infinity, which the product that
// makes the scores starts from.
template <typename T, int DP, int TK, bool MASK> struct KeyTiles {
    typedef Stage<T, DP, TK> S;
    S ks, vs;
    u32 ka[S::N], va[S::N];
    uint8_t kept[MASK ? S::N : 1], mine = 0;
    const T *kp, *vp;
    const uint8_t* mp;
    int64_t ldk, ldv, nk, left = 0;
    __device__ __forceinline__ KeyTiles(const SeqAttendArgs& a, const Span& sp, int kvh, int64_t nk)
        : kp((const T*)a.k + sp.k0 * a.ldk + (int64_t)kvh * a.dim), vp((const T*)a.v + sp.k0 * a.ldv + (int64_t)kvh * a.dim),
          mp(MASK ? a.key_mask + sp.k0 : nullptr), ldk(a.ldk), ldv(a.ldv), nk(nk) {
        S::places(ka, ldk, a.dim);
        S::places(va, ldv, a.dim);
    }
    __device__ __forceinline__ void begin(int64_t t) {   // the first tile; the others are asked for in their order
        kp += t * TK * ldk;
        vp += t * TK * ldv;
        if (MASK) mp += t * TK;
        left = nk - t * TK;
    }
    __device__ __forceinline__ void request() {
        const u32 n = (u32)min(left, (int64_t)TK);
        ks.request(buffer_of(kp, n * (u32)ldk * (u32)sizeof(T)), ka);
        vs.request(buffer_of(vp, n * (u32)ldv * (u32)sizeof(T)), va);
        kp += TK * (u32)ldk;
        vp += TK * (u32)ldv;
        left -= TK;
        if constexpr (MASK) {
            const __amdgpu_buffer_rsrc_t rs = buffer_of(mp, n);
            mp += TK;
#pragma unroll
            for (int i = 0; i < S::N; ++i) kept[i] = __builtin_amdgcn_raw_buffer_load_b8(rs, S::row(i), 0, 0);
            mine = __builtin_amdgcn_raw_buffer_load_b8(rs, threadIdx.x, 0, 0);
        }
    }
    __device__ __forceinline__ void put(T* k, T* v, float* bias) const {
        auto keep = [&](int i) { return !MASK || kept[i] != 0; };
        ks.put(k, keep);
        vs.put(v, keep);
        if (MASK && threadIdx.x < TK) bias[threadIdx.x] = mine ? 0.f : -INFINITY;
    }
    // without a mask: which of the 32 keys of a block of tile t count
    __device__ __forceinline__ u32 bits(int64_t t, int block) const {
        const int64_t n = nk - t * TK - block * 32;
        return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    }
};
// A masked key's score is what its zeros make of the query, plus -infinity: NaN where the query holds NaN or infinities.  That changes nothing where a key counts, whose
// score then is no finite number either; where none of the keys [from, to) does, the sums are taken back.  A row of NaN without a maximum asks the mask.
// Causal: of the keys below the row's own `limit`.
template <bool MASK, bool CAUSAL, int NB>
__device__ __forceinline__ void take_back(const SeqAttendArgs& a, const Span& sp, int64_t from, int64_t to, int64_t limit, float& m, float& l, f32x16 (&acc)[NB]) {
    if (!MASK || !__any(m == -INFINITY && l != l)) return;
    if constexpr (CAUSAL) {
        int64_t first = -1;   // (the row's limit may lie behind `to`)
        for (int64_t i = from; i < to && first < 0; i += 64) {
            const int64_t k = i + (threadIdx.x & 63);
            const u64 on = __ballot(k < to && a.key_mask[sp.k0 + min(k, to - 1)] != 0);
            if (on) first = i + __builtin_ctzll(on);
        }
        if ((first >= 0 && first < limit) || !(m == -INFINITY && l != l)) return;
    } else {
        bool some = false;
        for (int64_t i = from + (threadIdx.x & 63); i < to; i += 64) some |= a.key_mask[sp.k0 + i] != 0;
        if (__any(some)) return;
    }
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
}
// A lane's 16 of a block's 32 floats.
__device__ __forceinline__ f32x16 lane_values(const float* p, int h) {
    f32x16 x;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float4 y = *reinterpret_cast<const float4*>(p + 8 * q + 4 * h);
        x[4 * q] = y.x; x[4 * q + 1] = y.y; x[4 * q + 2] = y.z; x[4 * q + 3] = y.w;
    }
    return x;
}
__device__ __forceinline__ bool bit_of(u32 bits, int h, int i) { return (bits >> (4 * h + 8 * (i / 4) + i % 4)) & 1u; }
template <typename T, int DP>   // a column's fragments straight from memory: element s * KC + half * E ..
__device__ __forceinline__ void load_column(typename Elem<T>::frag (&f)[DP / Elem<T>::KC], const T* p, int dim, int h) {
#pragma unroll
    for (int s = 0; s < DP / Elem<T>::KC; ++s) {
        const int c = s * Elem<T>::KC + h * Elem<T>::E;
        const uint4 u = p && c < dim ? *reinterpret_cast<const uint4*>(p + c) : make_uint4(0u, 0u, 0u, 0u);
        f[s] = __builtin_bit_cast(typename Elem<T>::frag, u);
    }
}
template <typename T> __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d);
template <> __device__ __forceinline__ void store4<float>(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
template <> __device__ __forceinline__ void store4<bf16_t>(bf16_t* p, float a, float b, float c, float d) { *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(a, b), f2bf2(c, d)); }
template <typename T, int NB>   // a column's values, scaled
__device__ __forceinline__ void store_column(T* p, int dim, const f32x16 (&acc)[NB], float scale, int h) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = 32 * b + 8 * q + 4 * h;
            if (c < dim) store4<T>(p + c, scale * acc[b][4 * q], scale * acc[b][4 * q + 1], scale * acc[b][4 * q + 2], scale * acc[b][4 * q + 3]);
        }
}
// The accumulators of waves that share columns, added in the order of the waves into the first of them.
template <int NB>
__device__ __forceinline__ void add_waves(f32x16 (&acc)[NB], float* lds, int lane, int part, int n_parts, int slot) {
    // the parts hand over one after the other through one area per slot: [slot][NB * 16][64]
    float* area = lds + (size_t)slot * NB * 16 * 64;
    for (int w = 1; w < n_parts; ++w) {
        __syncthreads();
        if (part == w)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) area[(b * 16 + i) * 64 + lane] = acc[b][i];
        __syncthreads();
        if (part == 0)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[b][i] += area[(b * 16 + i) * 64 + lane];
    }
}
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);   // {lower, lower}, {upper, upper}
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// One workgroup puts the sequences in order, the longest first, by their keys or by their queries: a workgroup of the kernels below takes as long as
// its sequence is, and the long ones are not to come last.
enum { RANKED = 256 };   // most sequences
__device__ __forceinline__ void rank_sequences(const SeqAttendArgs& a, bool by_keys, int32_t* order) {
    __shared__ __align__(16) u32 len[RANKED];
    const int i = threadIdx.x, n = (int)a.n_seqs;
    const int64_t* off = by_keys ? a.k_offsets : a.q_offsets;
    const u32 mine = i < n ? (u32)min(max(by_keys && a.k_lengths ? a.k_lengths[i] : off[i + 1] - off[i], (int64_t)0), (int64_t)0x7fffffff) : 0u;
    len[i] = mine;
    __syncthreads();
    if (i >= n) return;
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += len[j] > mine || (len[j] == mine && j < i);
    order[rank] = i;
}
// ------------------------------------------------------------------------------------------------ forward
// For the forward pass in front of a large call (the gradient's ranks are made beside its other preparation).
__global__ __launch_bounds__(256) void seq_attend_order_kernel(SeqAttendArgs a) { rank_sequences(a, true, const_cast<int32_t*>(a.order)); }

// Few rows, and fp32.  A workgroup owns 32 * WR rows of one (history, key head); its four waves are WR along the rows and WK = 4 / WR along the keys.
// A tile of 32 * KS * WK keys and values lies in LDS (two of them where that leaves room for two workgroups on a compute unit), the
// next one is on its way in registers.  Bound: with few rows memory, keys and values read once (64 users' slots of 4,096 keys, one query of 8 heads over 2
// key heads of 64, bf16: 19 us, 3.9 TB/s, and 4 for the join; the call 22); fp32 with many rows the matrix
// cores' fp32 rate.
// The maximum that exponents are taken from is raised only when a score exceeds it by more than 2^RAISE would hold: what has been
// summed is rescaled in the first tile and seldom after it (with the maximum of every tile nearly every one moves it for some row).
#define RAISE 8.f
template <typename T, int DP, int WR, int KS> struct AttendTile {
    enum { WK = 4 / WR, TK = 32 * KS * WK, LD = Ld<T, DP>::V, ONE = 2 * TK * LD * (int)sizeof(T) + TK * 4, BUFS = 2 * ONE <= 79 * 1024 ? 2 : 1, BYTES = ONE * BUFS };
};
// Two workgroups on a compute unit, 256 registers a lane, but where the tensors' tiles alone take more.
template <typename T, int DP, int WR, int KS, bool MASK, bool CAUSAL>
__global__ __launch_bounds__(256, DP == 128 && sizeof(T) == 4 ? 1 : 2) void seq_attend_kernel(SeqAttendArgs a) {
    typedef AttendTile<T, DP, WR, KS> Tile;
    constexpr int WK = Tile::WK, TK = Tile::TK, NS = DP / Elem<T>::KC, NB = DP / 32, LD = Tile::LD, BUFS = Tile::BUFS;
    typedef typename Elem<T>::frag frag;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wk = wave / WR;
    const u32 blocks = (u32)((a.longest_q * a.group + 32 * WR - 1) / (32 * WR));
    const Work w = work_of(a, workgroup(), blocks * a.splits);
    if (w.seq < 0) return;
    const int split = (int)(w.block % a.splits), kvh = w.kvh;
    const Span sp = span_of(a, w.seq);
    // (causal: the blocks with the longest way over the keys first)
    const int64_t rows = sp.nq * a.group, r0 = (CAUSAL ? blocks - 1 - w.block / a.splits : w.block / a.splits) * 32 * WR;
    if (!sp.ok || r0 >= rows) return;
    const int heads = a.kv_heads * a.group;
    const int64_t r = r0 + wr * 32 + l32, rc = min(r, rows - 1);
    const int64_t qi = sp.q0 + (u32)rc / (u32)a.group;
    // keys that this row sees, that the wave's first and last row and the workgroup's last do
    const int limit = CAUSAL ? (int)seen_by(sp, qi - sp.q0) : 0, least = __builtin_amdgcn_readfirstlane(limit), most = __builtin_amdgcn_readlane(limit, 31);
    const int64_t nk = CAUSAL ? seen_by(sp, (u32)(min(r0 + 32 * WR, rows) - 1) / (u32)a.group) : sp.nk;
    const int head = kvh * a.group + (int)((u32)rc % (u32)a.group);

    frag qf[NS];
    load_column<T, DP>(qf, r < rows ? (const T*)a.q + qi * a.ldq + (int64_t)head * a.dim : nullptr, a.dim, h);
    // the keys of this workgroup: tiles [t0, t1)
    const int64_t tiles = (nk + TK - 1) / TK, per = (tiles + a.splits - 1) / a.splits;
    const int64_t t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);
    KeyTiles<T, DP, TK, MASK> next(a, sp, kvh, nk);
    f32x16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    float m = -INFINITY, l = 0.f;      // of the row's unscaled scores; l: this lane's share
    const float c2 = a.scale * LOG2E;
    auto tile = [&](int64_t t) { return smem + (BUFS == 2 ? (t - t0) & 1 : 0) * (int)Tile::ONE; };
    auto take = [&](int64_t t) {       // the requested tile to LDS
        T* k = reinterpret_cast<T*>(tile(t));
        next.put(k, k + TK * LD, reinterpret_cast<float*>(k + 2 * TK * LD));
    };
    if (t0 < t1) {
        next.begin(t0);
        next.request();
        take(t0);
        if (t0 + 1 < t1) next.request();
    }
    for (int64_t t = t0; t < t1; ++t) {
        lds_barrier();
        const T* Ks = reinterpret_cast<const T*>(tile(t));
        const T* Vs = Ks + TK * LD;
        const float* bias = reinterpret_cast<const float*>(Vs + TK * LD);
        u32 bits[KS];
#pragma unroll
        for (int j = 0; j < KS; ++j) bits[j] = MASK || CAUSAL ? 0u : next.bits(t, wk * KS + j);
        f32x16 sc[KS];
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const T* krow = Ks + ((wk * KS + j) * 32 + l32) * LD + h * Elem<T>::E;
            sc[j] = MASK ? lane_values(bias + (wk * KS + j) * 32, h) : f32x16{};
#pragma unroll
            for (int q = 0; q < NS; ++q)
                if (used<T>(q, a.dim)) Elem<T>::mma(sc[j], *reinterpret_cast<const frag*>(krow + q * Elem<T>::KC), qf[q]);
        }
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const int first = (int)t * TK + (wk * KS + j) * 32;
            if (CAUSAL && first + 32 > least) {
                const int n = in_block(limit - first, h);
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[j][i] = among(n, i) ? sc[j][i] : -INFINITY;
            }
            if (!CAUSAL && !MASK && bits[j] != ~0u) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[j][i] = bit_of(bits[j], h, i) ? sc[j][i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[j][i]);
        }
        top = fmaxf(top, other_half(top));
        if (__ballot((top - m) * c2 > RAISE)) {
            top = fmaxf(top, m);
            const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * c2);   // (m = -infinity: 0)
            l *= f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[b][i] *= f;
            m = top;
        }
        const float base = m == -INFINITY ? 0.f : m * c2;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(fmaf(sc[j][i], c2, -base));
                l += p[i];
            }
            if (CAUSAL ? (int)t * TK + (wk * KS + j) * 32 < most : MASK || bits[j]) mma_tile_t<NB>(acc, Vs + (wk * KS + j) * 32 * LD, LD, p, lane);
        }
        if (t + 1 < t1) {
            if (BUFS == 1) lds_barrier();
            take(t + 1);
            if (t + 2 < t1) next.request();
        }
    }
    l += other_half(l);
    take_back<MASK, CAUSAL>(a, sp, t0 * TK, min(t1 * TK, nk), limit, m, l, acc);
    if constexpr (WK > 1) {   // the waves' rows over their keys, joined
        float* st = reinterpret_cast<float*>(smem);   // [4 waves][32][2]
        __syncthreads();
        if (h == 0) {
            st[(wave * 32 + l32) * 2] = m;
            st[(wave * 32 + l32) * 2 + 1] = l;
        }
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int o = 0; o < WK; ++o) top = fmaxf(top, st[((o * WR + wr) * 32 + l32) * 2]);
        const float base = top == -INFINITY ? 0.f : top;
        l = 0.f;
#pragma unroll
        for (int o = 0; o < WK; ++o) {
            const float* q = st + ((o * WR + wr) * 32 + l32) * 2;
            l += q[1] * __builtin_amdgcn_exp2f((q[0] - base) * c2);
        }
        const float f = __builtin_amdgcn_exp2f((m - base) * c2);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[b][i] *= f;
        m = top;
        add_waves<NB>(acc, st + 256, lane, wk, WK, wr);
        if (wk) return;
    }
    if (r >= rows) return;
    const int64_t at = qi * heads + head;
    if (a.splits > 1) {
        const int64_t place = split * (a.n_queries * heads) + at;
        if (h == 0) {
            a.part_ml[place * 2] = m;
            a.part_ml[place * 2 + 1] = l;
        }
        if (m > -INFINITY || l > 0.f || l != l) store_column<float, NB>(a.part_o + place * a.dim, a.dim, acc, 1.f, h);
    } else {
        const bool none = m == -INFINITY && l == 0.f;
        store_column<T, NB>((T*)a.out + qi * a.ldout + (int64_t)head * a.dim, a.dim, acc, none ? 0.f : 1.f / l, h);
        if (h == 0) a.lse[at] = none ? -INFINITY : fmaf(__builtin_amdgcn_logf(l), LN2, m * a.scale);
    }
}

// Many rows, bf16: four waves of 32 rows over tiles of 64 keys, in steps of 32.  A step forms the scores of the next 32 keys and adds the
// values of the last 32 on the matrix cores while the vector units take the exponentials of its own: the two have nothing to do with each
// other, and the compiler is told to deal them out alternately.  So keys lie in LDS a step earlier than values, in two buffers each,
// with one barrier a tile: what is put at a tile's beginning (its values, the next one's keys) is read behind the barrier
// after its first step, over what was last read in front of the previous tile's.  Bound: the matrix cores, fed at 740 to 920 TFLOP/s where users are of
// equal sizes (512 queries and 2,048 keys each; a large library product reaches 1,250); 64 ragged users of up to that, heads of 128: 122 to 128 us, 680 to 720 TFLOP/s.
// Products and exponentials one after the other: 158 us.
template <int DP> struct WideTile {
    enum { TK = 64, LDK = DP + 8, LDV = DP == 32 ? 32 : DP + 32, BYTES = 2 * TK * (LDK + LDV) * 2 + 3 * TK * 4 };   // (rows of transposing reads 16 banks apart)
};
template <int DP, bool MASK, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void seq_attend_wide_kernel(SeqAttendArgs a) {
    typedef WideTile<DP> Tile;
    typedef Elem<bf16_t> E;
    typedef Stage<bf16_t, DP, 64> S;
    constexpr int TK = Tile::TK, LDK = Tile::LDK, LDV = Tile::LDV, NS = DP / E::KC, NB = DP / 32;
    extern __shared__ __align__(16) char smem[];
    bf16_t* const Kb = reinterpret_cast<bf16_t*>(smem);
    bf16_t* const Vb = Kb + 2 * TK * LDK;
    float* const Bb = reinterpret_cast<float*>(Vb + 2 * TK * LDV);   // (three of them: a tile's is read a step longer than its keys)
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32 blocks = (u32)((a.longest_q * a.group + 127) / 128);
    const Work w = work_of(a, workgroup(), blocks * a.splits, a.order);
    if (w.seq < 0) return;
    const int split = (int)(w.block % a.splits), kvh = w.kvh;
    const Span sp = span_of(a, w.seq);
    const int64_t rows = sp.nq * a.group, r0 = (CAUSAL ? blocks - 1 - w.block / a.splits : w.block / a.splits) * 128;
    if (!sp.ok || r0 >= rows) return;
    const int heads = a.kv_heads * a.group;
    const int64_t r = r0 + wave * 32 + l32, rc = min(r, rows - 1);
    const int64_t qi = sp.q0 + (u32)rc / (u32)a.group;
    const int64_t nk = CAUSAL ? seen_by(sp, (u32)(min(r0 + 128, rows) - 1) / (u32)a.group) : sp.nk;   // keys that the workgroup's last row sees
    const int limit = CAUSAL ? (int)seen_by(sp, qi - sp.q0) : 0, least = __builtin_amdgcn_readfirstlane(limit);   // of this row, of the wave's first
    const int head = kvh * a.group + (int)((u32)rc % (u32)a.group);
    bf16x8 qf[NS];
    load_column<bf16_t, DP>(qf, r < rows ? (const bf16_t*)a.q + qi * a.ldq + (int64_t)head * a.dim : nullptr, a.dim, h);
    const int64_t tiles = (nk + TK - 1) / TK, per = (tiles + a.splits - 1) / a.splits;
    const int64_t t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);
    const bf16_t* kp = (const bf16_t*)a.k + sp.k0 * a.ldk + (int64_t)kvh * a.dim;
    const bf16_t* vp = (const bf16_t*)a.v + sp.k0 * a.ldv + (int64_t)kvh * a.dim;
    const uint8_t* mp = MASK ? a.key_mask + sp.k0 : nullptr;
    S ks, vs;
    u32 ka[S::N], va[S::N];
    S::places(ka, a.ldk, a.dim);
    S::places(va, a.ldv, a.dim);
    uint8_t keep_k[MASK ? S::N : 1], mine = 0;
    u32 keep_v = 0;   // (a bit for each piece: of the values that are put next)
    auto rest = [&](int64_t t) { return min(nk - t * TK, (int64_t)TK); };
    auto request_k = [&](int64_t t) {
        ks.request(buffer_of(kp + t * TK * a.ldk, rest(t) * a.ldk * 2), ka);
        if constexpr (MASK) {
            const __amdgpu_buffer_rsrc_t rs = buffer_of(mp + t * TK, rest(t));
#pragma unroll
            for (int i = 0; i < S::N; ++i) keep_k[i] = __builtin_amdgcn_raw_buffer_load_b8(rs, S::row(i), 0, 0);
            mine = __builtin_amdgcn_raw_buffer_load_b8(rs, threadIdx.x, 0, 0);
        }
    };
    auto put_k = [&](int64_t t) {
        ks.template put<LDK>(Kb + (t & 1) * TK * LDK, [&](int i) { return !MASK || keep_k[i] != 0; });
        if (MASK && threadIdx.x < TK) Bb[t % 3 * TK + threadIdx.x] = mine ? 0.f : -INFINITY;
    };
    auto keep_values = [&]() {   // of the tile whose keys have been put
        keep_v = 0;
        if constexpr (MASK)
#pragma unroll
            for (int i = 0; i < S::N; ++i) keep_v |= keep_k[i] ? 1u << i : 0u;
    };
    auto request_v = [&](int64_t t) { vs.request(buffer_of(vp + t * TK * a.ldv, rest(t) * a.ldv * 2), va); };
    f32x16 acc[NB], sc, sn;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    sc = sn = f32x16{};
    bf16x8 pf[2] = {};
    float m = -INFINITY, l = 0.f;
    const float c2 = a.scale * LOG2E;
    auto scores = [&](const bf16_t* block, const float* bias) {
        f32x16 x = MASK ? lane_values(bias, h) : f32x16{};
        const bf16_t* krow = block + l32 * LDK + h * E::E;
#pragma unroll
        for (int q = 0; q < NS; ++q) E::mma(x, *reinterpret_cast<const bf16x8*>(krow + q * E::KC), qf[q]);
        return x;
    };
    // a step: kn, bn the next block of keys, vl the last block of values (not in the first step)
    auto step = [&](auto first, const bf16_t* kn, const float* bn, const bf16_t* vl, int64_t t, int j) {
        const int64_t n = rest(t) - j * 32;
        if (CAUSAL ? (int)t * TK + j * 32 + 32 > least : !MASK && n < 32) {
            if constexpr (CAUSAL) {
                const int k = in_block(limit - (int)t * TK - j * 32, h);
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = among(k, i) ? sc[i] : -INFINITY;
            } else {
                const u32 b = n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = bit_of(b, h, i) ? sc[i] : -INFINITY;
            }
        }
        // the next scores beside this step's maximum: a product, the read that a product two later takes, a share of the maximum
        constexpr int MA = NS, MB = 2 * NB, EA = 16 / MA, EB = 16 / MB;
        const bf16_t* krow = kn + l32 * LDK + h * E::E;
        auto kread = [&](int q) { return *reinterpret_cast<const bf16x8*>(krow + q * E::KC); };
        auto vread = [&](int i) { return transposed(vl, LDV, i >> 1, i & 1, lane); };
        bf16x8 kf[MA], vf[MB];
        kf[0] = kread(0);
        kf[1] = kread(1);
        sn = MASK ? lane_values(bn, h) : f32x16{};
        float top = sc[0];
#pragma unroll
        for (int q = 0; q < MA; ++q) {
            if (q + 2 < MA) kf[q + 2] = kread(q + 2);
            else if constexpr (!first.value) vf[q + 2 - MA] = vread(q + 2 - MA);
            E::mma(sn, kf[q], qf[q]);
#pragma unroll
            for (int i = q * EA; i < (q + 1) * EA; ++i) top = fmaxf(top, sc[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
        top = max_halves(top);
        const bool grew = (top - m) * c2 > RAISE;
        const float f = grew ? __builtin_amdgcn_exp2f((m - top) * c2) : 1.f;   // (m = -infinity: 0)
        m = grew ? top : m;
        const float base = m == -INFINITY ? 0.f : m * c2;
        l *= f;
        // the last values beside this step's exponentials
        float p[16];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            if constexpr (!first.value) {
                if (i + 2 < MB) vf[i + 2] = vread(i + 2);
                E::mma(acc[i >> 1], vf[i], pf[i & 1]);
            }
#pragma unroll
            for (int e = i * EB; e < (i + 1) * EB; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], c2, -base));
                l += p[e];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        bf16x8 pn[2];
        pack_block(p, pn);
        asm volatile("" : "+v"(pn[0]), "+v"(pn[1]));   // (here, not behind the branch)
        pf[0] = pn[0];
        pf[1] = pn[1];
        if (!first.value && __ballot(grew)) {   // (what was added in this step was still relative to the former maximum)
#pragma unroll
            for (int q = 0; q < NB; ++q)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[q][i] *= f;
        }
        sc = sn;
    };
    if (t0 < t1) {
        request_k(t0);
        request_v(t0);
        put_k(t0);
        keep_values();
        if (t0 + 1 < t1) request_k(t0 + 1);
        lds_barrier();
        sc = scores(Kb + (t0 & 1) * TK * LDK, Bb + t0 % 3 * TK);
    }
    for (int64_t t = t0; t < t1; ++t) {
        vs.template put<LDV>(Vb + (t & 1) * TK * LDV, [&](int i) { return !MASK || (keep_v >> i & 1u); });
        if (t + 1 < t1) {
            put_k(t + 1);
            keep_values();
            request_v(t + 1);
            if (t + 2 < t1) request_k(t + 2);
        }
        const bf16_t* K0 = Kb + (t & 1) * TK * LDK;
        const bf16_t* V0 = Vb + (t & 1) * TK * LDV;
        const bf16_t* K1 = Kb + ((t + 1) & 1) * TK * LDK;    // (behind the last tile: read, never used)
        const bf16_t* V1 = Vb + ((t + 1) & 1) * TK * LDV;
        const float *B0 = Bb + t % 3 * TK, *B1 = Bb + (t + 1) % 3 * TK;
        if (t == t0) step(std::true_type(), K0 + 32 * LDK, B0 + 32, nullptr, t, 0);
        else step(std::false_type(), K0 + 32 * LDK, B0 + 32, V1 + 32 * LDV, t, 0);
        lds_barrier();
        step(std::false_type(), K1, B1, V0, t, 1);
    }
    if (t0 < t1) mma_packed_t<NB>(acc, Vb + ((t1 - 1) & 1) * TK * LDV + 32 * LDV, LDV, pf, lane);
    l += other_half(l);
    take_back<MASK, CAUSAL>(a, sp, t0 * TK, min(t1 * TK, nk), limit, m, l, acc);
    if (r >= rows) return;
    const int64_t at = qi * heads + head;
    if (a.splits > 1) {
        const int64_t place = split * (a.n_queries * heads) + at;
        if (h == 0) {
            a.part_ml[place * 2] = m;
            a.part_ml[place * 2 + 1] = l;
        }
        if (m > -INFINITY || l > 0.f || l != l) store_column<float, NB>(a.part_o + place * a.dim, a.dim, acc, 1.f, h);
    } else {
        const bool none = m == -INFINITY && l == 0.f;
        store_column<bf16_t, NB>((bf16_t*)a.out + qi * a.ldout + (int64_t)head * a.dim, a.dim, acc, none ? 0.f : 1.f / l, h);
        if (h == 0) a.lse[at] = none ? -INFINITY : fmaf(__builtin_amdgcn_logf(l), LN2, m * a.scale);
    }
}

// The splits of a row, joined by exp(m_s - m): a wave a (query, head), a lane a split for the statistics and two elements for the sum, eight splits' reads in
// flight.  Bound: latency.
enum { SPLITS = 64 };   // at most
template <typename T>
__global__ __launch_bounds__(256) void seq_attend_join_kernel(SeqAttendArgs a) {
    const int heads = a.kv_heads * a.group, lane = threadIdx.x & 63;
    const int64_t n = a.n_queries * heads, at = (int64_t)workgroup() * 4 + (threadIdx.x >> 6);
    if (at >= n) return;
    const float c2 = a.scale * LOG2E;
    const float2 ml = lane < a.splits ? *reinterpret_cast<const float2*>(a.part_ml + (lane * n + at) * 2) : make_float2(-INFINITY, 0.f);
    float m = ml.x;
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -INFINITY ? 0.f : m;
    const float w = __builtin_amdgcn_exp2f((ml.x - base) * c2);
    float total = ml.y * w;
#pragma unroll
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    const bool none = m == -INFINITY && total == 0.f;
    const u64 some = __ballot(!(ml.x == -INFINITY && ml.y == 0.f));   // (the others wrote no values)
    const int c = lane * 2;
    float2 o = make_float2(0.f, 0.f);
    const float* p = a.part_o + at * a.dim + (c < a.dim ? c : 0);
    for (int s0 = 0; s0 < a.splits; s0 += 8) {
        float2 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = s0 + j < a.splits && (some >> (s0 + j) & 1) ? *reinterpret_cast<const float2*>(p + (s0 + j) * n * a.dim) : make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = __shfl(w, (s0 + j) & 63);
            if (some >> (s0 + j) & 1) o = make_float2(fmaf(f, x[j].x, o.x), fmaf(f, x[j].y, o.y));
        }
    }
    const float f = none ? 0.f : 1.f / total;
    if (c < a.dim) {
        Pack<T, 2> y;
        const float v[2] = {f * o.x, f * o.y};
        y.put(v);
        *reinterpret_cast<Pack<T, 2>*>((T*)a.out + at / heads * a.ldout + (at % heads) * a.dim + c) = y;
    }
    if (lane == 0) a.lse[at] = none ? -INFINITY : fmaf(__builtin_amdgcn_logf(total), LN2, m * a.scale);
}

// ------------------------------------------------------------------------------------------------ gradient
// What the gradient needs of every (query, head): lse * log2(e) (0 for a row without keys) and delta = dout . o; 16 lanes each.  Bound: memory, o and dout
// read once (64 ragged users of up to 256 queries x 8 heads of 64: 7 of the call's 96 us; formed in the walk over the rows instead, once a block of keys,
// the gradient of long sequences takes 7 to 20 % longer).
template <typename T>
__global__ __launch_bounds__(256) void seq_attend_stat_kernel(SeqAttendArgs a, u32 ranks) {
    const u32 id = workgroup();
    if (id < ranks) {
        rank_sequences(a, id == 0, const_cast<int32_t*>(a.order) + id * RANKED);
        return;
    }
    const int heads = a.kv_heads * a.group, l = threadIdx.x & 15;
    const int64_t at = (int64_t)(id - ranks) * 16 + (threadIdx.x >> 4);
    if (at >= a.n_queries * heads) return;
    const T* o = (const T*)a.o + at / heads * a.ldo + (at % heads) * a.dim;
    const T* d = (const T*)a.dout + at / heads * a.lddo + (at % heads) * a.dim;
    float sum = 0.f;
    for (int c = l * 4; c < a.dim; c += 64) {
        const Pack<T, 4> x = *reinterpret_cast<const Pack<T, 4>*>(o + c), y = *reinterpret_cast<const Pack<T, 4>*>(d + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = fmaf(x.get(e), y.get(e), sum);
    }
#pragma unroll
    for (int k = 8; k; k >>= 1) sum += __shfl_xor(sum, k);
    const float lse = a.lse[at];
    if (l == 0) a.stat[at] = make_float2(lse == -INFINITY ? 0.f : lse * LOG2E, sum);
}

// dq of few rows, of heads of 32 and of fp32: the forward kernel's layout; a wave's columns are 32 rows, it walks over the keys.  Bound: the latency of a
// tile's five steps (fp32: of the matrix cores' rate, an eighth of that of bf16).
template <typename T, int DP, int WR, int KS, bool MASK, bool CAUSAL>
__device__ __forceinline__ void dq_block(const SeqAttendArgs& a, char* smem, u32 id) {
    typedef AttendTile<T, DP, WR, KS> Tile;
    constexpr int WK = Tile::WK, TK = Tile::TK, NS = DP / Elem<T>::KC, NB = DP / 32, LD = Tile::LD, BUFS = Tile::BUFS;
    typedef typename Elem<T>::frag frag;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wk = wave / WR;
    const u32 blocks = (u32)((a.longest_q * a.group + 32 * WR - 1) / (32 * WR));
    const Work w = work_of(a, id, blocks, a.order);
    if (w.seq < 0) return;
    const int kvh = w.kvh;
    const Span sp = span_of(a, w.seq);
    const int64_t rows = sp.nq * a.group, r0 = (CAUSAL ? blocks - 1 - w.block : w.block) * 32 * WR;
    if (!sp.ok || r0 >= rows) return;
    const int heads = a.kv_heads * a.group;
    const int64_t r = r0 + wr * 32 + l32, rc = min(r, rows - 1);
    const int64_t qi = sp.q0 + (u32)rc / (u32)a.group;
    const int head = kvh * a.group + (int)((u32)rc % (u32)a.group);
    frag qf[NS], df[NS];
    load_column<T, DP>(qf, r < rows ? (const T*)a.q + qi * a.ldq + (int64_t)head * a.dim : nullptr, a.dim, h);
    load_column<T, DP>(df, r < rows ? (const T*)a.dout + qi * a.lddo + (int64_t)head * a.dim : nullptr, a.dim, h);
    const float2 stat = a.stat[qi * heads + head];
    const bool none = (MASK || CAUSAL) && a.lse[qi * heads + head] == -INFINITY;   // (no key counts: no gradient, whatever the row holds)
    const float c2 = a.scale * LOG2E, base = stat.x, delta = stat.y;
    const int limit = CAUSAL ? (int)seen_by(sp, qi - sp.q0) : 0, least = __builtin_amdgcn_readfirstlane(limit), most = __builtin_amdgcn_readlane(limit, 31);
    const int64_t nk = CAUSAL ? seen_by(sp, (u32)(min(r0 + 32 * WR, rows) - 1) / (u32)a.group) : sp.nk;
    const int64_t tiles = (nk + TK - 1) / TK;
    KeyTiles<T, DP, TK, MASK> next(a, sp, kvh, nk);
    f32x16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    auto tile = [&](int64_t t) { return smem + (BUFS == 2 ? t & 1 : 0) * (int)Tile::ONE; };
    auto take = [&](int64_t t) {
        T* k = reinterpret_cast<T*>(tile(t));
        next.put(k, k + TK * LD, reinterpret_cast<float*>(k + 2 * TK * LD));
    };
    if (tiles) {
        next.begin(0);
        next.request();
        take(0);
        if (1 < tiles) next.request();
    }
    for (int64_t t = 0; t < tiles; ++t) {
        lds_barrier();
        const T* Ks = reinterpret_cast<const T*>(tile(t));
        const T* Vs = Ks + TK * LD;
        const float* bias = reinterpret_cast<const float*>(Vs + TK * LD);
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const int row0 = (wk * KS + j) * 32;
            const u32 bits = MASK || CAUSAL ? ~0u : next.bits(t, wk * KS + j);
            const int first = (int)t * TK + row0;
            if (CAUSAL ? first >= most : !bits) continue;
            f32x16 sc = MASK ? lane_values(bias + row0, h) : f32x16{}, dp = f32x16{};
#pragma unroll
            for (int q = 0; q < NS; ++q) {
                if (!used<T>(q, a.dim)) break;
                Elem<T>::mma(sc, *reinterpret_cast<const frag*>(Ks + (row0 + l32) * LD + h * Elem<T>::E + q * Elem<T>::KC), qf[q]);
                Elem<T>::mma(dp, *reinterpret_cast<const frag*>(Vs + (row0 + l32) * LD + h * Elem<T>::E + q * Elem<T>::KC), df[q]);
            }
            float ds[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c2, -base)) * (dp[i] - delta);   // (masked: exp2(-infinity))
            if (CAUSAL && first + 32 > least) {
                const int n = in_block(limit - first, h);
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] = among(n, i) ? ds[i] : 0.f;
            }
            if (!CAUSAL && !MASK && bits != ~0u) {
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] = bit_of(bits, h, i) ? ds[i] : 0.f;
            }
            mma_tile_t<NB>(acc, Ks + row0 * LD, LD, ds, lane);
        }
        if (t + 1 < tiles) {
            if (BUFS == 1) lds_barrier();
            take(t + 1);
            if (t + 2 < tiles) next.request();
        }
    }
    if constexpr (WK > 1) {
        add_waves<NB>(acc, reinterpret_cast<float*>(smem), lane, wk, WK, wr);
        if (wk) return;
    }
    if (none) {
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
    }
    if (r < rows) store_column<T, NB>((T*)a.dq + qi * a.lddq + (int64_t)head * a.dim, a.dim, acc, a.scale, h);
}

// dk, dv: a workgroup owns 32 * WC keys of one (history, key head), a wave's columns are 32 keys, it walks over the rows;
// WC waves along the keys, 4 / WC along the rows.  37 ragged users of up to 61 queries and 243 keys, 4 heads of 40, fp32: 28.6 us the whole gradient.
template <typename T, int DP, int WC, int RS> struct DkvTile {
    enum { WW = 4 / WC, TR = 32 * RS * WW, LD = Ld<T, DP>::V, ONE = 2 * TR * LD * (int)sizeof(T) + 2 * TR * 4, BUFS = 2 * ONE <= 79 * 1024 ? 2 : 1, BYTES = ONE * BUFS };
};
template <typename T, int DP, int WC, int RS, bool CAUSAL>
__device__ __forceinline__ void dkv_block(const SeqAttendArgs& a, char* smem, u32 id) {
    typedef DkvTile<T, DP, WC, RS> Tile;
    constexpr int WW = Tile::WW, TR = Tile::TR, NS = DP / Elem<T>::KC, NB = DP / 32, LD = Tile::LD, BUFS = Tile::BUFS;
    typedef typename Elem<T>::frag frag;
    typedef Stage<T, DP, TR> S;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wc = wave % WC, ww = wave / WC;
    const Work w = work_of(a, id, (u32)((a.longest_k + 32 * WC - 1) / (32 * WC)), a.order ? a.order + RANKED : nullptr);
    if (w.seq < 0) return;
    const int kvh = w.kvh, heads = a.kv_heads * a.group;
    Span sp = span_of(a, w.seq);
    const int64_t c0 = w.block * 32 * WC;
    if (!sp.ok || c0 >= sp.nk) return;
    const int64_t key = c0 + wc * 32 + l32;
    // causal: the rows in front of `above` do not see this key; up to `most` they do not see all of the wave's
    const int64_t shift = CAUSAL ? seeing_span(a, sp, c0) : 0;
    const int above = (int)min(max((key - shift) * a.group, (int64_t)0), sp.nq * a.group), most = __builtin_amdgcn_readlane(above, 31);
    const int rows = (int)(sp.nq * a.group);
    const bool in = key < sp.nk, on = in && (!a.key_mask || a.key_mask[sp.k0 + key]);
    frag kf[NS], vf[NS];   // (zeros where the key does not count: its column of scores, and what is made of it, is left out at the end)
    load_column<T, DP>(kf, on ? (const T*)a.k + (sp.k0 + key) * a.ldk + (int64_t)kvh * a.dim : nullptr, a.dim, h);
    load_column<T, DP>(vf, on ? (const T*)a.v + (sp.k0 + key) * a.ldv + (int64_t)kvh * a.dim : nullptr, a.dim, h);
    const float c2 = a.scale * LOG2E;
    S qs, dos;
    float2 stat = make_float2(0.f, 0.f);
    // row r of the product is query r / group, head r % group; a tile's offsets are taken from its first query
    auto request = [&](int t) {
        const u32 g = (u32)a.group, first = (u32)(t * TR) / g, last = ((u32)min(rows, (t + 1) * TR) - 1u) / g, n = last - first + 1u;
        const int64_t head0 = (int64_t)kvh * a.group * a.dim;
        u32 qa[S::N], da[S::N];
#pragma unroll
        for (int i = 0; i < S::N; ++i) {
            const u32 r = (u32)(t * TR + S::row(i)), q = r / g, in_row = (r - q * g) * (u32)a.dim + (u32)S::col(i);
            const bool ok = S::row(i) < TR && (int)r < rows && S::col(i) < a.dim;
            qa[i] = ok ? ((q - first) * (u32)a.ldq + in_row) * (u32)sizeof(T) : NOWHERE;
            da[i] = ok ? ((q - first) * (u32)a.lddo + in_row) * (u32)sizeof(T) : NOWHERE;
        }
        qs.request(buffer_of((const T*)a.q + (sp.q0 + first) * a.ldq + head0, n * a.ldq * (int64_t)sizeof(T)), qa);
        dos.request(buffer_of((const T*)a.dout + (sp.q0 + first) * a.lddo + head0, n * a.lddo * (int64_t)sizeof(T)), da);
        if (threadIdx.x < TR) {
            const u32 r = (u32)(t * TR) + threadIdx.x, q = r / g;
            const int64_t at = (sp.q0 + q) * heads + kvh * a.group + (r - q * g);
            stat = (int)r < rows ? a.stat[at] : make_float2(0.f, 0.f);
        }
    };
    auto tile = [&](int t) { return smem + (BUFS == 2 ? t & 1 : 0) * (int)Tile::ONE; };
    auto take = [&](int t) {
        T* q = reinterpret_cast<T*>(tile(t));
        float* ls = reinterpret_cast<float*>(q + 2 * TR * LD);
        auto all = [](int) { return true; };
        qs.put(q, all);
        dos.put(q + TR * LD, all);
        if (threadIdx.x < TR) {
            ls[threadIdx.x] = stat.x;
            ls[TR + threadIdx.x] = stat.y;
        }
    };
    f32x16 ak[NB], av[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) { ak[b] = f32x16{}; av[b] = f32x16{}; }
    const int tiles = (rows + TR - 1) / TR;
    if (tiles) {
        request(0);
        take(0);
        if (1 < tiles) request(1);
    }
    for (int t = 0; t < tiles; ++t) {
        lds_barrier();
        const T* Qs = reinterpret_cast<const T*>(tile(t));
        const T* Ds = Qs + TR * LD;
        const float* Ls = reinterpret_cast<const float*>(Ds + TR * LD);
        const float* Es = Ls + TR;
#pragma unroll
        for (int j = 0; j < RS; ++j) {
            const int row0 = (ww * RS + j) * 32;
            if (t * TR + row0 >= rows) break;
            f32x16 sc = f32x16{}, dp = f32x16{};
#pragma unroll
            for (int q = 0; q < NS; ++q) {
                if (!used<T>(q, a.dim)) break;
                Elem<T>::mma(sc, *reinterpret_cast<const frag*>(Qs + (row0 + l32) * LD + h * Elem<T>::E + q * Elem<T>::KC), kf[q]);
                Elem<T>::mma(dp, *reinterpret_cast<const frag*>(Ds + (row0 + l32) * LD + h * Elem<T>::E + q * Elem<T>::KC), vf[q]);
            }
            float p[16], ds[16];
            const f32x16 lv = lane_values(Ls + row0, h), dv = lane_values(Es + row0, h);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c2, -lv[i]));
                ds[i] = p[i] * (dp[i] - dv[i]);
            }
            if (CAUSAL && t * TR + row0 < most) {
                const int n = in_block(above - t * TR - row0, h);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[i] = among(n, i) ? 0.f : p[i];
                    ds[i] = among(n, i) ? 0.f : ds[i];
                }
            }
            mma_tile_t<NB>(av, Ds + row0 * LD, LD, p, lane);
            mma_tile_t<NB>(ak, Qs + row0 * LD, LD, ds, lane);
        }
        if (t + 1 < tiles) {
            if (BUFS == 1) lds_barrier();
            take(t + 1);
            if (t + 2 < tiles) request(t + 2);
        }
    }
    if constexpr (WW > 1) {
        add_waves<NB>(ak, reinterpret_cast<float*>(smem), lane, ww, WW, wc);
        add_waves<NB>(av, reinterpret_cast<float*>(smem), lane, ww, WW, wc);
        if (ww) return;
    }
    if (!in) return;
    if (!on) {
#pragma unroll
        for (int b = 0; b < NB; ++b) { ak[b] = f32x16{}; av[b] = f32x16{}; }
    }
    store_column<T, NB>((T*)a.dk + (sp.k0 + key) * a.lddk + (int64_t)kvh * a.dim, a.dim, ak, a.scale, h);
    store_column<T, NB>((T*)a.dv + (sp.k0 + key) * a.lddv + (int64_t)kvh * a.dim, a.dim, av, 1.f, h);
}

// Many rows or keys, bf16: either half of the gradient as a walk in steps of 32 over the rows (KV: dk and dv of 128 keys) or the keys (dq of 128 rows).
// With X, Y the two matrices walked over (queries and dout, or keys and values) and the wave's columns in registers, step j takes
// the exponentials of block j on the vector units while the matrix cores add up block j - 1 (dk += X^T ds, dv += Y^T p), and then forms the two products
// of block j + 1.  A block of X and Y lies in one of four places of LDS: one is read by rows, one transposed, one is being filled and one
// idle, so one barrier a step is enough; what is filled in was asked for two steps before.  16-byte units of a row are stored
// at unit ^ turn(row): the 16 rows of a row-wise read and the four of a transposing one lie in banks of their own, without padding.
// Bound: issue slots -- a block's seven products (the scores are formed in both halves), its exponentials and the packing of p and ds take turns with the
// matrix cores.  Equal users: 510 to 640 TFLOP/s of the five products that no form can leave out; 64 ragged users of up to 256 queries and 1,024 keys,
// 8 heads over 4 of 64, a mask: 94 to 96 us (tiles without the overlap 117).
template <int DP> struct Walk {
    enum { UNITS = DP / 8, N = DP / 64, HALF = 32 * DP, SLOT = 2 * HALF * 2 + 64 * 4, BYTES = 4 * SLOT };
    static __device__ __forceinline__ int turn(int row) {
        return DP == 64 ? ((row >> 1) & 1) << 2 | ((row >> 2) & 3) : (row & 3) << 2 | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int row, int unit) { return row * DP + (unit ^ turn(row)) * 8; }
};
template <int DP, bool KV, bool MASK, bool CAUSAL>
__device__ __forceinline__ void walk_block(const SeqAttendArgs& a, char* smem, u32 id) {
    typedef Walk<DP> W;
    typedef Elem<bf16_t> E;
    constexpr int NS = DP / E::KC, NB = DP / 32, N = W::N;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32 blocks = (u32)(((KV ? a.longest_k : a.longest_q * a.group) + 127) / 128);
    const Work w = work_of(a, id, blocks, KV && a.order ? a.order + RANKED : a.order);
    if (w.seq < 0) return;
    const int kvh = w.kvh, heads = a.kv_heads * a.group;
    Span sp = span_of(a, w.seq);
    const u32 g = (u32)a.group;
    const int64_t c00 = (CAUSAL && !KV ? blocks - 1 - w.block : w.block) * 128;
    if (!sp.ok || c00 >= (KV ? sp.nk : sp.nq * a.group)) return;
    const int c0 = (int)c00, col = c0 + wave * 32 + l32;
    // causal: of the rows walked over, those in front of `above` do not see this key; of the keys, this row does not see those from `above` on.  `edge`: where the
    // wave's first differ
    int above = 0, edge = 0;
    if (CAUSAL && KV) {
        const int64_t shift = seeing_span(a, sp, c0);
        above = (int)min(max((col - shift) * a.group, (int64_t)0), sp.nq * a.group);
        edge = __builtin_amdgcn_readlane(above, 31);
    }
    const int rows = (int)(sp.nq * a.group), cols = KV ? (int)sp.nk : rows;
    if (CAUSAL && !KV) {
        above = (int)seen_by(sp, (u32)min(col, rows - 1) / g);
        edge = __builtin_amdgcn_readfirstlane(above);
    }
    const int n = KV ? rows : CAUSAL ? __builtin_amdgcn_readfirstlane((int)seen_by(sp, (u32)(min(c0 + 128, rows) - 1) / g)) : (int)sp.nk;
    const bool in = col < cols;
    // the columns
    const int64_t head0 = (int64_t)kvh * a.group * a.dim, key0 = (int64_t)kvh * a.dim;
    const u32 cq = (u32)min(col, cols - 1) / g;
    const int64_t query = sp.q0 + cq, key = sp.k0 + min(col, cols - 1);
    const int head = kvh * a.group + (int)((u32)min(col, cols - 1) - cq * g);
    const bool on = in && (!KV || !a.key_mask || a.key_mask[key]);
    bf16x8 xf[NS], yf[NS];
    load_column<bf16_t, DP>(xf, !on ? nullptr : KV ? (const bf16_t*)a.k + key * a.ldk + key0 : (const bf16_t*)a.q + query * a.ldq + (int64_t)head * a.dim, a.dim, h);
    load_column<bf16_t, DP>(yf, !on ? nullptr : KV ? (const bf16_t*)a.v + key * a.ldv + key0 : (const bf16_t*)a.dout + query * a.lddo + (int64_t)head * a.dim, a.dim, h);
    const float c2 = a.scale * LOG2E;
    float col_base = 0.f, col_delta = 0.f;
    bool none = KV && !on;   // (a key or a row that has no gradient, whatever was made of it)
    if (!KV) {
        const float2 stat = a.stat[query * heads + head];
        col_base = stat.x;
        col_delta = stat.y;
        none = (MASK || CAUSAL) && a.lse[query * heads + head] == -INFINITY;
    }
    // the blocks on their way: a thread's 16-byte pieces of X and Y, two blocks ahead
    const int64_t ldx = KV ? a.ldq : a.ldk, ldy = KV ? a.lddo : a.ldv;
    const bf16_t* xp = KV ? (const bf16_t*)a.q + sp.q0 * ldx + head0 : (const bf16_t*)a.k + sp.k0 * ldx + key0;
    const bf16_t* yp = KV ? (const bf16_t*)a.dout + sp.q0 * ldy + head0 : (const bf16_t*)a.v + sp.k0 * ldy + key0;
    const u32 group = KV ? g : 1u;
    const bool even = 32u % group == 0;      // a block begins with a query's first head
    auto prow = [&](int i) { return (int)(threadIdx.x + 256 * i) / W::UNITS; };
    auto punit = [&](int i) { return (int)(threadIdx.x + 256 * i) % W::UNITS; };
    u32 xa[N], ya[N];
    auto places = [&](u32 r0, u32 first) {   // of the block that begins with row r0; offsets from query `first`
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32 r = r0 + (u32)prow(i), q = r / group, in_row = (r - q * group) * (u32)a.dim + 8u * (u32)punit(i);
            const bool ok = 8 * punit(i) < a.dim && (int)r < n;
            xa[i] = ok ? ((q - first) * (u32)ldx + in_row) * 2u : NOWHERE;
            ya[i] = ok ? ((q - first) * (u32)ldy + in_row) * 2u : NOWHERE;
        }
    };
    // (the offsets of the first block, without its end: they are every block's where `even`, whose buffer ends with its last row)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const u32 r = (u32)prow(i), q = r / group, in_row = (r - q * group) * (u32)a.dim + 8u * (u32)punit(i);
        const bool ok = 8 * punit(i) < a.dim;
        xa[i] = ok ? (q * (u32)ldx + in_row) * 2u : NOWHERE;
        ya[i] = ok ? (q * (u32)ldy + in_row) * 2u : NOWHERE;
    }
    // (blocks are asked for in their order: what moves from one to the next is added, not multiplied out)
    const int steps = (n + 31) / 32;
    const u32 tail = (u32)(n - 32 * (steps - 1)) / group;                 // queries (or keys) of the last block
    const u32 x_full = 32u / group * (u32)ldx * 2u, y_full = 32u / group * (u32)ldy * 2u, x_tail = tail * (u32)ldx * 2u, y_tail = tail * (u32)ldy * 2u;
    const char *xn = reinterpret_cast<const char*>(xp), *yn = reinterpret_cast<const char*>(yp);
    const char* sn = KV ? reinterpret_cast<const char*>(a.stat + sp.q0 * heads + kvh * a.group) : MASK ? reinterpret_cast<const char*>(a.key_mask + sp.k0) : nullptr;
    const u32 s_step = KV ? 32u / group * (u32)heads * 8u : 32u;          // (statistics of a block's rows, or its mask)
    const u32 sq = (u32)l32 / group, s_at = threadIdx.x < 32 ? (sq * (u32)heads + (u32)l32 - sq * group) * 8u : NOWHERE;
    u32x4 xs[2][N], ys[2][N];
    float2 st[2] = {};                              // KV: of row tid
    uint8_t keep[2][MASK && !KV ? N : 1], mine[2];
    auto request = [&](int j, auto d) {
        const bool full = j + 1 < steps;
        u32 xb = full ? x_full : x_tail, yb = full ? y_full : y_tail, sb = full ? s_step : KV ? tail * (u32)heads * 8u : tail, sa = s_at;
        if (!even) {   // a block begins inside a query: its offsets are its own
            const u32 r0 = (u32)j * 32u, first = r0 / group, count = ((u32)min(n, (int)r0 + 32) - 1u) / group - first + 1u;
            places(r0, first);
            xn = reinterpret_cast<const char*>(xp + first * ldx);
            yn = reinterpret_cast<const char*>(yp + first * ldy);
            xb = count * (u32)ldx * 2u;
            yb = count * (u32)ldy * 2u;
            sn = reinterpret_cast<const char*>(a.stat + (sp.q0 + first) * heads + kvh * a.group);
            const u32 r = r0 + (u32)l32, q = r / group;
            sb = count * (u32)heads * 8u;
            sa = threadIdx.x < 32 && (int)r < n ? ((q - first) * (u32)heads + r - q * group) * 8u : NOWHERE;
        }
        const __amdgpu_buffer_rsrc_t rx = buffer_of(xn, xb), ry = buffer_of(yn, yb);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            xs[d][i] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)xa[i], 0, 0);
            ys[d][i] = __builtin_amdgcn_raw_buffer_load_b128(ry, (int)ya[i], 0, 0);
        }
        if constexpr (KV) {
            if (wave == 0) st[d] = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(buffer_of(sn, sb), (int)sa, 0, 0));
        } else if constexpr (MASK) {
            const __amdgpu_buffer_rsrc_t rs = buffer_of(sn, sb);
#pragma unroll
            for (int i = 0; i < N; ++i) keep[d][i] = __builtin_amdgcn_raw_buffer_load_b8(rs, prow(i), 0, 0);
            mine[d] = __builtin_amdgcn_raw_buffer_load_b8(rs, threadIdx.x, 0, 0);
        }
        xn += x_full;
        yn += y_full;
        if (KV || MASK) sn += s_step;
    };
    auto slot = [&](int j) { return reinterpret_cast<bf16_t*>(smem + (j & 3) * (int)W::SLOT); };
    auto stats = [&](int j) { return reinterpret_cast<float*>(slot(j) + 2 * W::HALF); };
    auto put = [&](int j, auto d) {
        bf16_t* x = slot(j);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool kept = KV || !MASK || keep[d][MASK && !KV ? i : 0] != 0;
            *reinterpret_cast<u32x4*>(x + W::at(prow(i), punit(i))) = kept ? xs[d][i] : u32x4{0u, 0u, 0u, 0u};
            *reinterpret_cast<u32x4*>(x + W::HALF + W::at(prow(i), punit(i))) = kept ? ys[d][i] : u32x4{0u, 0u, 0u, 0u};
        }
        if constexpr (KV) {
            if (threadIdx.x < 32) {
                stats(j)[threadIdx.x] = st[d].x;
                stats(j)[32 + threadIdx.x] = st[d].y;
            }
        } else if (threadIdx.x < 32) {
            stats(j)[threadIdx.x] = MASK ? (mine[d] ? 0.f : -INFINITY) : j * 32 + (int)threadIdx.x < n ? 0.f : -INFINITY;
        }
    };
    // LDS places of this lane inside a half
    int row_at[NS], tr_at[2 * NB];
#pragma unroll
    for (int q = 0; q < NS; ++q) row_at[q] = W::at(l32, 2 * q + h);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            tr_at[2 * b + k] = W::at(8 * k + 4 * h + ((lane & 15) >> 2), 4 * b + ((lane & 16) >> 3) + ((lane & 3) >> 1)) + (lane & 1) * 4;
    auto by_row = [&](const bf16_t* half, int q) { return *reinterpret_cast<const bf16x8*>(half + row_at[q]); };
    auto across = [&](const bf16_t* half, int b, int s) {
        typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(half + tr_at[2 * b] + 16 * s * DP));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(half + tr_at[2 * b + 1] + 16 * s * DP));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x16 ax[NB], ay[KV ? NB : 1], sc, dp;
#pragma unroll
    for (int b = 0; b < NB; ++b) ax[b] = f32x16{};
#pragma unroll
    for (int b = 0; b < (KV ? NB : 1); ++b) ay[b] = f32x16{};
    bf16x8 pf[2] = {}, df[2] = {};
    // the two products of block j
    auto products = [&](int j) {
        const bf16_t* x = slot(j);
        const bf16_t* y = x + W::HALF;
        sc = KV ? f32x16{} : lane_values(stats(j), h);
        dp = f32x16{};
        bf16x8 fx[NS], fy[NS];
        fx[0] = by_row(x, 0);
        fy[0] = by_row(y, 0);
#pragma unroll
        for (int q = 0; q < NS; ++q) {
            if (q + 1 < NS) {
                fx[q + 1] = by_row(x, q + 1);
                fy[q + 1] = by_row(y, q + 1);
            }
            E::mma(sc, fx[q], xf[q]);
            E::mma(dp, fy[q], yf[q]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // product i of the sums over block j: X^T ds and, for dk and dv, Y^T p in turn
    constexpr int MS = KV ? 4 * NB : 2 * NB, EL = 16 / MS;
    auto operand = [&](int j, int i) {
        const bf16_t* x = slot(j);
        return KV ? across(i & 1 ? x + W::HALF : x, i >> 2, (i >> 1) & 1) : across(x, i >> 1, i & 1);
    };
    auto add = [&](int i, bf16x8 f) {
        if (!KV) E::mma(ax[i >> 1], f, df[i & 1]);
        else if (i & 1) E::mma(ay[KV ? i >> 2 : 0], f, pf[(i >> 1) & 1]);
        else E::mma(ax[i >> 2], f, df[(i >> 1) & 1]);
    };
    // (order: some of the block's scores are hidden by the causal order.  Steps of their own: the branch inside a step cost registers, and spilled ones are waited for
    // with the blocks on their way; 64 ragged histories of up to 1,024, a mask, heads of 64: 220 -> 214 us; equal ones, heads of 128 974 -> 818.)
    auto step = [&](auto first, auto order, int j, auto d) {
        lds_barrier();
        const int hidden = order.value ? in_block(above - j * 32, h) : 0;
        if (j + 2 < steps) {
            put(j + 2, d);
            if (j + 4 < steps) request(j + 4, d);
        }
        const float* sj = stats(j);
        float p[16], ds[16];
        bf16x8 f[MS];
        float4 L[4], D[4];
        if constexpr (!first.value) {
            f[0] = operand(j - 1, 0);
            f[1] = operand(j - 1, 1);
        }
        if constexpr (KV) {
            L[0] = *reinterpret_cast<const float4*>(sj + 4 * h);
            D[0] = *reinterpret_cast<const float4*>(sj + 32 + 4 * h);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < MS; ++i) {
            if constexpr (!first.value) {
                if (i + 2 < MS) f[i + 2] = operand(j - 1, i + 2);
                add(i, f[i]);
            }
#pragma unroll
            for (int e = i * EL; e < (i + 1) * EL; ++e) {
                float lv = col_base, dv = col_delta;
                if constexpr (KV) {
                    if (e % 4 == 0 && e + 4 < 16) {
                        L[e / 4 + 1] = *reinterpret_cast<const float4*>(sj + 2 * e + 8 + 4 * h);
                        D[e / 4 + 1] = *reinterpret_cast<const float4*>(sj + 32 + 2 * e + 8 + 4 * h);
                    }
                    const float4 l4 = L[e / 4], d4 = D[e / 4];
                    lv = e % 4 == 0 ? l4.x : e % 4 == 1 ? l4.y : e % 4 == 2 ? l4.z : l4.w;
                    dv = e % 4 == 0 ? d4.x : e % 4 == 1 ? d4.y : e % 4 == 2 ? d4.z : d4.w;
                }
                float x = sc[e];
                if constexpr (order.value) x = among(hidden, e) != KV ? x : -INFINITY;
                p[e] = __builtin_amdgcn_exp2f(fmaf(x, c2, -lv));
                ds[e] = p[e] * (dp[e] - dv);
                asm volatile("" : "+v"(ds[e]));   // (here: element by element, not all sixteen behind the products)
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (KV) pack_block(p, pf);
        pack_block(ds, df);
        products(j + 1);      // (behind the last block: of what lies there, never used)
    };
    if (steps) {
        const std::integral_constant<int, 0> even_step{};
        const std::integral_constant<int, 1> odd_step{};
        request(0, even_step);
        if (steps > 1) request(1, odd_step);
        put(0, even_step);
        if (steps > 2) request(2, even_step);
        if (steps > 1) put(1, odd_step);
        if (steps > 3) request(3, odd_step);
        lds_barrier();
        products(0);
        const std::integral_constant<bool, CAUSAL> ordered{};
        int j = 1;
        auto two_steps = [&](auto order) {
            step(std::false_type(), order, j, odd_step);
            if (j + 1 < steps) step(std::false_type(), order, j + 1, even_step);
            j += 2;
        };
        step(std::true_type(), ordered, 0, even_step);
        // (the waves' edges differ, the number of their steps and so of barriers does not)
        if (CAUSAL && KV)
            while (j < steps && j * 32 < edge) two_steps(ordered);
        while (j < steps && (!CAUSAL || KV || j * 32 + 64 <= edge)) two_steps(std::false_type());
        if (CAUSAL && !KV)
            while (j < steps) two_steps(ordered);
#pragma unroll
        for (int i = 0; i < MS; ++i) add(i, operand(steps - 1, i));
    }
    if (!in) return;
    if (none) {
#pragma unroll
        for (int b = 0; b < NB; ++b) ax[b] = f32x16{};
#pragma unroll
        for (int b = 0; b < (KV ? NB : 1); ++b) ay[b] = f32x16{};
    }
    if constexpr (KV) {
        store_column<bf16_t, NB>((bf16_t*)a.dk + key * a.lddk + key0, a.dim, ax, a.scale, h);
        store_column<bf16_t, NB>((bf16_t*)a.dv + key * a.lddv + key0, a.dim, ay, 1.f, h);
    } else {
        store_column<bf16_t, NB>((bf16_t*)a.dq + query * a.lddq + (int64_t)head * a.dim, a.dim, ax, a.scale, h);
    }
}
// Heads of 32: a step's products are too few to hide what a walk adds to it (64 users x 256 queries x 1,024 keys x 8 heads: 121 us, tiles 104).
template <typename T, int DP, int WAVES> constexpr bool walks() { return sizeof(T) == 2 && WAVES == 4 && DP >= 64; }
template <typename T, int DP, int WC, int RS, bool CAUSAL>
__device__ __forceinline__ void dkv_any(const SeqAttendArgs& a, char* smem, u32 id) {
    if constexpr (walks<T, DP, WC>()) walk_block<DP, true, false, CAUSAL>(a, smem, id);
    else dkv_block<T, DP, WC, RS, CAUSAL>(a, smem, id);
}
template <typename T, int DP, int WR, int KS, bool MASK, bool CAUSAL>
__device__ __forceinline__ void dq_any(const SeqAttendArgs& a, char* smem, u32 id) {
    if constexpr (walks<T, DP, WR>()) walk_block<DP, false, MASK, CAUSAL>(a, smem, id);
    else dq_block<T, DP, WR, KS, MASK, CAUSAL>(a, smem, id);
}
// All of the gradient in one launch: n_dkv workgroups make dk and dv, n_dq dq.  Neither needs anything of the other, and the
// rest of the one fills what the other leaves idle; those with the longer way to walk come first.
// (causal, fp32, four waves along the keys: 256 registers, two workgroups on a compute unit, for 8 of them spilled: 64 users of 512, 8 heads over 4 of 64: 549 -> 448 us; with fewer
// waves along the keys 70 and more are.)
template <typename T, int DP, int WR, int WC, int KS, int RS, bool MASK, bool CAUSAL>
__global__ __launch_bounds__(256, sizeof(T) == 2 || (CAUSAL && WC == 4) ? 2 : 1) void seq_attend_grad_kernel(SeqAttendArgs a, u32 n_dkv, u32 n_dq, int dq_first) {
    extern __shared__ __align__(16) char smem[];
    const u32 id = workgroup(), before = dq_first ? n_dq : n_dkv;
    if ((id < before) == (dq_first != 0)) dq_any<T, DP, WR, KS, MASK, CAUSAL>(a, smem, dq_first ? id : id - before);
    else dkv_any<T, DP, WC, RS, CAUSAL>(a, smem, dq_first ? id - before : id);
}
// Heads of more than 64: dk and dv take all of a lane's registers, dq half of them; they run one after the other.
template <typename T, int DP, int WC, int RS, bool CAUSAL>
__global__ __launch_bounds__(256, 1) void seq_attend_dkv_kernel(SeqAttendArgs a) {
    extern __shared__ __align__(16) char smem[];
    dkv_any<T, DP, WC, RS, CAUSAL>(a, smem, workgroup());
}
template <typename T, int DP, int WR, int KS, bool MASK, bool CAUSAL>
__global__ __launch_bounds__(256, sizeof(T) == 4 || WR < 4 ? 1 : 2) void seq_attend_dq_kernel(SeqAttendArgs a) {
    extern __shared__ __align__(16) char smem[];
    dq_any<T, DP, WR, KS, MASK, CAUSAL>(a, smem, workgroup());
}

// ------------------------------------------------------------------------------------------------ launches
static size_t lds_bytes(size_t tiles, int dp, int parts, int slots) {   // the tiles, or what joining the waves takes
    return std::max(tiles, parts > 1 ? 1024 + (size_t)slots * (dp / 32) * 16 * 64 * 4 : 0);
}
template <typename F>
static void launch_lds(hipStream_t st, F f, int64_t grid, size_t lds, const SeqAttendArgs& a) {
    if (lds > 64 * 1024) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    hipLaunchKernelGGL(f, workgroups(grid), dim3(256), lds, st, a);
}
// A workgroup's four waves: as many along its rows as still leave the device enough workgroups, the others along the keys of the same rows.
static int64_t pairs_of(const SeqAttendArgs& a) { return a.n_seqs * a.kv_heads; }
static int64_t blocks_of(int64_t rows, int waves) { return (rows + 32 * waves - 1) / (32 * waves); }
// four, two: workgroups from which on four or two waves lie along the rows
static int waves_along(int64_t pairs, int64_t rows, int64_t four, int64_t two) {
    if (rows > 64 && pairs * blocks_of(rows, 4) >= four) return 4;
    return rows > 32 && pairs * blocks_of(rows, 2) >= two ? 2 : 1;
}
// us with 1 / 2 / 4 waves along the rows (pairs of a user and a key head; rows; keys), forward:
//   bf16, heads of 64     32; 512; 1,024    16 /  26 /  29      128; 256; 1,024   28 /  21 /  36     256; 256; 256    22 /  17 /  15
//   bf16, heads of 128    64; 256; 512      18 /  31 /  27       16; 2,048; 2,048 83 /  80 /  65     256; 256; 256    43 /  38 /  23
//   fp32, heads of 64     16; 512; 512      20 /  25 /  34      128; 256; 1,024   92 /  81 /  86     256; 256; 256    63 /  51 /  46
//   fp32, heads of 128   148; 61; 243       38 /  30 /   -       64; 256; 512     62 /  51 /  68     256; 512; 128   196 / 133 / 130
// (bf16 with heads of 128: two along the rows leave room for one workgroup on a compute unit, four for two.)  Gradient, waves along the rows for dq:
//   bf16, heads of 64      2; 256; 4,096    37 /  50 /  78       32; 512; 1,024   39 /  32 /  34      64; 512; 1,024  64 /  55 /  58
//   fp32, heads of 128    16; 512; 512     138 / 160 / 201       32; 512; 1,024  304 / 284 / 374      64; 512; 1,024 594 / 553 / 534
// and two or four along the keys for dk and dv: bf16, heads of 64, 16; 512; 512 19 / 24, 128; 256; 1,024 66 / 58; fp32, heads of 128, 201 / 270, 594 / 565.
// Few rows and many keys: the keys are split over so many workgroups that the device holds them at a time (two of bf16 on a compute unit, one of fp32's larger
// tiles), 256 keys each at least.  us, one / two workgroups a compute unit: 64 users' ragged slots of 4,096 keys, one query of 8 heads: bf16 24.5 / 22.1; 64 of 1,000 keys,
// heads of 128: fp32 47 / 63; pieces of 512 keys: one user of 4,096 keys, fp32, 31 / 47.
// Causal, dk and dv: the first keys of a sequence are seen by all of its rows and the last ones by few, so the workgroup with the longest way decides where workgroups are
// few.  us of the gradient with 1 / 2 / 4 waves along the keys (users; longest; heads over key heads of a width):
//   bf16   1; 4,096; 8 over 2 of 64       215 / 302 / 450     4; 2,048; 8 over 2 of 64   115 / 158 / 233     16; 512; 8 over 4 of 64   36 / 31 / 41
//          16; 1,024; 8 over 4 of 64       77 /  65 /  76     64; 512; 8 over 2 of 64     90 /  82 /  87     64; 1,024; 8 over 4 of 64  - / 217 / 217
//          8; 4,096; 8 over 4 of 64       726 / 628 / 582     32; 1,024; 8 over 4 of 128   - / 250 / 216    256; 256; 8 over 2 of 64    - / 142 / 124
//   fp32   2; 1,024; 8 over 4 of 128      292 / 382 / 658     16; 512; 8 over 4 of 64    138 / 128 / 197     64; 300; 4 over 2 of 32   69 / 50 / 64
//          37; 243; 4 over 4 of 40         71 /  64 /  54     64; 512; 8 over 4 of 64    474 / 456 / 448    256; 200; 4 over 2 of 64  282 / 343 / 238
// The border of 256 rows for fp32 with few workgroups, 2 / 4 waves: below it 64; 200; 4 over 4 of 64 107 / 80, 64; 256; 4 over 4 of 64 125 / 97, of 250 and 32 wide 65 / 56, 128 wide 224 / 198,
// 64; 128; 8 over 4 of 64 74 / 65; above it 64; 150; 8 over 4 of 64 75 / 89, 64; 160; 8 over 4 of 40 67 / 78, 32; 300; 4 over 4 of 64 65 / 71, of 350 and 128 wide 169 / 197; from 400 on either may be: 32; 400;
// 4 over 4 of 64 102 / 98, 64; 200; 8 over 4 of 64 175 / 121, 16; 512 above 128 / 197.
static int causal_key_waves(const SeqAttendArgs& a, int n_cus, int bf16) {
    const int64_t pairs = pairs_of(a);
    if (pairs * blocks_of(a.longest_k, 2) <= n_cus) return 1;
    return pairs * blocks_of(a.longest_k, 4) >= 3 * n_cus || (!bf16 && a.longest_q * a.group <= 256) ? 4 : 2;
}
void seq_attend_shape(SeqAttendArgs& a, int n_cus, int bf16, int grad) {
    const int64_t pairs = pairs_of(a), rows = a.longest_q * a.group;
    a.splits = a.key_waves = 1;
    if (grad) {
        a.row_waves = waves_along(pairs, rows, bf16 ? n_cus / 2 : n_cus, n_cus / 4);
        a.key_waves = waves_along(pairs, a.longest_k, n_cus / 2 + 1, 0) == 4 ? 4 : 2;
        if (a.causal) a.key_waves = causal_key_waves(a, n_cus, bf16);
        return;
    }
    if (bf16 && a.dim > 64) a.row_waves = rows > 32 && pairs * blocks_of(rows, 4) >= n_cus ? 4 : 1;
    else a.row_waves = waves_along(pairs, rows, 2 * n_cus, bf16 ? 2 * n_cus : n_cus / 2 + 1);
    // (causal, a handful of new rows over long slots: two waves along 33 to 64 rows, so that keys and values are read once: 64 users' 16 rows of 8 heads over 2 of 64 and
    // slots of 4,096 31.4 -> 27.4 us, fp32 109 -> 104; up to 32 rows 23.0 / 24.8, more than 64 37.0 / 38.6)
    if (a.causal && rows > 32 && rows <= 64 && !(bf16 && a.dim > 64)) a.row_waves = 2;
    const int64_t groups = pairs * blocks_of(rows, a.row_waves);
    if (groups > 0) a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(bf16 ? 2 : 1) * n_cus / groups, a.longest_k / 256, SPLITS}));
}

// The most (piece, query, head) that a call of no more sequences, rows and keys has.  Only few workgroups are cut into pieces, so many that n_cus (bf16: twice as many) hold all
// of them, and then a workgroup has one wave's rows, or two in causal order, of 33 rows and more; but for bf16 with wide heads, where n_cus workgroups of four are cut in two.
int64_t seq_attend_pieces(const SeqAttendArgs& a, int n_cus, int bf16) {
    const int64_t slots = (bf16 ? 2 : 1) * n_cus, most = std::min<int64_t>({slots, a.longest_k / 256, SPLITS}), rows = std::min<int64_t>(a.longest_q * a.group, bf16 && a.dim > 64 ? 128 : 64);
    return most > 1 ? std::min(most * a.n_queries * a.kv_heads * a.group, slots * rows) : 0;
}

template <bool CAUSAL, typename T, int DP, int WR>
static void attend_rows(hipStream_t st, const SeqAttendArgs& a) {
    constexpr int KS = WR == 1 ? 1 : 2;
    const int64_t grid = work_grid(a, (a.longest_q * a.group + 32 * WR - 1) / (32 * WR) * a.splits);
    const size_t lds = lds_bytes(AttendTile<T, DP, WR, KS>::BYTES, DP, 4 / WR, WR);
    if (a.key_mask) launch_lds(st, seq_attend_kernel<T, DP, WR, KS, true, CAUSAL>, grid, lds, a);
    else launch_lds(st, seq_attend_kernel<T, DP, WR, KS, false, CAUSAL>, grid, lds, a);
}
template <bool CAUSAL, int DP>
static void attend_wide(hipStream_t st, SeqAttendArgs a) {
    const int64_t grid = work_grid(a, (a.longest_q * a.group + 127) / 128 * a.splits);
    // (a launch of its own, 4 us, where the call is large: 64 ragged users of 512 queries and 2,048 keys 143 -> 128 us, equal ones 188 -> 192; 256 and 1,024 keys each
    // 57 -> 60: not there)
    if (a.n_seqs > RANKED || a.n_seqs < 2 || grid * (a.longest_k / 64) < 32768) a.order = nullptr;
    if (a.order) hipLaunchKernelGGL(seq_attend_order_kernel, dim3(1), dim3(256), 0, st, a);
    if (a.key_mask) launch_lds(st, seq_attend_wide_kernel<DP, true, CAUSAL>, grid, WideTile<DP>::BYTES, a);
    else launch_lds(st, seq_attend_wide_kernel<DP, false, CAUSAL>, grid, WideTile<DP>::BYTES, a);
}
template <bool CAUSAL, typename T, int DP, int WR, int WC>
static void grad_tiles(hipStream_t st, const SeqAttendArgs& a) {
    constexpr int KS = WR == 1 ? 1 : 2, RS = WC == 4 && !(DP == 128 && sizeof(T) == 4) ? 2 : 1;
    const int64_t n_dq = a.n_queries > 0 ? work_grid(a, (a.longest_q * a.group + 32 * WR - 1) / (32 * WR)) : 0;
    const int64_t n_dkv = a.n_keys > 0 ? work_grid(a, (a.longest_k + 32 * WC - 1) / (32 * WC)) : 0;
    const size_t lds_q = walks<T, DP, WR>() ? (size_t)Walk<DP>::BYTES : lds_bytes(AttendTile<T, DP, WR, KS>::BYTES, DP, 4 / WR, WR);
    const size_t lds_k = walks<T, DP, WC>() ? (size_t)Walk<DP>::BYTES : lds_bytes(DkvTile<T, DP, WC, RS>::BYTES, DP, 4 / WC, WC);
    if constexpr (DP <= 64) {
        auto both = [&](auto f) {
            const size_t lds = std::max(lds_q, lds_k);
            if (lds > 64 * 1024) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            hipLaunchKernelGGL(f, workgroups(n_dq + n_dkv), dim3(256), lds, st, a, (u32)n_dkv, (u32)n_dq, a.longest_k > a.longest_q * a.group ? 1 : 0);
        };
        if (a.key_mask) both(seq_attend_grad_kernel<T, DP, WR, WC, KS, RS, true, CAUSAL>);
        else both(seq_attend_grad_kernel<T, DP, WR, WC, KS, RS, false, CAUSAL>);
    } else {
        if (n_dkv) launch_lds(st, seq_attend_dkv_kernel<T, DP, WC, RS, CAUSAL>, n_dkv, lds_k, a);
        if (n_dq && a.key_mask) launch_lds(st, seq_attend_dq_kernel<T, DP, WR, KS, true, CAUSAL>, n_dq, lds_q, a);
        else if (n_dq) launch_lds(st, seq_attend_dq_kernel<T, DP, WR, KS, false, CAUSAL>, n_dq, lds_q, a);
    }
}
template <bool CAUSAL, typename T, int DP, int WR>
static void grad_rows(hipStream_t st, const SeqAttendArgs& a) {
    if constexpr (CAUSAL) {
        if (a.key_waves == 1) return grad_tiles<CAUSAL, T, DP, WR, 1>(st, a);
    }
    if (a.key_waves == 4) grad_tiles<CAUSAL, T, DP, WR, 4>(st, a);
    else grad_tiles<CAUSAL, T, DP, WR, 2>(st, a);
}
template <bool CAUSAL, typename T, int DP>
static void attend_dim(hipStream_t st, const SeqAttendArgs& a) {
    if (a.row_waves == 1) attend_rows<CAUSAL, T, DP, 1>(st, a);
    else if constexpr (sizeof(T) == 2) {
        if constexpr (DP == 128) attend_wide<CAUSAL, DP>(st, a);
        else if (a.row_waves == 2) attend_rows<CAUSAL, T, DP, 2>(st, a);
        else attend_wide<CAUSAL, DP>(st, a);
    } else if (a.row_waves == 2) attend_rows<CAUSAL, T, DP, 2>(st, a);
    else attend_rows<CAUSAL, T, DP, 4>(st, a);
}
template <bool CAUSAL, typename T, int DP>
static void grad_dim(hipStream_t st, const SeqAttendArgs& a) {
    if (a.row_waves == 1) grad_rows<CAUSAL, T, DP, 1>(st, a);
    else if (a.row_waves == 2) grad_rows<CAUSAL, T, DP, 2>(st, a);
    else grad_rows<CAUSAL, T, DP, 4>(st, a);
}
template <bool CAUSAL, typename T>
static void attend_type(hipStream_t st, const SeqAttendArgs& a) {
    if (a.dim <= 32) attend_dim<CAUSAL, T, 32>(st, a);
    else if (a.dim <= 64) attend_dim<CAUSAL, T, 64>(st, a);
    else attend_dim<CAUSAL, T, 128>(st, a);
    if (a.splits > 1) hipLaunchKernelGGL((seq_attend_join_kernel<T>), workgroups((a.n_queries * a.kv_heads * a.group + 3) / 4), dim3(256), 0, st, a);
}
template <bool CAUSAL, typename T>
static void grad_type(hipStream_t st, SeqAttendArgs a) {
    if (a.n_seqs > RANKED || a.n_seqs < 2) a.order = nullptr;
    const u32 ranks = a.order ? 2 : 0;
    const int64_t stat = (a.n_queries * a.kv_heads * a.group + 15) / 16 + ranks;
    if (stat > 0) hipLaunchKernelGGL((seq_attend_stat_kernel<T>), workgroups(stat), dim3(256), 0, st, a, ranks);
    if (a.dim <= 32) grad_dim<CAUSAL, T, 32>(st, a);
    else if (a.dim <= 64) grad_dim<CAUSAL, T, 64>(st, a);
    else grad_dim<CAUSAL, T, 128>(st, a);
}
void launch_seq_attend(hipStream_t st, const SeqAttendArgs& a, int bf16) {
    if (a.n_queries <= 0 || a.n_seqs <= 0) return;
    if (a.causal) bf16 ? attend_type<true, bf16_t>(st, a) : attend_type<true, float>(st, a);
    else bf16 ? attend_type<false, bf16_t>(st, a) : attend_type<false, float>(st, a);
}
void launch_seq_attend_grad(hipStream_t st, const SeqAttendArgs& a, int bf16) {
    if (a.n_seqs <= 0 || (a.n_queries <= 0 && a.n_keys <= 0)) return;
    if (a.causal) bf16 ? grad_type<true, bf16_t>(st, a) : grad_type<true, float>(st, a);
    else bf16 ? grad_type<false, bf16_t>(st, a) : grad_type<false, float>(st, a);
}
