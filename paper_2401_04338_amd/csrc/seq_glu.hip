// A gated feed-forward block: both projections of the rows, the activation and the product in one kernel,
//   g = x Wg + bg,  u = x Wu + bu,  y = act(g) u,
// and its gradients, from g and u as they were kept:
//   dg = dy u act'(g),  du = dy act(g),  dx = dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du,  dbg, dbu = sums of dg, du over the rows.
// One matrix product serves the three forms.  A workgroup owns a tile of the result; its operands pass through LDS 128 bytes of contraction at a time, in two
// stages: a step's fragments are read while the one before is multiplied, the next tile is put into the other stage and the one after it asked for in the middle,
// so there is one barrier a tile.  An operand whose contraction index is its slowest (weights going forward; rows, for the weights' gradients) lies in LDS as in
// memory and is read across: transposing LDS reads for bf16, an element a lane for fp32.
// The second operand goes into the matrix instruction first, so that a lane holds one row of the result and four consecutive columns at a time.
//   forward: half of the tile's columns are of Wg, half the same columns of Wu, dealt so that a wave has both of a column and the product needs no exchange;
//   dx:      one contraction over [dg | du] and then Wg, Wu;
//   dW:      a contraction over the rows, cut into pieces where the weights have few tiles; the pieces are added in their order by a launch of their own.
// Tiles are 256 x 256 for eight waves, one workgroup on a compute unit, where they give every unit one: a step's fragments take as long out of LDS as its products take.  (65,536 rows,
// 512 to 2 x 1,024, bf16, us forward / dx / dW: 164 / 144 to 160 / 139 to 157; four waves and half as large a tile twice on a unit, 32 values of contraction at a time: 187 to 191 / 190 to
// 202 / 177 to 183; 128 x 128 tiles: 205 / - / -.)  Smaller tiles where those would leave units idle.
// dg and du are written once in between, rounded to the tensors' type: they are operands of two products (formed while an operand is staged they would be made
// once a column of tiles, and a tile's exponentials take longer than its products).  All sums are fp32.
#include <algorithm>
#include <type_traits>

#include "gm_internal.h"

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

#define LOG2E 1.44269504088896340736f

// ------------------------------------------------------------------------------------------------ activations
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * LOG2E)); }
// The normal distribution's function and its density.  exp(z^2) erfc(z) = t (c0 + c1 t + .. + c8 t^8) with t = 1 / (1 + 0.375 z) for z >= 0; the coefficients have the least largest
// relative error over z <= 9.6, where the tail ends below 2^-126 (least squares whose weights grow with the error): 1.5e-8 of the value.  With the roundings, x^2 times for the
// exponent's, the tail is off by (1.5 x^2 + 36) 2^-24 of itself; a formula that is off by 0.75e-7 of 1, three products shorter, by 1e-3 of itself at -5.  (65,536 rows, bf16: 64 to
// 2 x 1,024, where the exponentials bound, 60 -> 65 us; 512 to 2 x 1,024 199 either way.)
__device__ __forceinline__ void normal(float x, float& phi, float& density) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.375f * 0.70710678118654752440f, fabsf(x), 1.f)), e = __builtin_amdgcn_exp2f(x * x * (-0.5f * LOG2E));
    float p = 0.0308483057f;   // (half of the coefficients)
    p = fmaf(p, t, -0.144037679f);
    p = fmaf(p, t, 0.21694687f);
    p = fmaf(p, t, -0.115538195f);
    p = fmaf(p, t, 0.137422055f);
    p = fmaf(p, t, 0.0605194829f);
    p = fmaf(p, t, 0.102715209f);
    p = fmaf(p, t, 0.105316751f);
    p = fmaf(p, t, 0.105807208f);
    const float tail = e * (t * p);
    phi = x < 0.f ? tail : 1.f - tail;
    density = 0.39894228040143267794f * e;
}
// act(g), and with it act'(g)
template <int ACT> __device__ __forceinline__ float activation(float g) {
    if constexpr (ACT == GLU_SILU) return g * sigmoid(g);
    else if constexpr (ACT == GLU_GELU) {
        float phi, density;
        normal(g, phi, density);
        return g * phi;
    } else if constexpr (ACT == GLU_SIGMOID) return sigmoid(g);
    else return g > 0.f ? g : g != g ? g : 0.f;
}
template <int ACT> __device__ __forceinline__ float activation(float g, float& slope) {
    if constexpr (ACT == GLU_SILU) {
        const float s = sigmoid(g);
        slope = fmaf(g * s, sigmoid(-g), s);
        return g * s;
    } else if constexpr (ACT == GLU_GELU) {
        float phi, density;
        normal(g, phi, density);
        slope = fmaf(g, density, phi);
        return g * phi;
    } else if constexpr (ACT == GLU_SIGMOID) {
        const float s = sigmoid(g);
        slope = s * sigmoid(-g);
        return s;
    } else {
        slope = g > 0.f ? 1.f : 0.f;
        return g > 0.f ? g : g != g ? g : 0.f;
    }
}

// ------------------------------------------------------------------------------------------------ the product
template <typename T> struct Mat;
template <> struct Mat<bf16_t> {
    enum { E = 8, GK = 64, KC = 16, PADK = 32 };   // elements of 16 bytes; contraction of a tile, of a fragment; pad of the LDS rows that are read across (banks apart)
    typedef bf16x8 frag;
    enum { PARTS = 1 };   // instructions of a fragment
    static __device__ __forceinline__ void mma(f32x16& c, frag a, frag b, int) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    // contraction step kk of column c0 + lane % 32 of a tile whose rows are contraction values: 16 lanes at a time, lane i points at four consecutive columns
    // of row i / 4 and receives column i of the four rows
    static __device__ __forceinline__ frag across(const bf16_t* tile, int ld, int c0, int kk, int lane) {
        typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
        const bf16_t* p = tile + (kk * KC + (lane >> 5) * 8 + ((lane & 15) >> 2)) * ld + c0 + (lane & 16) + (lane & 3) * 4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * ld));
        return __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
template <> struct Mat<float> {
    enum { E = 4, GK = 32, KC = 8, PADK = 24 };
    typedef float4 frag;
    enum { PARTS = 4 };
    static __device__ __forceinline__ void mma(f32x16& c, frag a, frag b, int e) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(e == 0 ? a.x : e == 1 ? a.y : e == 2 ? a.z : a.w, e == 0 ? b.x : e == 1 ? b.y : e == 2 ? b.z : b.w, c, 0, 0, 0);
    }
    static __device__ __forceinline__ frag across(const float* tile, int ld, int c0, int kk, int lane) {
        const float* p = tile + (kk * KC + (lane >> 5) * 4) * ld + c0 + (lane & 31);
        return make_float4(p[0], p[ld], p[2 * ld], p[3 * ld]);
    }
};

// Rows x columns of a matrix in memory, on their way to LDS in 16-byte pieces through a buffer that ends with the last row: what lies outside reads as zeros.
#define NOWHERE (1u << 31)   // an offset behind every tile
// Rows of a tile along the contraction are 128 bytes; their 16-byte pieces lie at piece ^ turn(row), so that the two rows that 16 lanes write and the 16 rows that 16 lanes
// read lie in all banks (dx of 65,536 rows, 2,048 to 512: 144 to 150 us; rows padded by 16 bytes instead 155 to 160).
__device__ __forceinline__ int turn(int row) { return (row >> 1) & 7; }
template <typename T, int ROWS, int COLS, int NT> struct Tile {
    enum { E = Mat<T>::E, PR = COLS / E, N = ROWS * PR / NT };
    static_assert(ROWS * PR % NT == 0 && NT % PR == 0, "whole rounds of pieces");
    u32x4 x[N];
    static __device__ __forceinline__ int tid() { return (int)threadIdx.x % NT; }   // in the waves that share the tile
    static __device__ __forceinline__ int col() { return tid() % PR * E; }
    static __device__ __forceinline__ int row(int i) { return tid() / PR + NT / PR * i; }
    // p: the first row; rows: how many there are; left: how many columns lie at and behind `at`, where the tile begins
    __device__ __forceinline__ void request(const T* p, int rows, u32 ld, u32 at, int left) {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)((u32)max(rows, 0) * ld * (u32)sizeof(T)), 0x00020000);
        const u32 o = col() < left ? ((u32)row(0) * ld + at + (u32)col()) * (u32)sizeof(T) : NOWHERE;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(o + (u32)(NT / PR * i) * ld * (u32)sizeof(T)), 0, 0);
    }
    template <int LD> __device__ __forceinline__ void put(T* lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + row(i) * LD + col()) = x[i];
    }
    __device__ __forceinline__ void put_turned(T* lds) const {   // rows of eight pieces
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + row(i) * COLS + (col() / E ^ turn(row(i))) * E) = x[i];
    }
};
enum { FORM_GLU, FORM_DX, FORM_DW };
// WM x WN waves share a tile of BM rows and BN columns; WK such groups take turns at its operand tiles, and their sums are added in the groups' order.
template <typename T, int BM, int BN, int WM, int WN, int WK_, int FORM> struct Product {
    typedef Mat<T> M;
    static constexpr bool KA = FORM == FORM_DW, KB = FORM != FORM_DX;      // the contraction index is the slowest
    static constexpr int GK = M::GK, WK = WK_, NT = 64 * WM * WN, MI = BM / (32 * WM), NI = BN / (32 * WN), HALVES = FORM == FORM_GLU ? 2 : 1, NP = NI / HALVES;
    static constexpr int LDA = KA ? BM + (int)M::PADK : GK, LDB = KB ? BN + (int)M::PADK : GK;
    static constexpr int A_ELEMS = (KA ? GK : BM) * LDA, ELEMS = A_ELEMS + (KB ? GK : BN) * LDB;
    // a wave's strip of results in LDS, of SB blocks side by side, in a stage that nobody reads
    static constexpr int strip(int blocks) { return FORM == FORM_DW || (FORM == FORM_DX && BM == 64) || sizeof(T) == 4 ? 32 * (blocks * 32 + 4) * 4 : 32 * (blocks * 32 + 8) * 2; }
    static constexpr int SB = WM * WN * strip(NP) <= ELEMS * (int)sizeof(T) ? NP : 1, STRIP = strip(SB);
    static constexpr int STAGE = WM * WN * STRIP <= ELEMS * (int)sizeof(T) ? ELEMS : WM * WN * STRIP / (int)sizeof(T), BYTES = WK * 2 * STAGE * (int)sizeof(T);
    static_assert(STAGE * (int)sizeof(T) % 16 == 0 && STRIP % 16 == 0, "stages and strips are 16-byte aligned");
    static_assert(WK == 1 || WM * WN * MI * NI * 4096 <= STAGE * (int)sizeof(T), "a group's sums fit a stage");
    // where in the tile a wave's blocks lie: forward both halves' blocks of the same columns
    static __device__ __forceinline__ int column(int wn, int j) { return j / NP * (BN / HALVES) + wn * (NP * 32) + j % NP * 32; }
};

__device__ __forceinline__ void lds_barrier() {   // (tiles on their way in registers need not be waited for, as __syncthreads would)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// A workgroup's results, `count` of them one after the other: the operand tiles of all of them are one stream, so that a result's first tiles are on their way, and in LDS, when
// the one before is finished, and what finish() stores is on its way while the next is made.
//   open(t): the t-th result's operands are asked for next; tiles(t): how many tiles of contraction it has (one at least); request(kt): asks for the opened one's
//   kt-th; put(stage): what was asked for, to LDS; finish(t, area): the sums are complete, area is LDS that nobody reads.
template <typename P, typename T, typename Open, typename Tiles, typename Request, typename Put, typename Finish>
__device__ __forceinline__ void multiply(f32x16 (&acc)[P::MI][P::NI], T* lds, int count, int wm, int wn, int lane, Open&& open, Tiles&& tiles, Request&& request, Put&& put,
                                         Finish&& finish) {
    typedef typename P::M M;
    typedef typename M::frag frag;
    const int l32 = lane & 31, h = lane >> 5;
    int along[4];   // where a lane's piece of step kk lies in a block of 32 rows along the contraction
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) along[kk] = l32 * P::GK + ((2 * kk + h) ^ turn(l32)) * M::E;
    auto read = [&](const T* stage, int kk, frag (&a)[P::MI], frag (&b)[P::NI]) {
        const T* B = stage + P::A_ELEMS;
#pragma unroll
        for (int i = 0; i < P::MI; ++i) {
            const int m = wm * (P::MI * 32) + i * 32;
            if constexpr (P::KA) a[i] = M::across(stage, P::LDA, m, kk, lane);
            else a[i] = *reinterpret_cast<const frag*>(stage + m * P::GK + along[kk]);
        }
#pragma unroll
        for (int j = 0; j < P::NI; ++j) {
            const int c = P::column(wn, j);
            if constexpr (P::KB) b[j] = M::across(B, P::LDB, c, kk, lane);
            else b[j] = *reinterpret_cast<const frag*>(B + c * P::GK + along[kk]);
        }
    };
    auto mmas = [&](const frag (&a)[P::MI], const frag (&b)[P::NI]) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int e = 0; e < M::PARTS; ++e)
#pragma unroll
            for (int i = 0; i < P::MI; ++i)
#pragma unroll
                for (int j = 0; j < P::NI; ++j) M::mma(acc[i][j], b[j], a[i], e);
        __builtin_amdgcn_s_setprio(0);
    };
    const int group = P::WK > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / P::NT) : 0;
    T* const smem = lds + group * 2 * P::STAGE;
    auto turns = [&](int t) { return (tiles(t) + P::WK - 1) / P::WK; };
    int rt = 0, rk = 0, rn = turns(0);   // what is asked for next
    auto next = [&]() {
        if (rt >= count) return;
        request(rk * P::WK + group);     // (behind the last tile: zeros)
        if (++rk < rn) return;
        rk = 0;
        if (++rt >= count) return;
        rn = turns(rt);
        open(rt);
    };
    u32 step = 0;
    auto tile = [&]() {
        const T* cur = smem + (step & 1) * P::STAGE;
        T* nxt = smem + (~step & 1) * P::STAGE;
        frag a0[P::MI], b0[P::NI], a1[P::MI], b1[P::NI];
        read(cur, 0, a0, b0);
        read(cur, 1, a1, b1);
        mmas(a0, b0);
        read(cur, 2, a0, b0);
        mmas(a1, b1);
        put(nxt);
        read(cur, 3, a1, b1);
        next();
        mmas(a0, b0);
        mmas(a1, b1);
        lds_barrier();
        ++step;
    };
    open(0);
    next();
    put(smem);
    next();
    lds_barrier();
    for (int t = 0; t < count; ++t) {
#pragma unroll
        for (int i = 0; i < P::MI; ++i)
#pragma unroll
            for (int j = 0; j < P::NI; ++j) acc[i][j] = f32x16{};
        // (the first tile apart: what it waits for was asked for in front of the stores of finish(), which need not have landed)
        const int n = turns(t);
        tile();
        for (int kt = 1; kt < n; ++kt) tile();
        T* const area = lds + (~step & 1) * P::STAGE;
        if constexpr (P::WK > 1) {
            constexpr int BLOCKS = P::MI * P::NI;
            auto place = [&](int g, int b) { return reinterpret_cast<f32x4*>(area + g * 2 * P::STAGE) + ((threadIdx.x % P::NT / 64 * BLOCKS + b) * 4) * 64 + lane; };
            if (group) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16& x = acc[b / P::NI][b % P::NI];
                        place(group, b)[q * 64] = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                    }
            }
            lds_barrier();
            if (!group) {
#pragma unroll
                for (int g = 1; g < P::WK; ++g)
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x4 y = place(g, b)[q * 64];
                            f32x16& x = acc[b / P::NI][b % P::NI];
                            x[4 * q] += y[0]; x[4 * q + 1] += y[1]; x[4 * q + 2] += y[2]; x[4 * q + 3] += y[3];
                        }
            }
        }
        if (!group) finish(t, reinterpret_cast<char*>(area));
        lds_barrier();
    }
}

// A strip of 32 rows by NB * 32 columns of results, as a wave's matrix instructions leave them (value(j, i): the i-th of block j), through the wave's own LDS
// to rows [0, rows) and columns [0, cols) at out, as whole row segments.
template <typename O, int NB, typename Value>
__device__ __forceinline__ void store_blocks(char* area, O* out, int64_t ld, int rows, int cols, int lane, Value&& value) {
    constexpr int E = 16 / sizeof(O), LDE = NB * 32 + E, CH = NB * 32 / E, RP = 64 / CH;   // pieces of a row, rows a pass
    O* strip = reinterpret_cast<O*>(area);
    const int h = lane >> 5, l32 = lane & 31;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {value(j, 4 * q), value(j, 4 * q + 1), value(j, 4 * q + 2), value(j, 4 * q + 3)};
            Pack<O, 4> k;
            k.put(v);
            *reinterpret_cast<Pack<O, 4>*>(strip + l32 * LDE + j * 32 + 8 * q + 4 * h) = k;
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the strip is the wave's own)
    const int r0 = lane / CH, c = lane % CH * E;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)out, 0, (int)((u32)min(max(rows, 0), 32) * (u32)ld * (u32)sizeof(O)), 0x00020000);
    const u32 at = c < cols ? ((u32)r0 * (u32)ld + (u32)c) * (u32)sizeof(O) : NOWHERE;
#pragma unroll
    for (int r = 0; r < 32; r += RP)
        __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4*>(strip + (r + r0) * LDE + c), rs, (int)(at + (u32)r * (u32)ld * (u32)sizeof(O)), 0, 0);
    asm volatile("" ::: "memory");
}
// A strip of NP blocks, SB at a time.
template <typename O, typename P, typename Value>
__device__ __forceinline__ void store_strip(char* area, O* out, int64_t ld, int rows, int cols, int lane, Value&& value) {
#pragma unroll
    for (int b = 0; b < P::NP; b += P::SB)
        store_blocks<O, P::SB>(area, out + b * 32, ld, rows, cols - b * 32, lane, [&](int j, int e) { return value(b + j, e); });
}
// The results of a workgroup.  Workgroups are dealt to the eight XCDs in turn; each XCD has a run of neighbouring tiles, which share rows, and its workgroups take
// turns at them.
struct Share {
    u32 first, stride;
    int count;
    __device__ __forceinline__ u32 tile(int t) const { return first + (u32)t * stride; }
};
__device__ __forceinline__ Share share_of(u32 n_tiles) {
    const u32 per = (n_tiles + 7) / 8, from = blockIdx.x % 8 * per, to = min(from + per, n_tiles), each = gridDim.x / 8;
    Share s{from + blockIdx.x / 8, each, 0};
    s.count = s.first < to ? (int)((to - s.first + each - 1) / each) : 0;
    return s;
}

// Bound: the matrix cores and LDS (each further 512 of contraction takes 116 us of 65,536 rows by 2 x 1,024, bf16: 1,180 TFLOP/s; fp32 135 of 157), then what a result's end takes:
// its exponentials, and its stores where the pre-activations are kept.  65,536 rows, 512 to 2 x 1,024, bf16: 164 us (840 TFLOP/s), kept 186 to 191; 64 rows 7 (latency).
template <typename T, int BM, int BN, int WM, int WN, int WK, bool KEEP>
__global__ __launch_bounds__(64 * WM * WN * WK) void seq_glu_kernel(SeqGluArgs a, u32 n_ntiles, u32 n_tiles) {
    typedef Product<T, BM, BN, WM, WN, WK, FORM_GLU> P;
    constexpr int NP = P::NP;
    extern __shared__ __align__(16) char smem[];
    const Share share = share_of(n_tiles);
    if (!share.count) return;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % (WM * WN), wm = wave / WN, wn = wave % WN;
    Tile<T, BM, P::GK, P::NT> xt;
    Tile<T, P::GK, BN / 2, P::NT> gt, ut;
    const T* x = nullptr;
    int n0 = 0, rows = 0;
    f32x16 acc[P::MI][P::NI];
    multiply<P>(acc, reinterpret_cast<T*>(smem), share.count, wm, wn, lane,
        [&](int t) {
            const u32 tile = share.tile(t);
            const int64_t m0 = (int64_t)(tile / n_ntiles) * BM;
            n0 = (int)(tile % n_ntiles) * (BN / 2);
            rows = (int)min(a.n - m0, (int64_t)BM);
            x = (const T*)a.x + m0 * a.ldx;
        },
        [&](int) { return (a.d_in + P::GK - 1) / P::GK; },
        [&](int kt) {
            const int k0 = kt * P::GK, left = a.d_in - k0;
            xt.request(x, rows, (u32)a.ldx, (u32)k0, left);
            gt.request((const T*)a.wg + k0 * a.ldwg, min(left, P::GK), (u32)a.ldwg, (u32)n0, a.d_out - n0);
            ut.request((const T*)a.wu + k0 * a.ldwu, min(left, P::GK), (u32)a.ldwu, (u32)n0, a.d_out - n0);
        },
        [&](T* to) {
            xt.put_turned(to);
            gt.template put<P::LDB>(to + P::A_ELEMS);
            ut.template put<P::LDB>(to + P::A_ELEMS + BN / 2);
        },
        [&](int t, char* area) {
            area += wave * P::STRIP;
            const u32 tile = share.tile(t);
            const int64_t m0 = (int64_t)(tile / n_ntiles) * BM;
            const int tile_rows = (int)min(a.n - m0, (int64_t)BM), c0 = (int)(tile % n_ntiles) * (BN / 2) + wn * (NP * 32), cols = a.d_out - c0;
            if (a.bg) {
#pragma unroll
                for (int j = 0; j < NP; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = j * 32 + 8 * q + 4 * h;
                        if (c >= cols) continue;
                        const float4 g = *reinterpret_cast<const float4*>(a.bg + c0 + c), u = *reinterpret_cast<const float4*>(a.bu + c0 + c);
#pragma unroll
                        for (int i = 0; i < P::MI; ++i) {
                            f32x16 &x0 = acc[i][j], &x1 = acc[i][NP + j];
                            x0[4 * q] += g.x; x0[4 * q + 1] += g.y; x0[4 * q + 2] += g.z; x0[4 * q + 3] += g.w;
                            x1[4 * q] += u.x; x1[4 * q + 1] += u.y; x1[4 * q + 2] += u.z; x1[4 * q + 3] += u.w;
                        }
                    }
            }
            auto strips = [&](auto act) {
#pragma unroll
                for (int i = 0; i < P::MI; ++i) {
                    const int r0 = wm * (P::MI * 32) + i * 32;
                    const int64_t m = m0 + r0;
                    if constexpr (KEEP) {
                        store_strip<T, P>(area, (T*)a.gate + m * a.ldgate + c0, a.ldgate, tile_rows - r0, cols, lane, [&](int j, int e) { return acc[i][j][e]; });
                        store_strip<T, P>(area, (T*)a.up + m * a.ldup + c0, a.ldup, tile_rows - r0, cols, lane, [&](int j, int e) { return acc[i][NP + j][e]; });
                    }
                    store_strip<T, P>(area, (T*)a.y + m * a.ldy + c0, a.ldy, tile_rows - r0, cols, lane,
                                       [&](int j, int e) { return activation<act.value>(acc[i][j][e]) * acc[i][NP + j][e]; });
                }
            };
            switch (a.act) {
                case GLU_SILU: strips(std::integral_constant<int, GLU_SILU>()); break;
                case GLU_GELU: strips(std::integral_constant<int, GLU_GELU>()); break;
                case GLU_SIGMOID: strips(std::integral_constant<int, GLU_SIGMOID>()); break;
                default: strips(std::integral_constant<int, GLU_RELU>()); break;
            }
        });
}

// ------------------------------------------------------------------------------------------------ gradient
// dg and du side by side, [n][2 d_out], and their column sums.  Bound: memory, three arrays read, two written (65,536 rows of 1,024, bf16: 115 us, 5.8 TB/s).  `lanes` neighbours share as many pieces
// of a row; a workgroup takes every blocks-th group of 256 / lanes rows.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void seq_glu_slope_kernel(SeqGluArgs a, int lanes, u32 column_blocks) {
    constexpr int V = Mat<T>::E;
    typedef Pack<T, V> P;
    __shared__ float area[2][64 * V];
    const u32 id = blockIdx.y * gridDim.x + blockIdx.x, block = id / column_blocks;
    if (block >= (u32)a.blocks) return;
    const int l = threadIdx.x % lanes, c = (int)(id % column_blocks * lanes + l) * V;
    const bool in = c < a.d_out;
    const int64_t rw = 256 / lanes;
    float sg[V] = {}, su[V] = {};
    if (in)
        for (int64_t r = block * rw + threadIdx.x / lanes; r < a.n; r += a.blocks * rw) {
            const P pd = *reinterpret_cast<const P*>((const T*)a.dy + r * a.lddy + c), pg = *reinterpret_cast<const P*>((const T*)a.gate + r * a.ldgate + c),
                    pu = *reinterpret_cast<const P*>((const T*)a.up + r * a.ldup + c);
            float dg[V], du[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float slope;
                const float d = pd.get(e), v = activation<ACT>(pg.get(e), slope);
                dg[e] = d * pu.get(e) * slope;
                du[e] = d * v;
                sg[e] += dg[e];
                su[e] += du[e];
            }
            P og, ou;
            og.put(dg);
            ou.put(du);
            T* out = (T*)a.d + r * (2 * (int64_t)a.d_out) + c;
            *reinterpret_cast<P*>(out) = og;
            *reinterpret_cast<P*>(out + a.d_out) = ou;
        }
    if (!a.dbg) return;
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int e = 0; e < V; ++e)
        for (int s = lanes; s < 64; s <<= 1) {
            sg[e] += __shfl_xor(sg[e], s);
            su[e] += __shfl_xor(su[e], s);
        }
    float* og = a.blocks > 1 ? a.colpart + (int64_t)block * 2 * a.d_out : a.dbg;
    float* ou = a.blocks > 1 ? og + a.d_out : a.dbu;
    for (int k = 0; k < 4; ++k) {
        if (wave == k && (threadIdx.x & 63) < (u32)lanes) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float g = k ? area[0][l * V + e] + sg[e] : sg[e], u = k ? area[1][l * V + e] + su[e] : su[e];
                if (k < 3) {
                    area[0][l * V + e] = g;
                    area[1][l * V + e] = u;
                } else if (in) {
                    og[c + e] = g;
                    ou[c + e] = u;
                }
            }
        }
        __syncthreads();
    }
}

// Bound: as forward (65,536 rows, 2 x 1,024 to 512, bf16: 144 to 150 us, 920 to 950 TFLOP/s; few rows: the latency of the contraction's turns).
template <typename T, int BM, int BN, int WM, int WN, int WK>
__global__ __launch_bounds__(64 * WM * WN * WK) void seq_glu_dx_kernel(SeqGluArgs a, u32 n_ntiles, u32 n_tiles) {
    typedef Product<T, BM, BN, WM, WN, WK, FORM_DX> P;
    extern __shared__ __align__(16) char smem[];
    const Share share = share_of(n_tiles);
    if (!share.count) return;
    constexpr bool SPLITS = BM == 64;   // (others are not cut into pieces)
    const int half = (a.d_out + P::GK - 1) / P::GK, per = SPLITS ? (2 * half + a.dx_splits - 1) / a.dx_splits : 2 * half;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % (WM * WN), wm = wave / WN, wn = wave % WN;
    const u32 per_split = SPLITS ? n_tiles / (u32)a.dx_splits : n_tiles;
    Tile<T, BM, P::GK, P::NT> dt;
    Tile<T, BN, P::GK, P::NT> wt;
    const T* d = nullptr;
    int n0 = 0, rows = 0, first = 0;
    f32x16 acc[P::MI][P::NI];
    multiply<P>(acc, reinterpret_cast<T*>(smem), share.count, wm, wn, lane,
        [&](int t) {
            const u32 id = share.tile(t), tile = id % per_split;
            const int64_t m0 = (int64_t)(tile / n_ntiles) * BM;
            n0 = (int)(tile % n_ntiles) * BN;
            rows = (int)min(a.n - m0, (int64_t)BM);
            first = (int)(id / per_split) * per;
            d = (const T*)a.d + m0 * 2 * a.d_out;
        },
        [&](int t) { return SPLITS ? max(min(2 * half - (int)(share.tile(t) / per_split) * per, per), 1) : 2 * half; },
        [&](int turn) {
            const int kt = SPLITS ? turn < per ? first + turn : 2 * half : turn;   // (behind the piece: nothing)
            const bool up = kt >= half;
            const int k0 = (up ? kt - half : kt) * P::GK, left = a.d_out - k0;
            const int64_t ld = up ? a.ldwu : a.ldwg;
            dt.request(d, rows, 2u * (u32)a.d_out, (u32)(k0 + (up ? a.d_out : 0)), left);
            wt.request((const T*)(up ? a.wu : a.wg) + n0 * ld, min(a.d_in - n0, BN), (u32)ld, (u32)k0, left);
        },
        [&](T* to) {
            dt.put_turned(to);
            wt.put_turned(to + P::A_ELEMS);
        },
        [&](int t, char* area) {
            area += wave * P::STRIP;
            const u32 id = share.tile(t), tile = id % per_split;
            const int64_t m0 = (int64_t)(tile / n_ntiles) * BM;
            const int tile_rows = (int)min(a.n - m0, (int64_t)BM), c0 = (int)(tile % n_ntiles) * BN + wn * (P::NP * 32);
#pragma unroll
            for (int i = 0; i < P::MI; ++i) {
                const int r0 = wm * (P::MI * 32) + i * 32;
                auto value = [&](int j, int e) { return acc[i][j][e]; };
                if (SPLITS && a.dx_splits > 1)
                    store_strip<float, P>(area, a.dx_partial + ((int64_t)(id / per_split) * a.n + m0 + r0) * a.d_in + c0, a.d_in, tile_rows - r0, a.d_in - c0, lane, value);
                else store_strip<T, P>(area, (T*)a.dx + (m0 + r0) * a.lddx + c0, a.lddx, tile_rows - r0, a.d_in - c0, lane, value);
            }
        });
}

// n_ntiles: of both weights.  Bound: as forward (65,536 rows, 512 by 2 x 1,024, bf16, 16 pieces: 137 to 144 us, 950 to 1,000 TFLOP/s, and 12 for the pieces' sums).
template <typename T, int BM, int BN, int WM, int WN, int WK>
__global__ __launch_bounds__(64 * WM * WN * WK) void seq_glu_dw_kernel(SeqGluArgs a, u32 n_ntiles, u32 n_tiles) {
    typedef Product<T, BM, BN, WM, WN, WK, FORM_DW> P;
    extern __shared__ __align__(16) char smem[];
    const Share share = share_of(n_tiles);
    if (!share.count) return;
    struct Place { u32 split; bool up; int m0, n0; int64_t r0, r1; };
    auto place = [&](int t) {
        const u32 id = share.tile(t), per_split = n_tiles / (u32)a.splits, tile = id % per_split, nt = tile % n_ntiles;
        Place p{id / per_split, nt >= n_ntiles / 2, (int)(tile / n_ntiles) * BM, (int)(nt % (n_ntiles / 2)) * BN, 0, 0};
        p.r0 = (int64_t)p.split * a.piece;
        p.r1 = min(p.r0 + a.piece, a.n);
        return p;
    };
    const int64_t ldd = 2 * (int64_t)a.d_out;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % (WM * WN), wm = wave / WN, wn = wave % WN;
    Tile<T, P::GK, BM, P::NT> xt;
    Tile<T, P::GK, BN, P::NT> dt;
    Place from{};
    f32x16 acc[P::MI][P::NI];
    multiply<P>(acc, reinterpret_cast<T*>(smem), share.count, wm, wn, lane,
        [&](int t) { from = place(t); },
        [&](int t) {
            const Place p = place(t);
            return max((int)((p.r1 - p.r0 + P::GK - 1) / P::GK), 1);   // (no rows: a tile of zeros)
        },
        [&](int kt) {
            const int64_t r = from.r0 + (int64_t)kt * P::GK;
            const int left = (int)min(from.r1 - r, (int64_t)P::GK);
            xt.request((const T*)a.x + r * a.ldx, left, (u32)a.ldx, (u32)from.m0, a.d_in - from.m0);
            dt.request((const T*)a.d + r * ldd, left, (u32)ldd, (u32)(from.n0 + (from.up ? a.d_out : 0)), a.d_out - from.n0);
        },
        [&](T* to) {
            xt.template put<P::LDA>(to);
            dt.template put<P::LDB>(to + P::A_ELEMS);
        },
        [&](int t, char* area) {
            area += wave * P::STRIP;
            const Place p = place(t);
            const int c0 = p.n0 + wn * (P::NP * 32);
#pragma unroll
            for (int i = 0; i < P::MI; ++i) {
                const int m = p.m0 + wm * (P::MI * 32) + i * 32;
                auto value = [&](int j, int e) { return acc[i][j][e]; };
                if (a.splits > 1)
                    store_strip<float, P>(area, a.partial + ((int64_t)p.split * a.d_in + m) * ldd + (p.up ? a.d_out : 0) + c0, ldd, a.d_in - m, a.d_out - c0, lane, value);
                else
                    store_strip<T, P>(area, (T*)(p.up ? a.dwu : a.dwg) + m * (p.up ? a.lddwu : a.lddwg) + c0, p.up ? a.lddwu : a.lddwg, a.d_in - m, a.d_out - c0, lane, value);
            }
        });
}
// The pieces' sums, in their order, four elements a thread: dW's, then dx's; the last workgroups add up the biases'.
__device__ __forceinline__ void add_pieces(float (&s)[4], const float* partial, int64_t n, int pieces) {
    float4 x = *reinterpret_cast<const float4*>(partial);
    s[0] = x.x; s[1] = x.y; s[2] = x.z; s[3] = x.w;
#pragma unroll 4
    for (int p = 1; p < pieces; ++p) {
        x = *reinterpret_cast<const float4*>(partial + p * n);
        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    }
}
template <typename T>
__global__ __launch_bounds__(256) void seq_glu_join_kernel(SeqGluArgs a, u32 n_dw, u32 n_dx, SumBlocks biases) {
    const u32 id = workgroup();
    float s[4];
    Pack<T, 4> k;
    if (id < n_dw) {
        const int64_t ld = 2 * (int64_t)a.d_out, n = a.d_in * ld, i = ((int64_t)id * 256 + threadIdx.x) * 4;
        if (i >= n) return;
        add_pieces(s, a.partial + i, n, a.splits);
        k.put(s);
        const int64_t row = i / ld;
        const int c = (int)(i % ld);
        T* out = c < a.d_out ? (T*)a.dwg + row * a.lddwg + c : (T*)a.dwu + row * a.lddwu + c - a.d_out;
        *reinterpret_cast<Pack<T, 4>*>(out) = k;
    } else if (id < n_dw + n_dx) {
        const int64_t n = a.n * a.d_in, i = ((int64_t)(id - n_dw) * 256 + threadIdx.x) * 4;
        if (i >= n) return;
        add_pieces(s, a.dx_partial + i, n, a.dx_splits);
        k.put(s);
        *reinterpret_cast<Pack<T, 4>*>((T*)a.dx + i / a.d_in * a.lddx + i % a.d_in) = k;
    } else sum_blocks(biases, id - n_dw - n_dx);
}

// ------------------------------------------------------------------------------------------------ launches
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// As many workgroups as the device holds at a time, which take turns at the tiles (a multiple of eight, for the XCDs).
template <typename F>
static void launch_tiles(hipStream_t st, F f, int64_t n_mtiles, int64_t n_ntiles, int64_t splits, int threads, int lds, const SeqGluArgs& a) {
    const int64_t n = n_mtiles * n_ntiles * splits, slots = (int64_t)a.n_cus * std::max(1, 160 * 1024 / lds);
    if (n <= 0) return;
    if (lds > 64 * 1024) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    hipLaunchKernelGGL(f, dim3((unsigned)(std::min(n + 7, std::max<int64_t>(slots, 8)) / 8 * 8)), dim3(threads), lds, st, a, (u32)n_ntiles, (u32)n);
}
template <typename T, int BM, int BN, int WM, int WN, int WK> static void glu_tiles(hipStream_t st, const SeqGluArgs& a) {
    auto go = [&](auto f) { launch_tiles(st, f, ceil_div(a.n, BM), ceil_div(a.d_out, BN / 2), 1, 64 * WM * WN * WK, Product<T, BM, BN, WM, WN, WK, FORM_GLU>::BYTES, a); };
    if (a.gate) go(seq_glu_kernel<T, BM, BN, WM, WN, WK, true>);
    else go(seq_glu_kernel<T, BM, BN, WM, WN, WK, false>);
}
template <typename T, int BM, int BN, int WM, int WN, int WK> static void dx_tiles(hipStream_t st, const SeqGluArgs& a) {
    launch_tiles(st, seq_glu_dx_kernel<T, BM, BN, WM, WN, WK>, ceil_div(a.n, BM), ceil_div(a.d_in, BN), BM == 64 ? a.dx_splits : 1, 64 * WM * WN * WK, Product<T, BM, BN, WM, WN, WK, FORM_DX>::BYTES, a);
}
template <typename T, int BM, int BN, int WM, int WN, int WK> static void dw_tiles(hipStream_t st, const SeqGluArgs& a) {
    launch_tiles(st, seq_glu_dw_kernel<T, BM, BN, WM, WN, WK>, ceil_div(a.d_in, BM), 2 * ceil_div(a.d_out, BN), a.splits, 64 * WM * WN * WK, Product<T, BM, BN, WM, WN, WK, FORM_DW>::BYTES, a);
}
// The largest tiles that still give every compute unit one.  (us forward, tiles of 256 / 128 / 64: bf16, 512 to 2 x 1,024, 8,192 rows 24 / 30 / -, 4,096 rows 21 / 16 / -, 64 rows
// 18 / 12 / 9; 20,000 rows, 256 to 2 x 1,024 45 / 52 / 70; fp32, 1,024 to 2 x 1,024, 4,096 rows 259 / 146 / 167.)
static int tile_of(int64_t rows, int64_t cols, int64_t cols_per_256, int n_cus) {
    if (ceil_div(rows, 256) * ceil_div(cols, cols_per_256) >= n_cus) return 256;
    return ceil_div(rows, 128) * ceil_div(cols, cols_per_256 / 2) >= n_cus ? 128 : 64;
}
// Pieces of the rows for the weights' gradients: so many that the tiles fill the device, of 1,024 rows at least with tiles of 256 (a piece's sums are written and read again), of
// 128 with smaller ones; the largest tiles with which they do.  (us, the whole gradient, with tiles of 256 / 128: 65,536 rows, 512 to 2 x 1,024, bf16 399 / 453; 20,000 rows, 256 to
// 2 x 1,024 118 / 111, 1,024 to 2 x 256 89 / 79; 8,192 rows, 512 to 2 x 512, fp32 237 / 178.)
void seq_glu_shape(SeqGluArgs& a, int n_cus, int bf16) {
    for (int tile : {256, 128, 64}) {
        const int64_t tiles = ceil_div(a.d_in, tile) * 2 * ceil_div(a.d_out, tile), fill = (tile == 256 ? 1 : 2) * n_cus, rows = tile == 256 ? 1024 : 128;
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>({fill / tiles, a.n / rows, 64}));
        a.dw_tile = tile;
        a.piece = std::max<int64_t>(64, ceil_div(ceil_div(a.n, want), 64) * 64);
        a.splits = (int)std::max<int64_t>(1, ceil_div(a.n, a.piece));
        const int64_t waste = tiles * tile * tile, least = 2 * (int64_t)a.d_in * a.d_out;   // (elements of the tiles, of the weights)
        if (tiles * want >= (tile == 256 ? fill * 3 / 4 : fill / 2) && waste <= least + least / 2) break;
    }
    const int v = bf16 ? 8 : 4;
    // few rows: dx's contraction in pieces of eight tiles at least, as many as give every compute unit a workgroup (1 and 64 rows, 2 x 1,024 to 512, bf16: 11.8 -> 7.0 and
    // 8.2 us; 512 rows, 2 x 256 to 128, fp32 14 -> 10; 817 rows, 2 x 1,024 to 64, fp32, the whole gradient 63 -> 31)
    a.dx_splits = 1;
    const int64_t dx_tiles = ceil_div(a.n, 64) * ceil_div(a.d_in, 64), contraction = 2 * ceil_div(a.d_out, bf16 ? 64 : 32);
    if (a.n > 0 && 2 * dx_tiles <= n_cus) a.dx_splits = (int)std::max<int64_t>(1, std::min<int64_t>({n_cus / dx_tiles, contraction / 8, 8}));
    const int64_t row = ceil_div(a.d_out, v);
    a.lanes = 64;   // (halved while a quarter of them and more would have no piece: 3,001 rows of 260, fp32 9.1 -> 7.6 us)
    while (a.lanes > 8 && ceil_div(row, a.lanes) * a.lanes * 4 >= row * 5) a.lanes /= 2;
    const int64_t column_blocks = ceil_div(row, a.lanes), groups = ceil_div(a.n, 256 / a.lanes);
    a.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(groups, std::max<int64_t>(1, 2048 / column_blocks)));
    a.n_cus = n_cus;
}
int64_t seq_glu_partials(const SeqGluArgs& a) { return a.splits > 1 ? (int64_t)a.splits * a.d_in * 2 * a.d_out : 0; }
int64_t seq_glu_dx_partials(const SeqGluArgs& a) { return a.dx_splits > 1 ? a.dx_splits * a.n * a.d_in : 0; }
int64_t seq_glu_column_partials(const SeqGluArgs& a) { return a.blocks > 1 ? (int64_t)a.blocks * 2 * a.d_out : 0; }
// The most of any call of no more rows and widths: pieces times tiles are no more than fill the device, of 256 x 256, or twice as many smaller ones, and a call of one
// piece has none; workgroups along the rows take four rows at least and each has sums of all of d_out, or they are 2,048 with those along a row, of 64 pieces of up to 8 elements.
int64_t seq_glu_most_partials(const SeqGluArgs& a, int n_cus) {
    return std::min<int64_t>(std::min<int64_t>(a.n / 128, 64) * a.d_in * 2 * a.d_out, (int64_t)n_cus * 65536);
}
int64_t seq_glu_most_dx_partials(const SeqGluArgs& a, int n_cus) { return std::min<int64_t>(8 * a.n * a.d_in, (int64_t)n_cus * 4096); }   // (pieces times tiles of 64 x 64)
int64_t seq_glu_most_column_partials(const SeqGluArgs& a) { return a.n > 4 ? std::min<int64_t>(ceil_div(a.n, 4) * 2 * a.d_out, 2048 * 2 * 512) : 0; }

template <typename T> static void glu_type(hipStream_t st, const SeqGluArgs& a) {
    switch (tile_of(a.n, a.d_out, 128, a.n_cus)) {
        case 256: glu_tiles<T, 256, 256, 2, 4, 1>(st, a); break;
        case 128: glu_tiles<T, 128, 128, 2, 2, 1>(st, a); break;
        default:
            // (fewer tiles than compute units: the contraction is dealt to two groups.  1 and 64 rows, 512 to 2 x 1,024, bf16: 8.8 -> 7.6 us, 512 rows 9.3 -> 8.6; 512 rows, 128 to
            // 2 x 256, fp32 9.7 -> 7.8)
            if (ceil_div(a.n, 64) * ceil_div(a.d_out, 32) <= a.n_cus) glu_tiles<T, 64, 64, 2, 1, 2>(st, a);
            else glu_tiles<T, 64, 64, 2, 1, 1>(st, a);
    }
}
template <typename T> static void glu_grad_type(hipStream_t st, const SeqGluArgs& a) {
    const int64_t column_blocks = ceil_div(a.d_out, a.lanes * Mat<T>::E);
    auto slopes = [&](auto f) { hipLaunchKernelGGL(f, workgroups(a.blocks * column_blocks), dim3(256), 0, st, a, a.lanes, (u32)column_blocks); };
    switch (a.act) {
        case GLU_SILU: slopes(seq_glu_slope_kernel<T, GLU_SILU>); break;
        case GLU_GELU: slopes(seq_glu_slope_kernel<T, GLU_GELU>); break;
        case GLU_SIGMOID: slopes(seq_glu_slope_kernel<T, GLU_SIGMOID>); break;
        default: slopes(seq_glu_slope_kernel<T, GLU_RELU>); break;
    }
    switch (tile_of(a.n, a.d_in, 256, a.n_cus)) {
        case 256: dx_tiles<T, 256, 256, 2, 4, 1>(st, a); break;
        case 128: dx_tiles<T, 128, 128, 2, 2, 1>(st, a); break;
        default:
            // (as above, to four: 64 rows, 2 x 1,024 to 512, bf16: 17.7 -> 11.8 us, 2,048 rows 19.4 -> 14.2; 512 rows, 2 x 256 to 128, fp32: 16.6 -> 13.9, 3,001 rows, 2 x 260 to 132:
            // 18.9 -> 17.9)
            if (ceil_div(a.n, 64) * ceil_div(a.d_in, 64) * a.dx_splits <= a.n_cus) dx_tiles<T, 64, 64, 2, 2, 4>(st, a);
            else dx_tiles<T, 64, 64, 2, 2, 1>(st, a);
    }
    if (a.dw_tile == 256) dw_tiles<T, 256, 256, 2, 4, 1>(st, a);
    else if (a.dw_tile == 128) dw_tiles<T, 128, 128, 2, 2, 1>(st, a);
    else dw_tiles<T, 64, 64, 2, 2, 1>(st, a);
    const SumBlocks biases{a.colpart, a.blocks, a.d_out, a.d_out, a.dbg, a.dbu};
    const int64_t n_dw = a.splits > 1 ? ceil_div((int64_t)a.d_in * 2 * a.d_out, 1024) : 0, n_dx = a.dx_splits > 1 ? ceil_div(a.n * a.d_in, 1024) : 0;
    const int64_t n = n_dw + n_dx + (a.dbg && a.blocks > 1 ? biases.workgroups() : 0);
    if (n > 0) hipLaunchKernelGGL((seq_glu_join_kernel<T>), workgroups(n), dim3(256), 0, st, a, (u32)n_dw, (u32)n_dx, biases);
}
void launch_seq_glu(hipStream_t st, const SeqGluArgs& a, int bf16) {
    if (a.n <= 0) return;
    if (bf16) glu_type<bf16_t>(st, a);
    else glu_type<float>(st, a);
}
// (without rows the sums are of nothing: the weights' gradients are one piece of no tiles, the biases' one block)
void launch_seq_glu_grad(hipStream_t st, const SeqGluArgs& a, int bf16) {
    if (bf16) glu_grad_type<bf16_t>(st, a);
    else glu_grad_type<float>(st, a);
}
