// Layer norm of rows, with the residual sum in front of it, and its gradients:
//   s = x + r,  mean = sum_c s_c / C,  rstd = 1 / sqrt(sum_c (s_c - mean)^2 / C + eps),  h = (s - mean) rstd,  y = w h + b
//   ds = rstd (g - sum_c g_c / C - h sum_c g_c h_c / C) + e,   g = w dy, e the gradient that reaches s by another way,
//   dw = sum_rows dy h,  db = sum_rows dy.
// All of it in fp32: the sum s is not rounded before the norm is taken of it (only where it is written), and the sum of squares is taken of the differences
// from the mean, of a row that stays in registers, not of the squares of the row (which loses the digits that mean and row share).
// Bound: memory, every array once.
#include <algorithm>

#include "gm_internal.h"

// 16 bytes of a row.  WHOLE: rows are 16-byte aligned and of a width that 16 bytes divide; else they begin at any element, which the memory pipeline takes in one access all the
// same, and the last piece may end with the row (100,000 rows of 845: bf16 174 us, 3.9 TB/s; fp32 360 and 3.7; rows of 1,024 5.5).
template <typename T, bool WHOLE> struct Piece {
    enum { V = 16 / sizeof(T) };
    typedef Pack<T, V> P;
    P k;
    __device__ __forceinline__ void load(const T* p, int left) {   // left: elements of the row from p on, one at least
        if (WHOLE) k = *reinterpret_cast<const P*>(p);
        else if (left >= V) __builtin_memcpy(&k, p, 16);
        else {
            T x[V];
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = e < left ? p[e] : T(0);
            __builtin_memcpy(&k, x, 16);
        }
    }
    __device__ __forceinline__ float get(int e) const { return k.get(e); }
    __device__ __forceinline__ void store(T* p, int left, const float (&v)[V]) {
        k.put(v);
        if (WHOLE) *reinterpret_cast<P*>(p) = k;
        else if (left >= V) __builtin_memcpy(p, &k, 16);
        else {
            T x[V];
            __builtin_memcpy(x, &k, 16);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < left) p[e] = x[e];
        }
    }
};
// V of the weights (or biases) from p on, of which `left` are there, one at least; zeros behind them.
template <int V, bool WHOLE> __device__ __forceinline__ void load_weights(float (&w)[V], const float* p, int left) {
    if (WHOLE || left >= V) __builtin_memcpy(w, p, 4 * V);
    else
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = e < left ? p[e] : 0.f;
}
template <typename T> __device__ __forceinline__ float one(const T* p) { return Pack<T, 1>{*p}.get(0); }
template <typename T> __device__ __forceinline__ void put_one(T* p, float x) {
    Pack<T, 1> k;
    const float v[1] = {x};
    k.put(v);
    *p = k.x;
}
__host__ __device__ __forceinline__ int norm_pad(int channels) { return (channels + 3) / 4 * 4; }   // of a row of partial sums
template <int L> __device__ __forceinline__ float sum_lanes(float x) {   // of L neighbouring lanes
#pragma unroll
    for (int d = 1; d < L; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float sum_workgroup(float x, float* area) {   // of 256 threads; area: four floats, free again behind the call's second barrier
    x = sum_lanes<64>(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) area[threadIdx.x >> 6] = x;
    __syncthreads();
    return (area[0] + area[1]) + (area[2] + area[3]);
}

template <int L> __device__ __forceinline__ float sum_row(float x, float* area) {
    if constexpr (L == 256) return sum_workgroup(x, area);
    else return sum_lanes<L>(x);
}

// ------------------------------------------------------------------------------------------------ forward
// A row is L lanes' (8 to 64, or a workgroup's), N pieces each.
template <typename T, bool WHOLE, int L, int N>
__global__ __launch_bounds__(256) void seq_norm_kernel(SeqNormArgs a) {
    typedef Piece<T, WHOLE> P;
    constexpr int V = P::V;
    __shared__ float sums[4];
    const int l = threadIdx.x % L;
    const int64_t row = (int64_t)workgroup() * (256 / L) + threadIdx.x / L;
    if (row >= a.n) return;
    auto at = [&](int i) { return (i * L + l) * V; };
    auto inside = [&](int i, int e) { return WHOLE || at(i) + e < a.channels; };   // of a piece that begins inside
    P x[N], r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (at(i) >= a.channels) continue;
        x[i].load((const T*)a.x + row * a.ldx + at(i), a.channels - at(i));
        if (a.res) r[i].load((const T*)a.res + row * a.ldr + at(i), a.channels - at(i));
    }
    float s[N][V], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s[i][e] = at(i) < a.channels ? a.res ? x[i].get(e) + r[i].get(e) : x[i].get(e) : 0.f;
            sum += s[i][e];
        }
    const float mean = sum_row<L>(sum, sums) / (float)a.channels;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = at(i) < a.channels && inside(i, e) ? s[i][e] - mean : 0.f;
            sq = fmaf(d, d, sq);
        }
    const float rstd = 1.f / sqrtf(sum_row<L>(sq, sums) / (float)a.channels + a.eps);
    if (a.stats && l == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = at(i), left = a.channels - c;
        if (left <= 0) continue;
        P out;
        if (a.sum) out.store((T*)a.sum + row * a.lds + c, left, s[i]);
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = (s[i][e] - mean) * rstd;
        float w[V];
        if (a.weight) {
            load_weights<V, WHOLE>(w, a.weight + c, left);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] *= w[e];
        }
        if (a.bias) {
            load_weights<V, WHOLE>(w, a.bias + c, left);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] += w[e];
        }
        out.store((T*)a.y + row * a.ldy + c, left, y);
    }
}
// Rows that no registers hold: a workgroup a row, which it reads three times (from its L2 after the first).
template <typename T>
__global__ __launch_bounds__(256) void seq_norm_wide_kernel(SeqNormArgs a) {
    __shared__ float area[4];
    const int64_t row = workgroup();
    if (row >= a.n) return;
    const T* x = (const T*)a.x + row * a.ldx;
    const T* r = a.res ? (const T*)a.res + row * a.ldr : nullptr;
    auto at = [&](int c) { return one(x + c) + (r ? one(r + c) : 0.f); };
    float sum = 0.f, sq = 0.f;
    for (int c = threadIdx.x; c < a.channels; c += 256) sum += at(c);
    const float mean = sum_workgroup(sum, area) / (float)a.channels;
    for (int c = threadIdx.x; c < a.channels; c += 256) sq = fmaf(at(c) - mean, at(c) - mean, sq);
    const float rstd = 1.f / sqrtf(sum_workgroup(sq, area) / (float)a.channels + a.eps);
    if (a.stats && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
    for (int c = threadIdx.x; c < a.channels; c += 256) {
        const float s = at(c), h = (s - mean) * rstd;
        if (a.sum) put_one((T*)a.sum + row * a.lds + c, s);
        put_one((T*)a.y + row * a.ldy + c, (a.weight ? h * a.weight[c] : h) + (a.bias ? a.bias[c] : 0.f));
    }
}

// ------------------------------------------------------------------------------------------------ gradient
// A workgroup takes every blocks-th group of 256 / L rows; a lane's columns are the same in all of them, so dw and db stay in its registers, are added over
// the workgroup's rows at the end, and over the workgroups by a second launch, both in a fixed order.  The next group's row is on its way while one is summed.
// (131,072 rows of 512, bf16, with e: 107 us, 5.0 TB/s; forward with a residual, 262,144 rows: 179 to 196 us, 5.5 to 6 TB/s.)
template <typename T, bool WHOLE, int L, int N>
__global__ __launch_bounds__(256) void seq_norm_grad_kernel(SeqNormArgs a) {
    typedef Piece<T, WHOLE> P;
    constexpr int V = P::V, RW = 256 / L;
    __shared__ float sums[4];
    const int l = threadIdx.x % L;
    const u32 block = workgroup();
    if (block >= (u32)a.blocks) return;
    auto at = [&](int i) { return (i * L + l) * V; };
    float w[N][V], dw[N][V], db[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = at(i) + e;
            w[i][e] = c >= a.channels ? 0.f : a.weight ? a.weight[c] : 1.f;
            dw[i][e] = db[i][e] = 0.f;
        }
    P nx[N], ny[N], ne[N];
    float2 nst = make_float2(0.f, 0.f);
    auto request = [&](int64_t row) {
        if (row >= a.n) return;
        nst = *reinterpret_cast<const float2*>(a.stats + 2 * row);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = at(i), left = a.channels - c;
            if (left <= 0) continue;
            nx[i].load((const T*)a.x + row * a.ldx + c, left);
            ny[i].load((const T*)a.dy + row * a.lddy + c, left);
            if (a.res) ne[i].load((const T*)a.res + row * a.ldr + c, left);
        }
    };
    const int64_t step = (int64_t)a.blocks * RW;
    int64_t row = (int64_t)block * RW + threadIdx.x / L;
    request(row);
    const float inv = 1.f / (float)a.channels;
    for (; row < a.n; row += step) {
        P px[N], py[N], pe[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { px[i] = nx[i]; py[i] = ny[i]; pe[i] = ne[i]; }
        const float2 st = nst;
        request(row + step);
        float h[N][V], g[N][V], s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool in = WHOLE ? at(i) < a.channels : at(i) + e < a.channels;
                h[i][e] = in ? (px[i].get(e) - st.x) * st.y : 0.f;
                const float y = in ? py[i].get(e) : 0.f;
                dw[i][e] = fmaf(y, h[i][e], dw[i][e]);
                db[i][e] += y;
                g[i][e] = y * w[i][e];
                s0 += g[i][e];
                s1 = fmaf(g[i][e], h[i][e], s1);
            }
        s0 = sum_row<L>(s0, sums) * inv;
        s1 = sum_row<L>(s1, sums) * inv;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = at(i), left = a.channels - c;
            if (left <= 0) continue;
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = st.y * (g[i][e] - s0 - h[i][e] * s1) + (a.res ? pe[i].get(e) : 0.f);
            P out;
            out.store((T*)a.dx + row * a.lddx + c, left, y);
        }
    }
    if (!a.dweight) return;
    // the workgroup's rows: lanes of a wave that hold the same columns, then the waves through LDS (5,003 rows of 845, fp32, the whole gradient 26 us; the waves one after the other
    // in one row of it 37)
    extern __shared__ __align__(16) float area[];   // [4][stride]
    const int stride = (a.channels + V - 1) / V * V, wave = threadIdx.x >> 6;
    float* out = a.blocks > 1 ? a.partial + (int64_t)block * 2 * norm_pad(a.channels) : nullptr;
    auto sum_rows = [&](float (&x)[N][V], float* to) {
        if constexpr (L == 256) {   // (every column is one thread's)
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (at(i) + e < a.channels) to[at(i) + e] = x[i][e];
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e)
#pragma unroll
                for (int d = L; d < 64; d <<= 1) x[i][e] += __shfl_xor(x[i][e], d);
            if ((threadIdx.x & 63) < L && at(i) < a.channels)
#pragma unroll
                for (int e = 0; e < V; e += 4)
                    *reinterpret_cast<float4*>(area + wave * stride + at(i) + e) = make_float4(x[i][e], x[i][e + 1], x[i][e + 2], x[i][e + 3]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.channels; c += 256) to[c] = (area[c] + area[stride + c]) + (area[2 * stride + c] + area[3 * stride + c]);
    };
    sum_rows(dw, out ? out : a.dweight);
    __syncthreads();
    sum_rows(db, out ? out + norm_pad(a.channels) : a.dbias);
}
// Wide rows: dx a workgroup a row; dw and db 256 columns and a range of rows a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void seq_norm_grad_wide_kernel(SeqNormArgs a) {
    __shared__ float area[4];
    const int64_t row = workgroup();
    if (row >= a.n) return;
    const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    auto h = [&](int c) { return (one((const T*)a.x + row * a.ldx + c) - st.x) * st.y; };
    auto g = [&](int c) { return one((const T*)a.dy + row * a.lddy + c) * (a.weight ? a.weight[c] : 1.f); };
    float s0 = 0.f, s1 = 0.f;
    for (int c = threadIdx.x; c < a.channels; c += 256) {
        s0 += g(c);
        s1 = fmaf(g(c), h(c), s1);
    }
    s0 = sum_workgroup(s0, area) / (float)a.channels;
    s1 = sum_workgroup(s1, area) / (float)a.channels;
    for (int c = threadIdx.x; c < a.channels; c += 256) {
        put_one((T*)a.dx + row * a.lddx + c, st.y * (g(c) - s0 - h(c) * s1) + (a.res ? one((const T*)a.res + row * a.ldr + c) : 0.f));
    }
}
template <typename T>
__global__ __launch_bounds__(256) void seq_norm_columns_kernel(SeqNormArgs a, u32 column_blocks) {
    const u32 id = workgroup(), block = id / column_blocks;
    const int c = (int)(id % column_blocks) * 256 + (int)threadIdx.x;
    if (block >= (u32)a.blocks || c >= a.channels) return;
    const int64_t per = (a.n + a.blocks - 1) / a.blocks, r0 = block * per, r1 = min(r0 + per, a.n);
    float dw = 0.f, db = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * r);
        const float y = one((const T*)a.dy + r * a.lddy + c);
        dw = fmaf(y, (one((const T*)a.x + r * a.ldx + c) - st.x) * st.y, dw);
        db += y;
    }
    float* out = a.blocks > 1 ? a.partial + (int64_t)block * 2 * norm_pad(a.channels) : nullptr;
    (out ? out : a.dweight)[c] = dw;
    (out ? out + norm_pad(a.channels) : a.dbias)[c] = db;
}
__global__ __launch_bounds__(256) void sum_blocks_kernel(SumBlocks a) { sum_blocks(a, workgroup()); }

// ------------------------------------------------------------------------------------------------ launches
enum { NORM_BLOCKS = 1024 };   // most workgroups of the gradient
static int norm_pieces(int channels, int bf16) { return (channels + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4); }
// Lanes of a row; 0: no registers hold one.  (bf16, 32,768 rows of 2,048, gradient: a wave a row 125 us, a workgroup a row 119; 8,192 rows of 4,096: forward 43 us, gradient 79, in
// three passes over the rows 126 and 122.)
static int norm_lanes(int channels, int bf16) {
    const int pieces = norm_pieces(channels, bf16);
    return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : pieces <= (bf16 ? 128 : 512) ? 64 : pieces <= 1024 ? 256 : 0;
}
// Workgroups of the gradient that sum the weights' over rows, as the launches have them and as many sums as are reserved: every one as many groups of rows, or a range of rows that
// no registers hold.
int seq_norm_blocks(int64_t n, int channels, int bf16) {
    const int lanes = norm_lanes(channels, bf16);
    if (!lanes) return (int)std::min<int64_t>((n + 15) / 16, std::max<int64_t>(1, NORM_BLOCKS / ((channels + 255) / 256)));
    const int64_t groups = (n + 256 / lanes - 1) / (256 / lanes), turns = std::max<int64_t>(1, (groups + NORM_BLOCKS - 1) / NORM_BLOCKS);
    return (int)((groups + turns - 1) / turns);
}
int64_t seq_norm_partials(const SeqNormArgs& a) { return a.blocks > 1 ? (int64_t)a.blocks * 2 * norm_pad(a.channels) : 0; }
// The most of any call of no more rows and channels, of either type: four rows a workgroup at least up to the 1,024 channels that a wave holds of both, then one.
int64_t seq_norm_most_partials(int64_t n, int channels) { return std::min<int64_t>(channels > 1024 ? n : (n + 3) / 4, NORM_BLOCKS) * 2 * norm_pad(channels); }

static bool whole_rows(const SeqNormArgs& a, int elem) {
    const int v = 16 / elem;
    bool ok = a.channels % v == 0;
    auto rows = [&](const void* p, int64_t ld) { ok = ok && (!p || ((uintptr_t)p % 16 == 0 && ld % v == 0)); };
    rows(a.x, a.ldx); rows(a.res, a.ldr); rows(a.y, a.ldy); rows(a.sum, a.lds); rows(a.dy, a.lddy); rows(a.dx, a.lddx);
    return ok;
}
template <typename T, bool WHOLE, int L, int N>
static void norm_rows(hipStream_t st, const SeqNormArgs& a, bool grad) {
    constexpr int V = 16 / sizeof(T);
    if (!grad) hipLaunchKernelGGL((seq_norm_kernel<T, WHOLE, L, N>), workgroups((a.n + 256 / L - 1) / (256 / L)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((seq_norm_grad_kernel<T, WHOLE, L, N>), dim3(a.blocks), dim3(256), L == 256 ? 0 : 4 * sizeof(float) * ((a.channels + V - 1) / V * V), st, a);
}
template <typename T, bool WHOLE>
static bool norm_width(hipStream_t st, const SeqNormArgs& a, bool grad) {   // false: too wide
    constexpr bool BF16 = sizeof(T) == 2;
    const int pieces = norm_pieces(a.channels, BF16);
    switch (norm_lanes(a.channels, BF16)) {
        case 8: norm_rows<T, WHOLE, 8, 1>(st, a, grad); break;
        case 16: norm_rows<T, WHOLE, 16, 1>(st, a, grad); break;
        case 32: norm_rows<T, WHOLE, 32, 1>(st, a, grad); break;
        case 64:
            if (pieces <= 64) norm_rows<T, WHOLE, 64, 1>(st, a, grad);
            else if (pieces <= 128) norm_rows<T, WHOLE, 64, 2>(st, a, grad);
            else if constexpr (!BF16) {
                if (pieces <= 256) norm_rows<T, WHOLE, 64, 4>(st, a, grad);
                else norm_rows<T, WHOLE, 64, 8>(st, a, grad);
            }
            break;
        case 256:
            if constexpr (BF16) {
                if (pieces <= 256) norm_rows<T, WHOLE, 256, 1>(st, a, grad);
                else if (pieces <= 512) norm_rows<T, WHOLE, 256, 2>(st, a, grad);
                else norm_rows<T, WHOLE, 256, 4>(st, a, grad);
            } else norm_rows<T, WHOLE, 256, 4>(st, a, grad);
            break;
        default: return false;
    }
    return true;
}
template <typename T>
static void norm_type(hipStream_t st, const SeqNormArgs& a, bool grad) {
    const bool fits = whole_rows(a, sizeof(T)) ? norm_width<T, true>(st, a, grad) : norm_width<T, false>(st, a, grad);
    if (!fits && !grad) hipLaunchKernelGGL((seq_norm_wide_kernel<T>), workgroups(a.n), dim3(256), 0, st, a);
    if (!fits && grad) {
        hipLaunchKernelGGL((seq_norm_grad_wide_kernel<T>), workgroups(a.n), dim3(256), 0, st, a);
        const int64_t columns = (a.channels + 255) / 256;
        if (a.dweight) hipLaunchKernelGGL((seq_norm_columns_kernel<T>), workgroups(a.blocks * columns), dim3(256), 0, st, a, (u32)columns);
    }
    if (grad && a.dweight && a.blocks > 1) {
        const SumBlocks sum{a.partial, a.blocks, a.channels, norm_pad(a.channels), a.dweight, a.dbias};
        hipLaunchKernelGGL(sum_blocks_kernel, workgroups(sum.workgroups()), dim3(256), 0, st, sum);
    }
}
void launch_seq_norm(hipStream_t st, const SeqNormArgs& a, int bf16) {
    if (a.n <= 0) return;
    if (bf16) norm_type<bf16_t>(st, a, false);
    else norm_type<float>(st, a, false);
}
void launch_seq_norm_grad(hipStream_t st, const SeqNormArgs& a, int bf16) {
    if (a.n <= 0) {   // no rows: sums of nothing
        if (a.dweight) launch_fill_f32(st, a.dweight, a.channels, 0.f);
        if (a.dweight) launch_fill_f32(st, a.dbias, a.channels, 0.f);
        return;
    }
    if (bf16) norm_type<bf16_t>(st, a, true);
    else norm_type<float>(st, a, true);
}
