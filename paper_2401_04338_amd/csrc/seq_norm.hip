// Layer norm of rows, with the residual sum in front of it, and its gradients:
//   s = x + r,  mean = sum_c s_c / C,  rstd = 1 / sqrt(sum_c (s_c - mean)^2 / C + eps),  h = (s - mean) rstd,  y = w h + b
//   ds = rstd (g - sum_c g_c / C - h sum_c g_c h_c / C) + e,   g = w dy, e the gradient that reaches s by another way,
//   dw = sum_rows dy h,  db = sum_rows dy.
// All of it in fp32: the sum s is not rounded before the norm is taken of it (only where it is written), and the sum of squares is taken of the differences
// from the mean, of a row that stays in registers, not of the squares of the row (which loses the digits that mean and row share).
// Bound: memory, every array once.
#include <algorithm>

#include "gm_internal.h"

template <typename T, int V> struct Values {   // V elements, as floats
    float v[V];
    __device__ __forceinline__ void load(const T* p) {
        const Pack<T, V> k = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = k.get(e);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
    }
    __device__ __forceinline__ void store(T* p) const {
        Pack<T, V> k;
        k.put(v);
        *reinterpret_cast<Pack<T, V>*>(p) = k;
    }
};
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

// ------------------------------------------------------------------------------------------------ forward
// A row is L lanes' (8 to 64), N packs of V elements each.
template <typename T, int V, int L, int N>
__global__ __launch_bounds__(256) void seq_norm_kernel(SeqNormArgs a) {
    const int l = threadIdx.x % L;
    const int64_t row = (int64_t)workgroup() * (256 / L) + threadIdx.x / L;
    if (row >= a.n) return;
    const T* x = (const T*)a.x + row * a.ldx;
    const T* r = (const T*)a.res + row * a.ldr;
    Values<T, V> s[N];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * L + l) * V;
        if (c < a.channels) s[i].load(x + c);
        else s[i].zero();
    }
    if (a.res) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * L + l) * V;
            if (c < a.channels) {
                Values<T, V> y;
                y.load(r + c);
#pragma unroll
                for (int e = 0; e < V; ++e) s[i].v[e] += y.v[e];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += s[i].v[e];
    const float mean = sum_lanes<L>(sum) / (float)a.channels;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if ((i * L + l) * V < a.channels)
#pragma unroll
            for (int e = 0; e < V; ++e) sq = fmaf(s[i].v[e] - mean, s[i].v[e] - mean, sq);
    const float rstd = 1.f / sqrtf(sum_lanes<L>(sq) / (float)a.channels + a.eps);
    if (a.stats && l == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * L + l) * V;
        if (c >= a.channels) continue;
        if (a.sum) s[i].store((T*)a.sum + row * a.lds + c);
        Values<T, V> y;
#pragma unroll
        for (int e = 0; e < V; ++e) y.v[e] = (s[i].v[e] - mean) * rstd;
        if (a.weight)
#pragma unroll
            for (int e = 0; e < V; ++e) y.v[e] *= a.weight[c + e];
        if (a.bias)
#pragma unroll
            for (int e = 0; e < V; ++e) y.v[e] += a.bias[c + e];
        y.store((T*)a.y + row * a.ldy + c);
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
    auto at = [&](int c) { return Pack<T, 1>{x[c]}.get(0) + (r ? Pack<T, 1>{r[c]}.get(0) : 0.f); };
    float sum = 0.f, sq = 0.f;
    for (int c = threadIdx.x; c < a.channels; c += 256) sum += at(c);
    const float mean = sum_workgroup(sum, area) / (float)a.channels;
    for (int c = threadIdx.x; c < a.channels; c += 256) sq = fmaf(at(c) - mean, at(c) - mean, sq);
    const float rstd = 1.f / sqrtf(sum_workgroup(sq, area) / (float)a.channels + a.eps);
    if (a.stats && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
    for (int c = threadIdx.x; c < a.channels; c += 256) {
        const float s = at(c), h = (s - mean) * rstd;
        Values<T, 1> v{{s}}, y{{(a.weight ? h * a.weight[c] : h) + (a.bias ? a.bias[c] : 0.f)}};
        if (a.sum) v.store((T*)a.sum + row * a.lds + c);
        y.store((T*)a.y + row * a.ldy + c);
    }
}

// ------------------------------------------------------------------------------------------------ gradient
// A workgroup takes every blocks-th group of 256 / L rows; a lane's columns are the same in all of them, so dw and db stay in its registers, are added over
// the workgroup's rows at the end, and over the workgroups by a second launch, both in a fixed order.  The next group's row is on its way while one is summed.
template <typename T, int V, int L, int N>
__global__ __launch_bounds__(256) void seq_norm_grad_kernel(SeqNormArgs a) {
    constexpr int RW = 256 / L;
    const int l = threadIdx.x % L;
    const u32 block = workgroup();
    if (block >= (u32)a.blocks) return;
    float w[N][V], dw[N][V], db[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = (i * L + l) * V + e;
            w[i][e] = c >= a.channels ? 0.f : a.weight ? a.weight[c] : 1.f;
            dw[i][e] = db[i][e] = 0.f;
        }
    Pack<T, V> nx[N], ny[N], ne[N];
    float2 nst = make_float2(0.f, 0.f);
    auto request = [&](int64_t row) {
        if (row >= a.n) return;
        nst = *reinterpret_cast<const float2*>(a.stats + 2 * row);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * L + l) * V;
            if (c >= a.channels) continue;
            nx[i] = *reinterpret_cast<const Pack<T, V>*>((const T*)a.x + row * a.ldx + c);
            ny[i] = *reinterpret_cast<const Pack<T, V>*>((const T*)a.dy + row * a.lddy + c);
            if (a.res) ne[i] = *reinterpret_cast<const Pack<T, V>*>((const T*)a.res + row * a.ldr + c);
        }
    };
    const int64_t step = (int64_t)a.blocks * RW;
    int64_t row = (int64_t)block * RW + threadIdx.x / L;
    request(row);
    const float inv = 1.f / (float)a.channels;
    for (; row < a.n; row += step) {
        Pack<T, V> px[N], py[N], pe[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { px[i] = nx[i]; py[i] = ny[i]; pe[i] = ne[i]; }
        const float2 st = nst;
        request(row + step);
        float h[N][V], g[N][V], s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool in = (i * L + l) * V < a.channels;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[i][e] = in ? (px[i].get(e) - st.x) * st.y : 0.f;
                const float y = in ? py[i].get(e) : 0.f;
                dw[i][e] = fmaf(y, h[i][e], dw[i][e]);
                db[i][e] += y;
                g[i][e] = y * w[i][e];
                s0 += g[i][e];
                s1 = fmaf(g[i][e], h[i][e], s1);
            }
        }
        s0 = sum_lanes<L>(s0) * inv;
        s1 = sum_lanes<L>(s1) * inv;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * L + l) * V;
            if (c >= a.channels) continue;
            Values<T, V> y;
#pragma unroll
            for (int e = 0; e < V; ++e) y.v[e] = st.y * (g[i][e] - s0 - h[i][e] * s1) + (a.res ? pe[i].get(e) : 0.f);
            y.store((T*)a.dx + row * a.lddx + c);
        }
    }
    if (!a.dweight) return;
    // the workgroup's rows: lanes of a wave that hold the same columns, then the waves one after the other
    extern __shared__ float area[];   // [2][channels]
    const int wave = threadIdx.x >> 6;
    const bool mine = (threadIdx.x & 63) < L;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e)
#pragma unroll
            for (int d = L; d < 64; d <<= 1) {
                dw[i][e] += __shfl_xor(dw[i][e], d);
                db[i][e] += __shfl_xor(db[i][e], d);
            }
    float* out_w = a.blocks > 1 ? a.partial + (int64_t)block * 2 * a.channels : a.dweight;
    float* out_b = a.blocks > 1 ? out_w + a.channels : a.dbias;
    for (int k = 0; k < 4; ++k) {
        if (wave == k && mine) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int c = (i * L + l) * V + e;
                    if (c >= a.channels) continue;
                    const float sw = k ? area[c] + dw[i][e] : dw[i][e], sb = k ? area[a.channels + c] + db[i][e] : db[i][e];
                    if (k == 3) {
                        out_w[c] = sw;
                        out_b[c] = sb;
                    } else {
                        area[c] = sw;
                        area[a.channels + c] = sb;
                    }
                }
        }
        __syncthreads();
    }
}
// Wide rows: dx a workgroup a row; dw and db 256 columns and a range of rows a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void seq_norm_grad_wide_kernel(SeqNormArgs a) {
    __shared__ float area[4];
    const int64_t row = workgroup();
    if (row >= a.n) return;
    const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    auto h = [&](int c) { return (Pack<T, 1>{((const T*)a.x + row * a.ldx)[c]}.get(0) - st.x) * st.y; };
    auto g = [&](int c) { return Pack<T, 1>{((const T*)a.dy + row * a.lddy)[c]}.get(0) * (a.weight ? a.weight[c] : 1.f); };
    float s0 = 0.f, s1 = 0.f;
    for (int c = threadIdx.x; c < a.channels; c += 256) {
        s0 += g(c);
        s1 = fmaf(g(c), h(c), s1);
    }
    s0 = sum_workgroup(s0, area) / (float)a.channels;
    s1 = sum_workgroup(s1, area) / (float)a.channels;
    for (int c = threadIdx.x; c < a.channels; c += 256) {
        Values<T, 1> y{{st.y * (g(c) - s0 - h(c) * s1) + (a.res ? Pack<T, 1>{((const T*)a.res + row * a.ldr)[c]}.get(0) : 0.f)}};
        y.store((T*)a.dx + row * a.lddx + c);
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
        const float y = Pack<T, 1>{((const T*)a.dy + r * a.lddy)[c]}.get(0);
        dw = fmaf(y, (Pack<T, 1>{((const T*)a.x + r * a.ldx)[c]}.get(0) - st.x) * st.y, dw);
        db += y;
    }
    float* out = a.blocks > 1 ? a.partial + (int64_t)block * 2 * a.channels : nullptr;
    (out ? out : a.dweight)[c] = dw;
    (out ? out + a.channels : a.dbias)[c] = db;
}
// The sums of `blocks` rows of 2 * half columns, 16 columns a workgroup: four threads a row take four columns each, 64 rows' runs side by side, then the runs are
// added in their order.  Bound: latency; a thread's loads are all on their way together (1,024 rows of 1,024 columns: SUM_NOW us, with a column a thread and 16 runs 19.4).
__global__ __launch_bounds__(256) void sum_blocks_kernel(const float* partial, int blocks, int64_t half, float* out0, float* out1) {
    __shared__ float area[64][17];
    const int quad = threadIdx.x & 3, run = threadIdx.x >> 2;
    const int64_t n = 2 * half, c0 = (int64_t)workgroup() * 16, c = c0 + 4 * quad;
    const int per = (blocks + 63) / 64, b0 = run * per, b1 = min(b0 + per, blocks);
    float sum[4] = {};
    if (n % 4 == 0) {
        if (c < n)
#pragma unroll 8
            for (int b = b0; b < b1; ++b) {
                const float4 x = *reinterpret_cast<const float4*>(partial + b * n + c);
                sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
            }
    } else {
#pragma unroll 8
        for (int b = b0; b < b1; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += partial[b * n + min(c + e, n - 1)];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) area[run][4 * quad + e] = sum[e];
    __syncthreads();
    const int col = threadIdx.x & 15, part = threadIdx.x >> 4;
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x += area[4 * part + i][col];
    __syncthreads();
    area[part][col] = x;
    __syncthreads();
    if (part || c0 + col >= n) return;
#pragma unroll
    for (int p = 1; p < 16; ++p) x += area[p][col];
    if (c0 + col < half) out0[c0 + col] = x;
    else out1[c0 + col - half] = x;
}
void launch_sum_blocks(hipStream_t st, const float* partial, int blocks, int64_t half, float* out0, float* out1) {
    hipLaunchKernelGGL(sum_blocks_kernel, workgroups((2 * half + 15) / 16), dim3(256), 0, st, partial, blocks, half, out0, out1);
}

// ------------------------------------------------------------------------------------------------ launches
enum { NORM_BLOCKS = 1024 };   // most workgroups of the gradient
int64_t seq_norm_partials(int64_t n, int channels) { return std::min<int64_t>((n + 3) / 4, NORM_BLOCKS) * 2 * channels; }

// The widest access that all rows allow: 16, 8 bytes or an element.
static int pack_of(const SeqNormArgs& a, int elem) {
    for (int bytes : {16, 8}) {
        const int v = bytes / elem;
        bool ok = a.channels % v == 0;
        auto rows = [&](const void* p, int64_t ld) { ok = ok && (!p || ((uintptr_t)p % bytes == 0 && ld % v == 0)); };
        rows(a.x, a.ldx); rows(a.res, a.ldr); rows(a.y, a.ldy); rows(a.sum, a.lds); rows(a.dy, a.lddy); rows(a.dx, a.lddx);
        if (ok) return v;
    }
    return 1;
}
template <typename T, int V, int L, int N>
static void norm_rows(hipStream_t st, SeqNormArgs& a, bool grad) {
    const int64_t groups = (a.n + 256 / L - 1) / (256 / L);
    if (!grad) {
        hipLaunchKernelGGL((seq_norm_kernel<T, V, L, N>), workgroups(groups), dim3(256), 0, st, a);
        return;
    }
    const int64_t turns = (groups + NORM_BLOCKS - 1) / NORM_BLOCKS;   // (every workgroup as many)
    a.blocks = (int)((groups + turns - 1) / turns);
    hipLaunchKernelGGL((seq_norm_grad_kernel<T, V, L, N>), dim3(a.blocks), dim3(256), 2 * sizeof(float) * a.channels, st, a);
}
template <typename T, int V>
static bool norm_width(hipStream_t st, SeqNormArgs& a, bool grad) {   // false: too wide
    const int packs = (a.channels + V - 1) / V;
    if (packs <= 8) norm_rows<T, V, 8, 1>(st, a, grad);
    else if (packs <= 16) norm_rows<T, V, 16, 1>(st, a, grad);
    else if (packs <= 32) norm_rows<T, V, 32, 1>(st, a, grad);
    else if (packs <= 64) norm_rows<T, V, 64, 1>(st, a, grad);
    else if (packs <= 128) norm_rows<T, V, 64, 2>(st, a, grad);
    else if (packs <= 256) norm_rows<T, V, 64, 4>(st, a, grad);
    else if (V < 8 && packs <= 512) norm_rows<T, V, 64, V < 8 ? 8 : 1>(st, a, grad);
    else if (V == 1 && packs <= 1024) norm_rows<T, V, 64, V == 1 ? 16 : 1>(st, a, grad);
    else return false;
    return true;
}
template <typename T>
static void norm_type(hipStream_t st, SeqNormArgs a, bool grad) {
    constexpr int V = 16 / sizeof(T);
    const int v = pack_of(a, sizeof(T));
    const bool fits = v == V ? norm_width<T, V>(st, a, grad) : v == V / 2 ? norm_width<T, V / 2>(st, a, grad) : norm_width<T, 1>(st, a, grad);
    if (!fits && !grad) hipLaunchKernelGGL((seq_norm_wide_kernel<T>), workgroups(a.n), dim3(256), 0, st, a);
    if (!fits && grad) {
        hipLaunchKernelGGL((seq_norm_grad_wide_kernel<T>), workgroups(a.n), dim3(256), 0, st, a);
        if (a.dweight) {
            const int64_t columns = (a.channels + 255) / 256;
            a.blocks = (int)std::min<int64_t>((a.n + 15) / 16, std::max<int64_t>(1, NORM_BLOCKS / columns));
            hipLaunchKernelGGL((seq_norm_columns_kernel<T>), workgroups(a.blocks * columns), dim3(256), 0, st, a, (u32)columns);
        }
    }
    if (grad && a.dweight && a.blocks > 1) launch_sum_blocks(st, a.partial, a.blocks, a.channels, a.dweight, a.dbias);
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
