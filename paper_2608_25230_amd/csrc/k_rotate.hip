// Queries and keys to their positions (fw_rotate_heads): each head's row x of d
// columns is normed,
//
//   y = x w / sqrt(mean x^2 + eps),
//
// and its pairs of columns turn by the position's angle, (u, v) -> (u cos a -
// v sin a, v cos a + u sin a), a = pos freq.  The angle is taken in float64 as
// a part of a full turn, so far positions lose nothing; what is left of it, at
// most half a turn, goes to float32.
//
// Memory bounds it: a row is read and written once, a dozen operations a
// column.  A token's sines and cosines are taken once, into LDS, for all its
// heads; a row lies in few lanes (8 for 128 columns of bf16), so that its sum of
// squares takes few shuffles, and the next row is loaded before the one at hand
// is done, the first one before the angles (16384 tokens of 40 heads of 128
// columns, bf16 with norms: 77 us without, 65 with, 5.2 TB/s).
#include <algorithm>

#include "fw_internal.hpp"

namespace fw {

namespace {
constexpr int RT = 256;      // threads of a workgroup
constexpr int kTokens = 8;   // tokens of a workgroup at most
constexpr int kLong = 4096;  // tokens that are many
constexpr int kPairs = 128;  // pairs of a row at most

struct RotateArgs {
    const void *in[2];                 // queries, keys
    void *out[2];
    const void *weight[2];
    int64_t row[2], head[2], orow[2], ohead[2];
    int H[2];
    int64_t T;
    int tokens;                        // of a workgroup
    int d, rot, lanes;                 // lanes of a row, a power of two
    const int64_t *pos;
    const float *freq;
    bool interleaved, norm, w32;
    float eps;
};

template <typename T> __device__ __forceinline__ T rnarrow(float x);
template <> __device__ __forceinline__ float rnarrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t rnarrow<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T, int V> struct alignas(V * sizeof(T)) Piece {
    T x[V];
};
template <typename T, int V>
__device__ __forceinline__ void put(T *p, const float (&y)[V]) {
    Piece<T, V> z;
#pragma unroll
    for (int i = 0; i < V; ++i) z.x[i] = rnarrow<T>(y[i]);
    *(Piece<T, V> *)p = z;
}

// A lane holds two pieces of V columns: of a row that turns by halves, columns
// c .. c + V and their partners; otherwise, and past the columns that turn, 2 V
// neighbouring columns.  NC such pairs of pieces a lane, so that 64 lanes hold
// any row.
template <typename T, int V, int NC>
__global__ void __launch_bounds__(RT) rotate_heads(RotateArgs a) {
    __shared__ float cs[kTokens][kPairs], sn[kTokens][kPairs];
    __shared__ float wt[2][2 * kPairs];
    const int tid = threadIdx.x, half = a.rot / 2;
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
    const int nt = a.T - t0 < a.tokens ? (int)(a.T - t0) : a.tokens;
    const int lane = tid & (a.lanes - 1), slot = tid / a.lanes, slots = RT / a.lanes;
    int c0[NC], c1[NC], pair[NC];  // columns of the two pieces, the first pair (-1: they do not turn)
    const int turning = half / V;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        const int i = lane + n * a.lanes;
        if (i < turning) {
            c0[n] = a.interleaved ? 2 * V * i : V * i;
            c1[n] = a.interleaved ? c0[n] + V : c0[n] + half;
            pair[n] = V * i;
        } else {
            c0[n] = a.rot + 2 * V * (i - turning);
            c1[n] = c0[n] + V;
            pair[n] = -1;
        }
    }
    const int heads = a.H[0] + a.H[1], rows = nt * heads;
    Piece<T, V> next[NC][2];  // a row ahead
    const auto load = [&](int r) {
        const int t = r / heads, hh = r - t * heads, s = hh >= a.H[0], h = hh - (s ? a.H[0] : 0);
        const T *p = (const T *)a.in[s] + (t0 + t) * a.row[s] + h * a.head[s];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            next[n][0] = next[n][1] = Piece<T, V>{};
            if (c0[n] < a.d) next[n][0] = *(const Piece<T, V> *)(p + c0[n]);
            if (c1[n] < a.d) next[n][1] = *(const Piece<T, V> *)(p + c1[n]);
        }
    };
    if (slot < rows) load(slot);
    for (int i = tid; i < nt * half; i += RT) {
        const int t = i / half, j = i - t * half;
        double turns = (double)a.pos[t0 + t] * (double)a.freq[j] * 0.15915494309189533577;
        turns -= rint(turns);
        sincospif((float)(2.0 * turns), &sn[t][j], &cs[t][j]);
    }
    if (a.norm)
        for (int i = tid; i < 2 * a.d; i += RT) {
            const int s = i >= a.d, c = i - s * a.d;
            const void *w = a.weight[s];
            wt[s][c] = !w ? 1.f : a.w32 ? ((const float *)w)[c] : bf16_bits_to_f32(((const uint16_t *)w)[c]);
        }
    __syncthreads();
    const float inv_d = 1.f / a.d;
    for (int r = slot; r < rows; r += slots) {
        const int t = r / heads, hh = r - t * heads, s = hh >= a.H[0], h = hh - (s ? a.H[0] : 0);
        T *o = (T *)a.out[s] + (t0 + t) * a.orow[s] + h * a.ohead[s];
        float x[NC][2][V];
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int i = 0; i < V; ++i)
                x[n][0][i] = Elem<T>::load(next[n][0].x, i), x[n][1][i] = Elem<T>::load(next[n][1].x, i);
        if (r + slots < rows) load(r + slots);
        if (a.norm) {
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int i = 0; i < V; ++i) sum += x[n][0][i] * x[n][0][i] + x[n][1][i] * x[n][1][i];
            for (int off = a.lanes / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
            const float f = 1.f / sqrtf(sum * inv_d + a.eps);
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (c0[n] < a.d) x[n][0][i] *= f * wt[s][c0[n] + i];
                    if (c1[n] < a.d) x[n][1][i] *= f * wt[s][c1[n] + i];
                }
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            if (pair[n] >= 0) {
                float y[2 * V];
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) y[i] = x[n][i / V][i % V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float c = cs[t][pair[n] + i], z = sn[t][pair[n] + i];
                    if (a.interleaved) {
                        const float u = y[2 * i], v = y[2 * i + 1];
                        x[n][(2 * i) / V][(2 * i) % V] = u * c - v * z;
                        x[n][(2 * i + 1) / V][(2 * i + 1) % V] = v * c + u * z;
                    } else {
                        const float u = y[i], v = y[V + i];
                        x[n][0][i] = u * c - v * z;
                        x[n][1][i] = v * c + u * z;
                    }
                }
            }
            if (c0[n] < a.d) put<T, V>(o + c0[n], x[n][0]);
            if (c1[n] < a.d) put<T, V>(o + c1[n], x[n][1]);
        }
    }
}

template <typename T>
hipError_t launch_width(RotateArgs &a, int v, hipStream_t st) {
    const int pieces = (a.d + 2 * v - 1) / (2 * v);
    a.lanes = 1;
    while (a.lanes < pieces && a.lanes < 64) a.lanes *= 2;
    // As many tokens as the threads take rows of at once, twice where tokens are many: a workgroup's first rows wait for
    // its tokens' angles, which a few rows do not make up for, and too few workgroups leave the card idle.  bf16 with
    // norms, by 1, 2, 4, 8 tokens: 1024 of 32 heads of 256 columns 12, 13, 21, 36 us; 4096 of 40 heads of 128 21, 19, 20,
    // 27; 16384 of those 67, 65, 64, 68; 65536 of 9 heads of 128 128, 87, 70, 63.  A grid holds 2^24 workgroups.
    const int heads = a.H[0] + a.H[1], rows = RT / a.lanes * (a.T >= kLong ? 2 : 1);
    a.tokens = std::max(std::min((rows + heads - 1) / heads, kTokens), (int)((a.T + (1 << 23) - 1) >> 23));
    const dim3 grid((unsigned)((a.T + a.tokens - 1) / a.tokens));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(RT), 0, st, a); };
    if constexpr (sizeof(T) == 2) {
        if (v == 8) return run(rotate_heads<T, 8, 1>), hipGetLastError();
    }
    if (v == 4) run(rotate_heads<T, 4, 1>);
    else if (v == 2) run(rotate_heads<T, 2, 1>);
    else if (pieces <= 64) run(rotate_heads<T, 1, 1>);
    else run(rotate_heads<T, 1, 2>);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_rotate(const fw_heads &h, void *q_out, int64_t qo_row, int64_t qo_head, void *k_out, int64_t ko_row,
                         int64_t ko_head, hipStream_t st) {
    RotateArgs a{};
    a.in[0] = h.q, a.in[1] = h.k, a.out[0] = q_out, a.out[1] = k_out;
    a.row[0] = h.q_row, a.row[1] = h.k_row, a.head[0] = h.q_head, a.head[1] = h.k_head;
    a.orow[0] = qo_row, a.orow[1] = ko_row, a.ohead[0] = qo_head, a.ohead[1] = ko_head;
    a.weight[0] = h.q_weight, a.weight[1] = h.k_weight, a.w32 = h.w_dtype == FW_F32;
    a.H[0] = (int)h.Hq, a.H[1] = (int)h.Hkv;
    a.T = h.T, a.d = (int)h.d, a.rot = (int)h.rot, a.pos = h.pos, a.freq = h.freq;
    a.interleaved = h.interleaved != 0, a.norm = h.norm != 0, a.eps = h.eps;
    // the widest pieces that columns, strides and addresses allow
    const int size = h.dtype == FW_F32 ? 4 : 2;
    int v = 16 / size;
    const auto fits = [&](int w) {
        if ((a.rot / 2) % w || (a.d - a.rot) % w) return false;
        for (int s = 0; s < 2; ++s)
            if (a.H[s] && ((uintptr_t)a.in[s] % (w * size) || (uintptr_t)a.out[s] % (w * size) || a.row[s] % w || a.head[s] % w ||
                           a.orow[s] % w || a.ohead[s] % w))
                return false;
        return true;
    };
    while (v > 1 && !fits(v)) v /= 2;
    return h.dtype == FW_F32 ? launch_width<float>(a, v, st) : launch_width<uint16_t>(a, v, st);
}

}  // namespace fw
