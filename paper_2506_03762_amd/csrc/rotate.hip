// Rotation of query and key rows by their positions, and its use in appending to a paged cache.
//
// Pair (x0, x1) -> (x0 cos t - x1 sin t, x0 sin t + x1 cos t) with t = position x frequency: three operations per
// element read and written, so the bytes bound it.  What keeps the angles off that path: a thread owns the same
// sixteen-byte chunks of a token's row in all heads, forms the sines and cosines of its eight pairs (fp32: four) once, while the
// first heads' rows travel, and then goes through the heads.  Positions may be far (2^31) and the frequency 1: the
// angle is formed in turns from a frequency in two doubles (with one it is off by up to 2^-52 of its turns, 7e-8 of a turn
// at 2^31), its whole turns are taken away there, and only the rest, at most half a turn, becomes an fp32
// number; what that rounds off (up to 2^-26 of a turn, 1e-7 of the result) turns the sine and cosine to first order.
//
// 32768 tokens of 32 + 8 heads, d = 128: 671 MB in 134 us, 5.0 TB/s (a copy reaches 4.8); 3 x 5003 tokens of 12 + 4 heads 26 us for the kernel, 29 a
// call.  64 single tokens: 6 us, the round trips of tail length, page and store.
#include <algorithm>

#include "aha_dev.h"
#include "aha_host.h"

namespace aha {

constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;  // 1 / (2 pi), and what is left of it

// A row of d channels as D / CE chunks of 16 bytes, two of them per thread: of the rotated channels those whose elements
// make pairs, of the others two neighbours.
template <class T>
struct RowChunks {
    static constexpr int CE = 16 / sizeof(T);  // elements of a chunk, pairs of a thread
    int first, second;
    bool turned;
    __device__ __forceinline__ RowChunks(int c, int rot, bool neighbours) {
        const int np = rot / (2 * CE);  // threads with pairs
        turned = c < np;
        first = turned && !neighbours ? c : 2 * c;
        second = turned && !neighbours ? c + np : 2 * c + 1;
    }
};

__device__ __forceinline__ void unpack(const u32x4 &w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
}
__device__ __forceinline__ void unpack(const u32x4 &w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
    __bf16 b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (__bf16)x[i];
    u32x4 w;
    __builtin_memcpy(&w, b, 16);
    return w;
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

// The two chunks of a row, turned in place.
template <class T, bool NEIGHBOURS>
__device__ __forceinline__ void turn(u32x4 &w0, u32x4 &w1, const float (&cs)[RowChunks<T>::CE], const float (&sn)[RowChunks<T>::CE]) {
    constexpr int CE = RowChunks<T>::CE;
    float a[CE], b[CE];
    unpack(w0, a);
    unpack(w1, b);
    if constexpr (NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < CE / 2; ++i) {
            const float x = a[2 * i], y = a[2 * i + 1];
            a[2 * i] = x * cs[i] - y * sn[i];
            a[2 * i + 1] = x * sn[i] + y * cs[i];
            const float u = b[2 * i], v = b[2 * i + 1];
            b[2 * i] = u * cs[CE / 2 + i] - v * sn[CE / 2 + i];
            b[2 * i + 1] = u * sn[CE / 2 + i] + v * cs[CE / 2 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < CE; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * cs[i] - y * sn[i];
            b[i] = x * sn[i] + y * cs[i];
        }
    }
    w0 = pack(a);
    w1 = pack(b);
}

constexpr int kHeadsAhead = 4;  // rows of a thread in flight

// A workgroup takes 256 / TPR tokens (TPR threads per row) and the heads [blockIdx.y * per, + per) of the Hq + Hkv (APPEND: +
// Hkv value heads, which are copied).
template <class T, int D, bool NEIGHBOURS, bool APPEND>
__global__ __launch_bounds__(256) void rotate_kernel(RotaryGeom g, int per) {
    constexpr int CE = RowChunks<T>::CE, TPR = D / (2 * CE), U = kHeadsAhead;
    const int c = threadIdx.x % TPR;
    const int64_t token = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (token >= (int64_t)g.batch * g.n) return;
    const int b = (int)token / g.n, t = (int)token - b * g.n;
    const int heads = g.Hq + (APPEND ? 2 : 1) * g.Hkv, h0 = blockIdx.y * per, h1 = min(heads, h0 + per);
    const RowChunks<T> ch(c, g.rot, NEIGHBOURS);
    int64_t k_at = 0, v_at = 0;  // APPEND: the token's row in the pools, without the head
    bool placed = true;
    int fresh = g.n;
    if constexpr (APPEND) {
        if (g.pages.new_len) fresh = min(g.pages.new_len[b], g.n);
        if (t >= fresh) return;  // padding
    }
    auto source = [&](int h) {
        const T *p = h < g.Hq            ? (const T *)g.q + b * g.qs[0] + h * g.qs[1] + t * g.qs[2]
                     : h < g.Hq + g.Hkv  ? (const T *)g.k + b * g.ks[0] + (h - g.Hq) * g.ks[1] + t * g.ks[2]
                                         : (const T *)g.v + b * g.vs[0] + (h - g.Hq - g.Hkv) * g.vs[1] + t * g.vs[2];
        return p;
    };
    auto target = [&](int h) {
        T *p = h < g.Hq           ? (T *)g.q_out + b * g.qo[0] + h * g.qo[1] + t * g.qo[2]
               : !APPEND          ? (T *)g.k_out + b * g.ko[0] + (h - g.Hq) * g.ko[1] + t * g.ko[2]
               : h < g.Hq + g.Hkv ? (T *)g.k_out + k_at + (h - g.Hq) * g.pages.ks[1]
                                  : (T *)g.v_out + v_at + (h - g.Hq - g.Hkv) * g.pages.vs[1];
        return p;
    };
    u32x4 w[U][2];
    auto request = [&](int h) {  // (past the last head: that one again)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const T *p = source(min(h + u, h1 - 1));
            w[u][0] = *(const u32x4 *)(p + ch.first * CE);
            w[u][1] = *(const u32x4 *)(p + ch.second * CE);
        }
    };
    request(h0);
    if constexpr (APPEND) {  // (looked up while the rows travel)
        const int64_t slot = (int64_t)g.pages.tail_len[b] - fresh + t, entry = slot >> g.pages.page_shift;
        placed = slot >= 0 && entry < g.pages.table_width;
        const int page = placed ? g.pages.table[(int64_t)b * g.pages.table_width + entry] : -1;
        placed = page >= 0 && page < g.pages.n_pages;
        const int row = (int)slot & ((1 << g.pages.page_shift) - 1);
        k_at = page * g.pages.ks[0] + row * g.pages.ks[2];
        v_at = page * g.pages.vs[0] + row * g.pages.vs[2];
    }
    float cs[CE], sn[CE];
#pragma unroll
    for (int i = 0; i < CE; ++i) cs[i] = 1.f, sn[i] = 0.f;
    if (ch.turned) {
#pragma unroll
        for (int i = 0; i < CE; ++i) {
            const int f = c * CE + i;
            const int axis = g.pair_axis ? min(max(g.pair_axis[f], 0), g.n_axes - 1) : 0;
            const int pos = g.positions[(int64_t)axis * g.batch * g.n + token];
            const double w = (double)g.inv_freq[f], w1 = w * kTurn, w2 = fma(w, kTurn, -w1) + w * kTurnRest;
            const double turns = fma((double)pos, w2, fma((double)pos, w1, -rint((double)pos * w1)));
            const float part = (float)turns, rest = (float)((turns - (double)part) * 6.283185307179586477);
            float s0, c0;
            sincospif(2.f * part, &s0, &c0);
            cs[i] = fmaf(-rest, s0, c0);
            sn[i] = fmaf(rest, c0, s0);
            if (g.transpose) sn[i] = -sn[i];
        }
    }
    for (int h = h0; h < h1; h += U) {
        u32x4 x[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u][0] = w[u][0], x[u][1] = w[u][1];
        if (h + U < h1) request(h + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h + u >= h1) break;
            const bool key = h + u >= g.Hq, value = APPEND && h + u >= g.Hq + g.Hkv;
            if (ch.turned && !value) turn<T, NEIGHBOURS>(x[u][0], x[u][1], cs, sn);
            if (key && !placed) continue;
            T *p = target(h + u);
            *(u32x4 *)(p + ch.first * CE) = x[u][0];
            *(u32x4 *)(p + ch.second * CE) = x[u][1];
        }
    }
}

template <class T, int D, bool NEIGHBOURS, bool APPEND>
static hipError_t launch_rotate_t(const RotaryGeom &g, hipStream_t st) {
    constexpr int tokens = 256 * 2 * RowChunks<T>::CE / D;
    const int64_t tiles = ((int64_t)g.batch * g.n + tokens - 1) / tokens;
    const int heads = g.Hq + (APPEND ? 2 : 1) * g.Hkv;
    // Heads are dealt over workgroups, each of which forms the angles again, until 384 workgroups have work (us with 256, 384, 512, 1024, 4096
    // of them: 8 x 821 tokens, 32 + 8 heads, turned 31.5, 31.6, 33.4, 35.8, 46.2; appended 37.3, 37.4, 39.8, 42.6, 50.6; 8 x 200 turned
    // 11.1, 11.2, 10.7, 13.1, 18.1).  Prompts of more than three tiles per CU whose heads' tokens lie together: nine heads or more
    // to a workgroup (bf16, d = 128; fp32 goes the same way: 20 heads with one, two, four workgroups to a tile 48.5, 50.2, 56.8 at 700 tiles, 58.0, 55.4, 62.3 at 780, 76.3,
    // 71.6, 80.2 at 1030; 40 heads 94.6, 96.0, 92.7; 113.5, 106.2, 102.6; 151.0, 143.3, 133.6; 8 heads 18.4, 23.8, 30.3 at 700, 29.2, 35.8, 42.2 at 1030; 72 heads
    // with one, four, eight 270.2, 246.3, 232.9).  Where a token's heads lie together one workgroup is within 3 % of the best at such lengths (40 heads,
    // 1024 tiles, one, two, four 146.7, 149.6, 151.2).
    const bool head_major = g.Hq > 1 ? g.qs[1] > g.qs[2] : g.ks[1] > g.ks[2];
    const int64_t dealt = !APPEND && head_major && tiles > 3 * 256 ? heads / 9 : (384 + tiles - 1) / tiles;
    const int64_t split = std::min<int64_t>(std::max<int64_t>(1, dealt), heads);
    const int per = (int)((heads + split - 1) / split);
    hipLaunchKernelGGL((rotate_kernel<T, D, NEIGHBOURS, APPEND>), dim3((unsigned)tiles, (heads + per - 1) / per), dim3(256), 0, st, g, per);
    return hipGetLastError();
}

template <class T, int D>
static hipError_t launch_rotate_d(const RotaryGeom &g, hipStream_t st) {
    if (g.neighbours) return g.append ? launch_rotate_t<T, D, true, true>(g, st) : launch_rotate_t<T, D, true, false>(g, st);
    return g.append ? launch_rotate_t<T, D, false, true>(g, st) : launch_rotate_t<T, D, false, false>(g, st);
}

hipError_t launch_rotate(const RotaryGeom &g, hipStream_t st) {
    if (g.dtype == AHA_BF16) return g.d == 64 ? launch_rotate_d<__bf16, 64>(g, st) : launch_rotate_d<__bf16, 128>(g, st);
    return g.d == 64 ? launch_rotate_d<float, 64>(g, st) : launch_rotate_d<float, 128>(g, st);
}

}  // namespace aha
