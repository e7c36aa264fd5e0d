// Attention of a batch's new tokens over the prefixes that its sequences share and over their own tails in pages.
#include "aha_dev.h"
#include "aha_host.h"

namespace aha {

// The keys of a sequence's row: prefix tokens [0, ahead), then tail tokens [0, behind).
struct RowKeys {
    int prefix, ahead, behind;
};
__device__ __forceinline__ RowKeys row_keys(const SharedGeom &g, int b, int t, int fresh) {
    RowKeys r{-1, 0, 0};
    int lo = 0, hi = g.n_prefixes;  // the last prefix that begins at or before b
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (g.prefix_first[mid] <= b) lo = mid + 1; else hi = mid;
    }
    if (lo > 0 && b < g.prefix_first[lo]) {
        r.prefix = lo - 1;
        r.ahead = min(max(g.prefix_len[r.prefix], 0), g.prefix_cap);
    }
    if (g.kt) {
        const int64_t seen = (int64_t)g.pages.tail_len[b] - fresh + t + 1;
        r.behind = (int)max((int64_t)0, min(seen, (int64_t)g.pages.table_width << g.pages.page_shift));
    }
    return r;
}

// A workgroup per row; keys in blocks of 256, one per thread, then a channel per thread.
template <class T, int D>
__global__ __launch_bounds__(256) void shared_attn_kernel(SharedGeom g) {
    constexpr int SL = 256 / D, CE = 16 / sizeof(T);
    const int rows = g.G * g.n, b = blockIdx.x / rows, rr = blockIdx.x % rows, gi = rr / g.n, t = rr % g.n;
    const int h = blockIdx.y, hq = h * g.G + gi, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int fresh = g.pages.new_len ? min(max(g.pages.new_len[b], 0), g.n) : g.n;
    if (t >= fresh) return;
    const RowKeys rk = row_keys(g, b, t, fresh);
    const int64_t keys = (int64_t)rk.ahead + rk.behind;
    __shared__ float s_q[D], s_p[256], s_red[4], s_o[SL][D];
    __shared__ const T *s_v[256];
    if (tid < D) s_q[tid] = (float)((const T *)g.q + b * g.qs[0] + hq * g.qs[1] + t * g.qs[2])[tid];
    __syncthreads();
    const float c_out = g.scale * kLog2e;
    const int c = tid % D, sl = tid / D;
    float m = -INFINITY, ssum = 0.f, o = 0.f;
    for (int64_t j0 = 0; j0 < keys; j0 += 256) {
        const int64_t j = j0 + tid;
        const T *kr = nullptr, *vr = nullptr;
        if (j < rk.ahead) {
            kr = (const T *)g.kp + rk.prefix * g.ks[0] + h * g.ks[1] + j * g.ks[2];
            vr = (const T *)g.vp + rk.prefix * g.vs[0] + h * g.vs[1] + j * g.vs[2];
        } else if (j < keys) {
            const int s = (int)(j - rk.ahead), row = s & ((1 << g.pages.page_shift) - 1);
            const int page = g.pages.table[(int64_t)b * g.pages.table_width + (s >> g.pages.page_shift)];
            if (page >= 0 && page < g.pages.n_pages) {
                kr = (const T *)g.kt + page * g.pages.ks[0] + h * g.pages.ks[1] + row * g.pages.ks[2];
                vr = (const T *)g.vt + page * g.pages.vs[0] + h * g.pages.vs[1] + row * g.pages.vs[2];
            }
        }
        float x = -INFINITY;
        if (kr) {
            float w = 0.f;
            for (int cc = 0; cc < D / CE; ++cc) {
                T e[CE];
                __builtin_memcpy(e, kr + cc * CE, 16);
                for (int i = 0; i < CE; ++i) w = fmaf(s_q[cc * CE + i], (float)e[i], w);
            }
            x = w * c_out;
        }
        const float wm = wave_max(x);
        if (lane == 0) s_red[wave] = wm;
        __syncthreads();
        const float mn = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
        const float mref = mn == -INFINITY ? 0.f : mn;
        const float pr = exp2f(x - mref);
        s_p[tid] = pr;
        s_v[tid] = vr;
        const float ws = wave_sum(pr);
        __syncthreads();
        if (lane == 0) s_red[wave] = ws;
        __syncthreads();
        const float corr = exp2f(m - mref);
        ssum = ssum * corr + (s_red[0] + s_red[1] + s_red[2] + s_red[3]);
        o *= corr;
        for (int jj = sl; jj < 256; jj += SL)
            if (s_v[jj]) o = fmaf(s_p[jj], (float)s_v[jj][c], o);
        m = mn;
        __syncthreads();
    }
    s_o[sl][c] = o;
    __syncthreads();
    if (tid < D) {
        float tot = 0.f;
        for (int t2 = 0; t2 < SL; ++t2) tot += s_o[t2][tid];
        ((T *)g.out + b * g.os[0] + hq * g.os[1] + t * g.os[2])[tid] = (T)(ssum == 0.f ? 0.f : tot / ssum);
        if (g.lse && tid == 0)
            g.lse[((int64_t)b * g.Hq + hq) * g.n + t] = ssum == 0.f ? -INFINITY : (m + log2f(ssum)) * 0.69314718055994531f;
    }
}

hipError_t launch_shared_attention(const SharedGeom &g, const SharedPlan &, void *, hipStream_t st) {
    const dim3 grid((unsigned)(g.batch * g.G * g.n), g.Hkv);
    if (g.dtype == AHA_BF16 && g.d == 64) hipLaunchKernelGGL((shared_attn_kernel<__bf16, 64>), grid, dim3(256), 0, st, g);
    else if (g.dtype == AHA_BF16) hipLaunchKernelGGL((shared_attn_kernel<__bf16, 128>), grid, dim3(256), 0, st, g);
    else if (g.d == 64) hipLaunchKernelGGL((shared_attn_kernel<float, 64>), grid, dim3(256), 0, st, g);
    else hipLaunchKernelGGL((shared_attn_kernel<float, 128>), grid, dim3(256), 0, st, g);
    return hipGetLastError();
}

}  // namespace aha
