// kv_attn: attention of new queries over the pages of the cache.
#include "aa_kv.h"

namespace aa {
namespace {

// Eight channels of a cached row as floats.
template <class T, bool FP4>
__device__ __forceinline__ void row8(const char* pool, const unsigned char* sc, const long long* cs, const long long* ss, int page, int h,
                                     int in, int c, float* x) {
    if constexpr (FP4) {
        const unsigned codes = *(const unsigned*)(pool + page * cs[0] + h * cs[1] + in * cs[2] + c / 2);
        const int byte = sc[page * ss[0] + h * ss[1] + c / kFp4Group * ss[2] + in];
        for (int e = 0; e < 8; ++e) x[e] = fp4_value(codes >> (4 * e) & 15, byte);
    } else {
        const T* p = (const T*)pool + page * cs[0] + h * cs[1] + in * cs[2] + c;
        for (int e = 0; e < 8; ++e) x[e] = (float)p[e];
    }
}

// One wave a row: 64 keys at a time, a key a lane for the scores, channels across the lanes for the sum.
template <class T, bool FP4, int D>
__global__ __launch_bounds__(64) void kv_attn_kernel(KvArgs a, const T* q, T* out, float* lse) {
    __shared__ float s_q[D], s_p[64];
    __shared__ int s_page[64];
    const int lane = threadIdx.x, b = blockIdx.z, h = blockIdx.y, i = blockIdx.x, hk = h / a.grp;
    const KvSeq sq = kv_seq(a, b);
    if (i >= sq.n) return;
    for (int c = lane; c < D; c += 64) s_q[c] = (float)q[kv_row(a, a.qs, b, sq.row0, i, h) + c];
    __syncthreads();
    const long long len = a.kv_len[b], room = (long long)a.max_pages << a.page_shift;
    long long see = a.causal ? len - sq.n + i + 1 : len;
    if (see > room) see = room;
    float m = -INFINITY, l = 0.f, acc[(D + 63) / 64] = {};
    for (long long j0 = 0; j0 < see; j0 += 64) {
        const long long j = j0 + lane;
        const int page = j < see ? kv_page(a, b, j) : -1, in = (int)j & ((1 << a.page_shift) - 1);
        float s = -INFINITY;
        if (page >= 0) {
            s = 0.f;
            for (int c = 0; c < D; c += 8) {
                float x[8];
                row8<T, FP4>(a.kc, a.ksc, a.kcs, a.kss, page, hk, in, c, x);
                for (int e = 0; e < 8; ++e) s = fmaf(x[e], s_q[c + e], s);
            }
            s *= a.sigma;
        }
        float t = s;
        for (int x = 32; x; x >>= 1) t = fmaxf(t, __shfl_xor(t, x));
        const float top = fmaxf(m, t), ref = top == -INFINITY ? 0.f : top;
        const float e = expf(s - ref), down = expf(m - ref);
        m = top;
        s_p[lane] = e;
        s_page[lane] = page;
        float sum = e;
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        l = l * down + sum;
        __syncthreads();
        for (int cc = 0; cc < (D + 63) / 64; ++cc) {
            const int c = cc * 64 + lane;
            acc[cc] *= down;
            if (c < D)
                for (int x = 0; x < 64; ++x) {
                    if (s_page[x] < 0) continue;
                    float v[8];
                    row8<T, FP4>(a.vc, a.vsc, a.vcs, a.vss, s_page[x], hk, (int)(j0 + x) & ((1 << a.page_shift) - 1), c & ~7, v);
                    acc[cc] = fmaf(s_p[x], v[c & 7], acc[cc]);
                }
        }
        __syncthreads();
    }
    for (int cc = 0; cc < (D + 63) / 64; ++cc) {
        const int c = cc * 64 + lane;
        if (c < D) out[kv_row(a, a.os, b, sq.row0, i, h) + c] = (T)(l == 0.f ? 0.f : acc[cc] / l);
    }
    if (lse && lane == 0)
        lse[a.cu ? h * a.total + sq.row0 + i : ((long long)b * a.Hq + h) * a.N + i] = l == 0.f ? -INFINITY : m + logf(l);
}

template <class T, bool FP4, int D>
int run(const KvArgs& a, const void* q, void* out, float* lse, hipStream_t st) {
    return (int)launch_kernel(kv_attn_kernel<T, FP4, D>, dim3(a.N, a.Hq, a.B), dim3(64), 0, st, a, (const T*)q, (T*)out, lse);
}

}  // namespace

KvSplit kv_split(int, int, int, int, int, int, long long) { return KvSplit{1, 0, 0}; }

int launch_kv_attn(const KvArgs& a, int dtype, int format, int d, const KvSplit&, const void* q, void* out, float* lse, float*,
                   hipStream_t st) {
    if (dtype == 0) return d == 32 ? run<float, false, 32>(a, q, out, lse, st) : d == 64 ? run<float, false, 64>(a, q, out, lse, st)
                         : d == 128 ? run<float, false, 128>(a, q, out, lse, st) : -1;
    if (format) return d == 64 ? run<__bf16, true, 64>(a, q, out, lse, st) : d == 128 ? run<__bf16, true, 128>(a, q, out, lse, st) : -1;
    return d == 64 ? run<__bf16, false, 64>(a, q, out, lse, st) : d == 128 ? run<__bf16, false, 128>(a, q, out, lse, st) : -1;
}

}  // namespace aa
