// kv_append and kv_read: rows of new tokens into the pages of the cache (rotated on the way) and out of them.
#include "aa_kv.h"

namespace aa {
namespace {

using u32x4 = __attribute__((ext_vector_type(4))) unsigned;

template <class T> struct Vec;                  // 16 bytes of a row
template <> struct Vec<float> { static constexpr int n = 4; };
template <> struct Vec<__bf16> { static constexpr int n = 8; };

template <class T> __device__ __forceinline__ void load16(const T* p, float* x) {
    union { u32x4 u; T t[Vec<T>::n]; } v;
    v.u = *(const u32x4*)p;
    for (int i = 0; i < Vec<T>::n; ++i) x[i] = (float)v.t[i];
}
template <class T> __device__ __forceinline__ void store16(T* p, const float* x) {
    union { u32x4 u; T t[Vec<T>::n]; } v;
    for (int i = 0; i < Vec<T>::n; ++i) v.t[i] = (T)x[i];
    *(u32x4*)p = v.u;
}

struct AppendArgs {
    KvArgs a;
    const void *q, *k, *v;
    const float* inv_freq;
    const int* positions;
    void *q_out, *k_out;
};

// Which sequence a row of the token axis belongs to: B if none.
__device__ __forceinline__ int seq_of_row(const KvArgs& a, long long row) {
    if (!a.cu) return (int)(row / a.N);
    int b = 0;
    for (int at = 0; at < a.B; at += 64) {      // sequences that end at or before the row
        const int i = at + (threadIdx.x & 63);
        b += __popcll(__ballot(i < a.B && a.cu[i + 1] <= row));
    }
    return b;
}

// One work-group a token: cosines and sines of its position first, once for all heads; then 16 bytes of a head's row a thread.
template <class T, bool FP4, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs p) {
    constexpr int V = Vec<T>::n, LANES = D / V;
    __shared__ double s_cos[D / 2], s_sin[D / 2];
    const KvArgs& a = p.a;
    const long long row = blockIdx.x;
    const int b = seq_of_row(a, row);
    if (b >= a.B) return;
    const KvSeq sq = kv_seq(a, b);
    const int i = (int)(row - sq.row0);
    if (i < 0 || i >= sq.n) return;
    const long long j = (long long)a.kv_len[b] - sq.n + i;
    const double pos = p.positions ? (double)p.positions[row] : (double)j;
    for (int f = threadIdx.x; f < a.rot / 2; f += 256) {
        double sn, cs;
        sincos(pos * (double)p.inv_freq[f], &sn, &cs);
        s_cos[f] = cs; s_sin[f] = sn;
    }
    __syncthreads();
    const int page = kv_page(a, b, j), in = (int)j & ((1 << a.page_shift) - 1);
    const int nq = p.q_out ? a.Hq : 0, nk = p.k ? a.Hkv : 0;
    for (int r = threadIdx.x / LANES; r < nq + 2 * nk; r += 256 / LANES) {
        const int c = threadIdx.x % LANES * V;
        const bool is_q = r < nq, is_v = r >= nq + nk;
        const int h = is_q ? r : is_v ? r - nq - nk : r - nq;
        const T* src = (const T*)(is_q ? p.q : is_v ? p.v : p.k) +
                       kv_row(a, is_q ? a.qs : is_v ? a.vs : a.ks, b, sq.row0, i, h);
        float x[V];
        double y[V];
        load16(src + c, x);
        for (int e = 0; e < V; ++e) y[e] = x[e];
        if (!is_v && c < a.rot) {
            float z[V];
            const int half = a.rot / 2, other = a.interleaved ? c : c < half ? c + half : c - half;
            load16(src + other, z);
            for (int e = 0; e < V; ++e) {
                const int f = a.interleaved ? (c + e) / 2 : (c < half ? c : c - half) + e;
                const bool first = a.interleaved ? !(e & 1) : c < half;
                const double mate = a.interleaved ? x[e ^ 1] : z[e];
                y[e] = first ? x[e] * s_cos[f] - mate * s_sin[f] : x[e] * s_cos[f] + mate * s_sin[f];
            }
        }
        float w[V];
        for (int e = 0; e < V; ++e) w[e] = (float)y[e];
        if (is_q) store16((T*)p.q_out + kv_row(a, a.os, b, sq.row0, i, h) + c, w);
        if (is_q) continue;
        if (!is_v && p.k_out) store16((T*)p.k_out + kv_row(a, a.kos, b, sq.row0, i, h) + c, w);
        const long long* cs = is_v ? a.vcs : a.kcs;
        char* pool = is_v ? a.vc : a.kc;
        if constexpr (!FP4) {
            if (page >= 0) store16((T*)pool + page * cs[0] + h * cs[1] + in * cs[2] + c, w);
        } else {
            uint64_t top = 0;
            for (int e = 0; e < V; ++e) {
                const uint64_t m = (uint64_t)__double_as_longlong(y[e]) & 0x7fffffffffffffffull;
                top = m > top ? m : top;
            }
            for (int s = 1; s < kFp4Group / V; s *= 2) {
                const uint64_t o = __shfl_xor((unsigned long long)top, s);
                top = o > top ? o : top;
            }
            const int byte = fp4_scale_byte(top);
            const double inv = fp4_inverse_scale(byte == 255 ? 127 : byte);
            unsigned codes = 0;
            for (int e = 0; e < V; ++e) codes |= fp4_code(y[e] * inv) << (4 * e);
            if (page >= 0) {
                *(unsigned*)(pool + page * cs[0] + h * cs[1] + in * cs[2] + c / 2) = codes;
                const long long* ss = is_v ? a.vss : a.kss;
                if (c % kFp4Group == 0)
                    (is_v ? a.vsc : a.ksc)[page * ss[0] + h * ss[1] + c / kFp4Group * ss[2] + in] = (unsigned char)byte;
            }
        }
    }
}

// One work-group a token: the cached rows of its heads.
template <class T, bool FP4, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a, T* k_out, T* v_out) {
    constexpr int V = Vec<T>::n, LANES = D / V;
    const long long row = blockIdx.x;
    const int b = seq_of_row(a, row);
    if (b >= a.B) return;
    const KvSeq sq = kv_seq(a, b);
    const int i = (int)(row - sq.row0);
    if (i < 0 || i >= sq.n) return;
    const long long j = (long long)a.kv_len[b] - sq.n + i;
    const int page = kv_page(a, b, j), in = (int)j & ((1 << a.page_shift) - 1);
    for (int r = threadIdx.x / LANES; r < 2 * a.Hkv; r += 256 / LANES) {
        const int c = threadIdx.x % LANES * V, h = r >> 1;
        const bool is_v = r & 1;
        T* out = is_v ? v_out : k_out;
        if (!out) continue;
        const long long* cs = is_v ? a.vcs : a.kcs;
        const char* pool = is_v ? a.vc : a.kc;
        float x[V] = {};
        if (page >= 0) {
            if constexpr (!FP4) {
                load16((const T*)pool + page * cs[0] + h * cs[1] + in * cs[2] + c, x);
            } else {
                const unsigned codes = *(const unsigned*)(pool + page * cs[0] + h * cs[1] + in * cs[2] + c / 2);
                const long long* ss = is_v ? a.vss : a.kss;
                const int byte = (is_v ? a.vsc : a.ksc)[page * ss[0] + h * ss[1] + c / kFp4Group * ss[2] + in];
                for (int e = 0; e < V; ++e) x[e] = fp4_value(codes >> (4 * e) & 15, byte);
            }
        }
        store16(out + kv_row(a, is_v ? a.vs : a.ks, b, sq.row0, i, h) + c, x);
    }
}

template <class T, bool FP4, int D>
int run_append(const AppendArgs& p, hipStream_t st) {
    return (int)launch_kernel(kv_append_kernel<T, FP4, D>, dim3((unsigned)p.a.total), dim3(256), 0, st, p);
}
template <class T, bool FP4, int D>
int run_read(const KvArgs& a, void* k, void* v, hipStream_t st) {
    return (int)launch_kernel(kv_read_kernel<T, FP4, D>, dim3((unsigned)a.total), dim3(256), 0, st, a, (T*)k, (T*)v);
}

}  // namespace

int launch_kv_append(const KvArgs& a, int dtype, int format, int d, const void* q, const void* k, const void* v,
                     const float* inv_freq, const int* positions, void* q_out, void* k_out, hipStream_t st) {
    const AppendArgs p = {a, q, k, v, inv_freq, positions, q_out, k_out};
    if (dtype == 0) return d == 32 ? run_append<float, false, 32>(p, st) : d == 64 ? run_append<float, false, 64>(p, st)
                         : d == 128 ? run_append<float, false, 128>(p, st) : -1;
    if (format) return d == 64 ? run_append<__bf16, true, 64>(p, st) : d == 128 ? run_append<__bf16, true, 128>(p, st) : -1;
    return d == 64 ? run_append<__bf16, false, 64>(p, st) : d == 128 ? run_append<__bf16, false, 128>(p, st) : -1;
}

int launch_kv_read(const KvArgs& a, int dtype, int format, int d, void* k, void* v, hipStream_t st) {
    if (dtype == 0) return d == 32 ? run_read<float, false, 32>(a, k, v, st) : d == 64 ? run_read<float, false, 64>(a, k, v, st)
                         : d == 128 ? run_read<float, false, 128>(a, k, v, st) : -1;
    if (format) return d == 64 ? run_read<__bf16, true, 64>(a, k, v, st) : d == 128 ? run_read<__bf16, true, 128>(a, k, v, st) : -1;
    return d == 64 ? run_read<__bf16, false, 64>(a, k, v, st) : d == 128 ? run_read<__bf16, false, 128>(a, k, v, st) : -1;
}

}  // namespace aa
