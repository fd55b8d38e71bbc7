// kv_append and kv_read: rows of new tokens into the pages of the cache (rotated on the way) and out of them.
//
//   y1 = x1 cos t - x2 sin t,  y2 = x2 cos t + x1 sin t,  t = position * inv_freq[pair]
//
// Memory traffic is all that they cannot do without: every row is read once and written once or twice, at some six operations an
// element.  A work-group takes a token, or four (see run_pairs): a wave for each works out where it lies and the cosines and sines of its
// position, one angle a lane, for all heads; then the threads take 16 bytes of a row each, a pair's other half being read a
// second time from the L1, and the rows of a token that one thread meets are in flight together.
// 51393 tokens of 32 / 8 heads, d = 128, bf16: 1.37 GB in 260 us, 5.3 TB/s (a copy of 4 GB: 4.7).  16384 tokens into 4 bits: 0.39 GB in
// 97 us, 4.0 TB/s, the 64-bit turning of the keys standing beside the traffic; kv_read of them 85 MB in 21 us, 4.0 TB/s.  One token: 3.3 us,
// which is a launch and four dependent reads (length, page, then the row).
#include <type_traits>

#include "aa_kv.h"
#include "aa_kv_turn.h"

namespace aa {
namespace {

using u32x4 = __attribute__((ext_vector_type(4))) unsigned;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;

template <class T> constexpr int kVec = 16 / (int)sizeof(T);       // elements of 16 bytes

template <class T> __device__ __forceinline__ void unpack(u32x4 u, float* x) {
    union { u32x4 u; T t[kVec<T>]; } v;
    v.u = u;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) x[i] = (float)v.t[i];
}
template <class T> __device__ __forceinline__ u32x4 pack(const float* x) {
    union { u32x4 u; T t[kVec<T>]; } v;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v.t[i] = (T)x[i];
    return v.u;
}

// Cosine and sine of the angle t.  The angle and what is left of it after whole quarter turns are 64-bit numbers (a position of a million
// leaves 32 bits four digits); 32 bits are enough from there on for results in 32 bits.
template <class S> __device__ __forceinline__ void cos_sin(double t, S* c, S* s) {
    const double turns = rint(t * 0.63661977236758134308);
    double r = fma(-turns, 1.57079632679489661923, t);
    r = fma(-turns, 6.12323399573676603587e-17, r);                // pi / 2 = 1.57..923 + 6.12..e-17
    S a, b;
    series((S)r, &a, &b);
    const int quarter = (int)(turns - 4. * floor(turns * 0.25));
    const S x = quarter & 1 ? b : a, y = quarter & 1 ? a : b;
    *c = quarter == 1 || quarter == 2 ? -x : x;
    *s = quarter >= 2 ? -y : y;
}

// y as a float that is on y's side of every number of a few bits: towards zero, with the last bit set if that lost anything.
__device__ __forceinline__ float to_odd(double y) {
    const float f = (float)y;
    const double back = (double)f;
    unsigned u = __float_as_uint(f);
    if (back != y) u = (fabs(back) > fabs(y) ? u - 1 : u) | 1u;    // NaN: u | 1, a NaN still
    return __uint_as_float(u);
}

// Eight channels of one lane as 4-bit codes, and the scale byte of the 32 that four neighbouring lanes hold.
__device__ __forceinline__ unsigned to_fp4(const float* x, int* byte) {
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned m = __float_as_uint(x[e]) & 0x7fffffffu;
        top = m > top ? m : top;
    }
#pragma unroll
    for (int s = 1; s < kFp4Group / 8; s *= 2) {
        const unsigned o = __shfl_xor(top, s);
        top = o > top ? o : top;
    }
    *byte = fp4_scale_byte(top);
    const float scale = __uint_as_float((unsigned)(*byte == 255 ? 127 : *byte) << 23);
    unsigned codes = 0;                                             // the instruction rounds to even and cuts to 6
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    return *byte == 255 ? 0u : codes;
}

// A new token: its sequence, its number there, its place in the cache.
struct Token { int b, i, page, in; long long row0, j; };
__device__ __forceinline__ Token token_of(const KvArgs& a, long long row) {
    Token t;
    t.b = 0;
    if (!a.cu) {
        t.b = (int)(row / a.N);
    } else {
        // sequences that end at or before the row: 64 of them looked at at once, then those between two of them (1024 sequences of a token
        // 8.3 us, and 12.2 with all of them looked at)
        for (int step = a.B; step > 1;) {
            const int end = t.b + step < a.B ? t.b + step : a.B;
            step = (step + 63) / 64;
            const int i = t.b + ((int)(threadIdx.x & 63) + 1) * step;
            t.b += step * __popcll(__ballot(i <= end && a.cu[i] <= row));
        }
    }
    t.i = -1;
    if (t.b >= a.B) return t;
    const KvSeq sq = kv_seq(a, t.b);
    if (row < sq.row0 || row - sq.row0 >= sq.n) return t;
    t.i = (int)(row - sq.row0);
    t.row0 = sq.row0;
    t.j = (long long)a.kv_len[t.b] - sq.n + t.i;
    t.page = kv_page(a, t.b, t.j);
    t.in = (int)t.j & ((1 << a.page_shift) - 1);
    return t;
}

struct AppendArgs {
    KvArgs a;
    const void *q, *k, *v;
    const float* inv_freq;
    const int* positions;
    void *q_out, *k_out;
};

enum { kNoPairs, kHalves, kNeighbours };        // which channels are turned together

__device__ __forceinline__ long long uniform(long long x) {
    return (long long)(unsigned)__builtin_amdgcn_readfirstlane((int)x) |
           (long long)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// TOKENS: of a work-group; PASSES rows of a token are on their way in a thread at once.
// (4 bits, three passes: four waves a SIMD with a few registers in scratch memory, 16000 tokens of 48 rows 115 us; three without, 118.)
template <class T, bool FP4, int D, int PAIRS, int TOKENS, int PASSES>
__global__ __launch_bounds__(256, (FP4 && PASSES == 3 ? 4 : 1)) void kv_append_kernel(AppendArgs p) {
    constexpr int V = kVec<T>, LANES = D / V, ROWS = 256 / LANES, item = sizeof(T);
    using S = typename std::conditional<FP4, double, float>::type;
    __shared__ S s_cs[TOKENS][D / 2][2];
    __shared__ float s_csf[FP4 ? TOKENS : 1][D / 2][2];              // 4 bits: the queries' own, rounded once
    __shared__ Token s_tok[TOKENS];
    const KvArgs& a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row_first = (long long)blockIdx.x * TOKENS;
    if (wave < TOKENS) {
        Token t;
        t.i = -1;
        if (row_first + wave < a.total) t = token_of(a, row_first + wave);
        if (lane == 0) s_tok[wave] = t;
        if (PAIRS != kNoPairs && t.i >= 0 && lane < a.rot / 2) {
            const double pos = p.positions ? (double)p.positions[row_first + wave] : (double)t.j;
            S c, s;
            cos_sin<S>(pos * (double)p.inv_freq[lane], &c, &s);
            s_cs[wave][lane][0] = c;
            s_cs[wave][lane][1] = s;
            if (FP4) {
                s_csf[wave][lane][0] = (float)c;
                s_csf[wave][lane][1] = (float)s;
            }
        }
    }
    __syncthreads();
    const int nq = p.q_out ? a.Hq : 0, nk = p.k ? a.Hkv : 0, rows = nq + 2 * nk;
    const int c = threadIdx.x % LANES * V, half = a.rot / 2;
    const bool turn = PAIRS != kNoPairs && c < a.rot, upper = PAIRS == kHalves && c >= half;
    const int other = !turn ? 0 : PAIRS == kHalves ? (upper ? -half : half) : 0;         // the pair's other chunk
    const int f0 = !turn ? 0 : PAIRS == kNeighbours ? c / 2 : upper ? c - half : c;
    for (int r0 = threadIdx.x / LANES + ROWS * PASSES * blockIdx.y; r0 < rows + threadIdx.x / LANES; r0 += ROWS * PASSES * gridDim.y) {
        // where a thread's rows lie from the token's on
        bool is_q[PASSES], is_v[PASSES];
        long long from[PASSES], to[PASSES], pool[PASSES];
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const int r = r0 + u * ROWS < rows ? r0 + u * ROWS : rows - 1;
            is_q[u] = r < nq;
            is_v[u] = r >= nq + nk;
            const int h = is_q[u] ? r : is_v[u] ? r - nq - nk : r - nq;
            from[u] = (long long)h * (is_q[u] ? a.qs[1] : is_v[u] ? a.vs[1] : a.ks[1]) + c;
            to[u] = (long long)h * (is_q[u] ? a.os[1] : a.kos[1]) + c;
            pool[u] = (long long)h * (is_v[u] ? a.vcs[1] : a.kcs[1]) + (FP4 ? c / 2 : c);
        }
#pragma unroll 1
        for (int tk = 0; tk < TOKENS; ++tk) {
            const int i = __builtin_amdgcn_readfirstlane(s_tok[tk].i), b = __builtin_amdgcn_readfirstlane(s_tok[tk].b);
            if (i < 0) continue;
            const long long row0 = uniform(s_tok[tk].row0);
            const T* q = (const T*)p.q + kv_row(a, a.qs, b, row0, i, 0);
            const T* k = (const T*)p.k + kv_row(a, a.ks, b, row0, i, 0);
            const T* v = (const T*)p.v + kv_row(a, a.vs, b, row0, i, 0);
            u32x4 x[PASSES], z[PASSES];
#pragma unroll
            for (int u = 0; u < PASSES; ++u) {
                const T* src = (is_q[u] ? q : is_v[u] ? v : k) + from[u];
                x[u] = *(const u32x4*)src;
                if (PAIRS == kHalves) z[u] = *(const u32x4*)(src + other);
            }
            {                                                // (the token once more: kept, it takes registers of the rows in flight)
                const int i = __builtin_amdgcn_readfirstlane(s_tok[tk].i), b = __builtin_amdgcn_readfirstlane(s_tok[tk].b);
                const int page = __builtin_amdgcn_readfirstlane(s_tok[tk].page), in = __builtin_amdgcn_readfirstlane(s_tok[tk].in);
                const long long row0 = uniform(s_tok[tk].row0);
                float cs[V], sn[V];
                if (PAIRS != kNoPairs) {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int g = f0 + (PAIRS == kNeighbours ? e / 2 : e);
                        if constexpr (FP4) { cs[e] = s_csf[tk][g][0]; sn[e] = s_csf[tk][g][1]; }
                        else { cs[e] = s_cs[tk][g][0]; sn[e] = s_cs[tk][g][1]; }
                        if (PAIRS == kNeighbours ? !(e & 1) : !upper) sn[e] = -sn[e];
                    }
                }
                T* qo = (T*)p.q_out + kv_row(a, a.os, b, row0, i, 0);
                T* ko = (T*)p.k_out + kv_row(a, a.kos, b, row0, i, 0);
                char* kc = a.kc + (page * a.kcs[0] + in * a.kcs[2]) * (FP4 ? 1 : item);
                char* vc = a.vc + (page * a.vcs[0] + in * a.vcs[2]) * (FP4 ? 1 : item);
#pragma unroll
                for (int u = 0; u < PASSES; ++u) {
                    float y[V], m[V];
                    unpack<T>(x[u], y);
                    if (PAIRS == kHalves) {
                        unpack<T>(z[u], m);
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) m[e] = y[e ^ 1];
                    }
                    const bool turned = turn && !is_v[u];
                    u32x4 w = x[u];
                    float t[V];
                    if (PAIRS != kNoPairs) {
#pragma unroll
                        for (int e = 0; e < V; ++e) t[e] = fmaf(m[e], sn[e], y[e] * cs[e]);
                        const u32x4 r = pack<T>(t);
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = turned ? r[e] : w[e];
                    }
                    if (r0 + u * ROWS >= rows) continue;
                    if (is_q[u]) {
                        *(u32x4*)(qo + to[u]) = w;
                        continue;
                    }
                    if (p.k_out && !is_v[u]) *(u32x4*)(ko + to[u]) = w;
                    if (page < 0) continue;
                    if constexpr (!FP4) {
                        *(u32x4*)((is_v[u] ? vc : kc) + pool[u] * item) = w;
                    } else {
                        // codes are taken from the 64-bit values: of two neighbours in 32 bits one may be on another code's side
                        if (turned) {
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                const int g = f0 + (PAIRS == kNeighbours ? e / 2 : e);
                                const double s64 = (PAIRS == kNeighbours ? !(e & 1) : !upper) ? -s_cs[tk][g][1] : s_cs[tk][g][1];
                                y[e] = to_odd(fma((double)m[e], s64, y[e] * (double)s_cs[tk][g][0]));
                            }
                        }
                        int byte;
                        *(unsigned*)((is_v[u] ? vc : kc) + pool[u]) = to_fp4(y, &byte);
                        if (c % kFp4Group) continue;
                        const int h = r0 + u * ROWS - nq - (is_v[u] ? nk : 0);
                        unsigned char* sc = is_v[u] ? a.vsc + page * a.vss[0] + h * a.vss[1] + c / kFp4Group * a.vss[2]
                                                    : a.ksc + page * a.kss[0] + h * a.kss[1] + c / kFp4Group * a.kss[2];
                        sc[in] = (unsigned char)byte;
                    }
                }
            }
        }
    }
}

template <class T, bool FP4, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a, T* k_out, T* v_out) {
    constexpr int V = kVec<T>, LANES = D / V, ROWS = 256 / LANES, TOKENS = 4, item = sizeof(T);
    __shared__ Token s_tok[TOKENS];
    const int wave = threadIdx.x >> 6;
    const long long row = (long long)blockIdx.x * TOKENS + wave;
    Token mine;
    mine.i = -1;
    if (row < a.total) mine = token_of(a, row);
    if ((threadIdx.x & 63) == 0) s_tok[wave] = mine;
    __syncthreads();
    const int c = threadIdx.x % LANES * V, nk = k_out ? a.Hkv : 0, rows = nk + (v_out ? a.Hkv : 0);
    for (int r = threadIdx.x / LANES; r < rows; r += ROWS) {
        const bool is_v = r >= nk;
        const int h = is_v ? r - nk : r;
        const long long pool = (long long)h * (is_v ? a.vcs[1] : a.kcs[1]) + (FP4 ? c / 2 : c);
        const long long to = (long long)h * (is_v ? a.vs[1] : a.ks[1]) + c;
        const long long scale_at = FP4 ? (long long)h * (is_v ? a.vss[1] : a.kss[1]) + c / kFp4Group * (is_v ? a.vss[2] : a.kss[2]) : 0;
        u32x4 x[TOKENS];
        unsigned byte[TOKENS];
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) {
            const int page = __builtin_amdgcn_readfirstlane(s_tok[t].page), in = __builtin_amdgcn_readfirstlane(s_tok[t].in);
            x[t] = u32x4{0, 0, 0, 0};
            byte[t] = 127;
            if (__builtin_amdgcn_readfirstlane(s_tok[t].i) < 0 || page < 0) continue;
            const char* kc = a.kc + (page * a.kcs[0] + in * a.kcs[2]) * (FP4 ? 1 : item);
            const char* vc = a.vc + (page * a.vcs[0] + in * a.vcs[2]) * (FP4 ? 1 : item);
            if constexpr (FP4) {
                x[t][0] = *(const unsigned*)((is_v ? vc : kc) + pool);
                byte[t] = ((is_v ? a.vsc + page * a.vss[0] : a.ksc + page * a.kss[0]) + in)[scale_at];
            } else {
                x[t] = *(const u32x4*)((is_v ? vc : kc) + pool * item);
            }
        }
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) {
            const int i = __builtin_amdgcn_readfirstlane(s_tok[t].i), b = __builtin_amdgcn_readfirstlane(s_tok[t].b);
            if (i < 0) continue;
            const long long row0 = uniform(s_tok[t].row0);
            u32x4 w = x[t];
            if constexpr (FP4) {
                union { u32x4 u; bf16x2 b[4]; } v;
                const float scale = __uint_as_float(byte[t] << 23);
                v.b[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x[t][0], scale, 0);
                v.b[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x[t][0], scale, 1);
                v.b[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x[t][0], scale, 2);
                v.b[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x[t][0], scale, 3);
                w = v.u;
            }
            T* k = k_out + kv_row(a, a.ks, b, row0, i, 0);
            T* v = v_out + kv_row(a, a.vs, b, row0, i, 0);
            *(u32x4*)((is_v ? v : k) + to) = w;
        }
    }
}

template <class T, bool FP4, int D, int PAIRS>
int run_pairs(const AppendArgs& p, hipStream_t st) {
    constexpr int ROWS = 256 / (D / kVec<T>);                      // rows of a token that a work-group takes at once
    const int rows = (p.q_out ? p.a.Hq : 0) + (p.k ? 2 * p.a.Hkv : 0);
    // A work-group a token, or four of them: what is worked out once a work-group is shared by more, but a token waits for the one before.
    // A token / four, us, d = 128, tokens 300, 2000, 8000, 51000, the same rows again and again: plain pages, 48 rows (32 / 8 heads) 4.6 / 7.9,
    // 10.7 / 11.9, 31.7 / 32.6, 217 / 229; 24 rows (8 / 8) 4.0 / 6.8, 8.5 / 9.4, 22.3 / 20.4, 152 / 133; 8 rows (4 / 2) 3.7 / 5.6, 7.2 / 7.0,
    // 20.1 / 14.3, 106 / 61; 4 bits, where the angles take 64 bits to the end, 48 rows 6.7 / 11.0, 16.0 / 15.5, 47.7 / 37.4, 307 / 251; 8 rows
    // 5.7 / 8.1, 11.3 / 9.2, 35.7 / 19.0, 204 / 87.
    if (p.a.total < (FP4 || rows <= ROWS ? 2000 : 4000) || (!FP4 && rows > 2 * ROWS)) {
        const int passes = (rows + 3 * ROWS - 1) / (3 * ROWS);
        return (int)launch_kernel(kv_append_kernel<T, FP4, D, PAIRS, 1, 3>, dim3((unsigned)p.a.total, passes < 64 ? passes : 64), dim3(256), 0, st, p);
    }
    const dim3 grid((unsigned)((p.a.total + 3) / 4));
    if (rows <= ROWS) return (int)launch_kernel(kv_append_kernel<T, FP4, D, PAIRS, 4, 1>, grid, dim3(256), 0, st, p);
    return (int)launch_kernel(kv_append_kernel<T, FP4, D, PAIRS, 4, 3>, grid, dim3(256), 0, st, p);
}
template <class T, bool FP4, int D>
int run_append(const AppendArgs& p, hipStream_t st) {
    return !p.a.rot ? run_pairs<T, FP4, D, kNoPairs>(p, st) : p.a.interleaved ? run_pairs<T, FP4, D, kNeighbours>(p, st)
                                                            : run_pairs<T, FP4, D, kHalves>(p, st);
}
template <class T, bool FP4, int D>
int run_read(const KvArgs& a, void* k, void* v, hipStream_t st) {
    return (int)launch_kernel(kv_read_kernel<T, FP4, D>, dim3((unsigned)((a.total + 3) / 4)), dim3(256), 0, st, a, (T*)k, (T*)v);
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
