// kv_attn: attention of new queries over the pages of the cache.
//
//   o_r = sum_j exp(s_rj - m_r) v_j / sum_j exp(s_rj - m_r),   s_rj = sigma <q_r, k_j>
//
// One pass over the keys with a running reference m and sum (online softmax), on the matrix cores.  The rows of a KV head's query
// heads and new tokens stand side by side (row r = token * grp + head): every key is read once for all of them.
//
// A wave takes 16 NT rows and a share of the keys and works alone until the end: no LDS and no barrier in the loop, K and V come from
// the pages straight into the registers that the matrix instruction reads.
//   S^T = K Q^T  (16x16: keys x rows).  A lane holds key lane % 16 of K, and 8 channels of each step at lane / 16 (=: g): 16 bytes of
//                a row as it lies.  Which channel stands where in the sum does not matter as long as Q has the same order.
//   O^T = V^T P^T (channels x rows).  The result of the first product is the second's right operand where it is: lane (row, g) holds
//                keys 4g .. 4g+3 of each half of the tile, and the sum over keys may run in that order too.  The left operand wants 8 keys of
//                one channel in a lane; a lane loads D/16 channels of each of its keys and two byte permutations turn four bf16 values.
// A lane's rows of S^T, O^T, m and the sum are all row lane % 16, so nothing crosses lanes unless a reference is raised.
#include "aa_kv_attn.h"

namespace aa {
namespace {

using u32x2 = __attribute__((ext_vector_type(2))) unsigned;
using u32x4 = __attribute__((ext_vector_type(4))) unsigned;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;

constexpr int kWaves = 4;
constexpr float kSlack = 8.f;       // a reference is raised when a score exceeds it by 2^8: weights stay below 256 in 32-bit sums

enum { kRows32, kRows16, kRows4 };  // cached rows: float, bf16, 4 bits

template <int F> struct RowType { using type = __bf16; };
template <> struct RowType<kRows32> { using type = float; };

// One tile of keys in registers: TT halves of 16 keys.
template <int F, int D> struct Tile;
template <int D> struct Tile<kRows16, D> {
    static constexpr int TT = 2;
    u32x4 k[TT][D / 32];
    unsigned v[TT][4][D / 32];
    int key;
    bool there[TT];
};
template <int D> struct Tile<kRows4, D> {
    static constexpr int TT = 2;
    unsigned k[TT][D / 32];
    unsigned v[TT][4];
    unsigned ks[TT], vs[TT];
    int key;
    bool there[TT];
};
template <int D> struct Tile<kRows32, D> {
    static constexpr int TT = 1;
    f32x4 k[TT][D / 16];
    float v[TT][4][D / 16];
    int key;
    bool there[TT];
};

template <int N> __device__ __forceinline__ void load_words(const char* p, unsigned* x) {
    static_assert(N == 1 || N == 2 || N % 4 == 0, "");
    if constexpr (N == 1) {
        x[0] = *(const unsigned*)p;
    } else if constexpr (N == 2) {
        const u32x2 u = *(const u32x2*)p;
        x[0] = u[0]; x[1] = u[1];
    } else {
        for (int i = 0; i < N; i += 4) {
            const u32x4 u = *(const u32x4*)(p + 4 * i);
            x[i] = u[0]; x[i + 1] = u[1]; x[i + 2] = u[2]; x[i + 3] = u[3];
        }
    }
}

// What a wave needs to find a tile: the pools from its head on, and a lane's place in 16 keys.
struct Where {
    const int* table;
    long long room;
    const char *k, *v;
    const unsigned char *ks, *vs;
    unsigned k_lane, v_lane, ks_lane, vs_lane;
    long long v_row;                 // bytes between rows of values
};

template <int F, int D>
__device__ __forceinline__ void load_tile(const KvArgs& a, const Where& w, int key, Tile<F, D>& t) {
    t.key = key;
    constexpr int item = F == kRows32 ? 4 : 2;
#pragma unroll
    for (int h = 0; h < Tile<F, D>::TT; ++h) {
        const int j = key + 16 * h;
        int page = -1;
        if (j < w.room) page = w.table[j >> a.page_shift];
        t.there[h] = (unsigned)page < (unsigned)a.n_pages;
        const long long pg = t.there[h] ? page : 0;         // some storage that exists; its keys are masked
        const int in = j & ((1 << a.page_shift) - 1);
        if constexpr (F == kRows4) {
            const char* k = w.k + pg * a.kcs[0] + in * a.kcs[2];
            const char* v = w.v + pg * a.vcs[0] + in * a.vcs[2];
            load_words<D / 32>(k + w.k_lane, t.k[h]);
            t.ks[h] = w.ks[pg * a.kss[0] + in + w.ks_lane];
            t.vs[h] = *(const unsigned*)(w.vs + pg * a.vss[0] + in + w.vs_lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const char* x = v + (w.v_lane + i * (unsigned)w.v_row);
                if constexpr (D == 128) t.v[h][i] = *(const unsigned*)x;
                else t.v[h][i] = *(const unsigned short*)x;
            }
        } else {
            const char* k = w.k + (pg * a.kcs[0] + in * a.kcs[2]) * item;
            const char* v = w.v + (pg * a.vcs[0] + in * a.vcs[2]) * item;
            constexpr int steps = D * item / 64;
#pragma unroll
            for (int s = 0; s < steps; ++s) {
                if constexpr (F == kRows32) t.k[h][s] = *(const f32x4*)(k + 64 * s + w.k_lane);
                else t.k[h][s] = *(const u32x4*)(k + 64 * s + w.k_lane);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words<D * item / 64>(v + (w.v_lane + i * (unsigned)w.v_row), (unsigned*)t.v[h][i]);
        }
    }
}

__device__ __forceinline__ unsigned fp4_pair(unsigned codes, float scale, int byte) {
    union { bf16x2 b; unsigned u; } r;
    switch (byte) {
        case 0: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0); break;
        case 1: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1); break;
        case 2: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2); break;
        default: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3); break;
    }
    return r.u;
}

// State of a wave's rows: NT tiles of 16.
template <int F, int D, int NT> struct Rows {
    static constexpr int Q = F == kRows32 ? D / 16 : D / 32;
    u32x4 q[NT][Q];
    f32x4 o[NT][D / 16];
    float m[NT], l[NT];              // l: this lane's keys alone
    int see[NT];                     // keys that the lane's row sees
};

template <int F, int D, int NT>
__device__ __forceinline__ void attend_tile(const AttnArgs& p, Tile<F, D>& t, int hi, int see_all, Rows<F, D, NT>& r) {
    constexpr int TT = Tile<F, D>::TT;
    const int g = (threadIdx.x & 63) >> 4;
    bool whole = t.key + 16 * TT <= hi;
#pragma unroll
    for (int h = 0; h < TT; ++h) whole = whole && t.there[h];
    if (!whole) {                    // rows of values that no row of the tile sees may hold anything: they become zeros
#pragma unroll
        for (int h = 0; h < TT; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool keep = t.there[h] && t.key + 16 * h + 4 * g + i < hi;
                if constexpr (F == kRows4) {
                    t.v[h][i] = keep ? t.v[h][i] : 0u;
                    if (!keep) t.vs[h] = (t.vs[h] & ~(255u << (8 * i))) | (127u << (8 * i));
                } else {
#pragma unroll
                    for (int e = 0; e < (F == kRows32 ? D / 16 : D / 32); ++e) t.v[h][i][e] = keep ? t.v[h][i][e] : 0;
                }
            }
    }
    // scores
    f32x4 s[NT][TT];
    if constexpr (F == kRows32) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            s[n][0] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                union { u32x4 u; f32x4 f; } q;
                q.u = r.q[n][c];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[0][c][e], q.f[e], s[n][0], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int h = 0; h < TT; ++h) {
            float scale = 0;
            if constexpr (F == kRows4) scale = __uint_as_float(t.ks[h] << 23);
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][h] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                union { u32x4 u; bf16x8 b; } k, q;
                if constexpr (F == kRows4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) k.u[e] = fp4_pair(t.k[h][c], scale, e);
                } else {
                    k.u = t.k[h][c];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    q.u = r.q[n][c];
                    s[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.b, q.b, s[n][h], 0, 0, 0);
                }
            }
        }
    }
    // weights
    const bool all = whole && t.key + 16 * TT <= see_all;
    union { bf16x8 b; __bf16 e[8]; } pb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int h = 0; h < TT; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][h][i] *= p.c;
                if (!all) s[n][h][i] = t.there[h] && t.key + 16 * h + 4 * g + i < r.see[n] ? s[n][h][i] : -INFINITY;
            }
        float top = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3]));
        if constexpr (TT == 2) top = fmaxf(top, fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3])));
        if (__any(top > r.m[n] + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m = fmaxf(top, r.m[n]);
            const float down = m == -INFINITY ? 1.f : exp2f(r.m[n] - m);
            r.m[n] = m;
            r.l[n] *= down;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) r.o[n][j] *= down;
        }
        const float ref = r.m[n] == -INFINITY ? 0.f : r.m[n];
#pragma unroll
        for (int h = 0; h < TT; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][h][i] = __builtin_amdgcn_exp2f(s[n][h][i] - ref);
                r.l[n] += s[n][h][i];
                if constexpr (F != kRows32) pb[n].e[4 * h + i] = (__bf16)s[n][h][i];
            }
    }
    // values
    if constexpr (F == kRows32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    r.o[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.v[0][i][j], s[n][0][i], r.o[n][j], 0, 0, 0);
    } else {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {              // two channels at a time
            unsigned x[TT][4];
#pragma unroll
            for (int h = 0; h < TT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (F == kRows4) x[h][i] = fp4_pair(t.v[h][i], __uint_as_float(((t.vs[h] >> (8 * i)) & 255u) << 23), c);
                    else x[h][i] = t.v[h][i][c];
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                union { u32x4 u; bf16x8 b; } v;
#pragma unroll
                for (int h = 0; h < TT; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        v.u[2 * h + i] = __builtin_amdgcn_perm(x[h][2 * i + 1], x[h][2 * i], e ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    r.o[n][2 * c + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.b, pb[n].b, r.o[n][2 * c + e], 0, 0, 0);
            }
        }
    }
}

template <int F, int D, int NT>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void kv_attn_kernel(AttnArgs p) {
    using T = typename RowType<F>::type;
    constexpr int item = sizeof(T), TT = Tile<F, D>::TT, TK = 16 * TT, R = 16 * NT, P = D + 4;
    __shared__ float s_o[kWaves][16][P];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const KvArgs& a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    AttnPart wp;
    if (!attn_part<R>(p, wp)) return;
    const int b = wp.b, hk = wp.hk, r0 = wp.r0, rows = wp.rows, lo = wp.lo, hi = wp.hi;
    const KvSeq sq = wp.sq;

    Rows<F, D, NT> r;
    const int n16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = r0 + 16 * n + n16 < rows ? r0 + 16 * n + n16 : rows - 1;
        const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
        r.see[n] = seen(a, wp.len, sq.n, i);
        r.m[n] = -INFINITY;
        r.l[n] = 0.f;
        const char* q = (const char*)p.q + kv_row(a, a.qs, b, sq.row0, i, h) * item;
#pragma unroll
        for (int c = 0; c < Rows<F, D, NT>::Q; ++c)
            r.q[n][c] = *(const u32x4*)(q + (F == kRows4 ? (D / 2) * g + 16 * c : 64 * c + 16 * g));
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.o[n][j] = f32x4{0, 0, 0, 0};
    }

    Where w;
    w.table = a.table + b * a.table_stride;
    w.room = (long long)a.max_pages << a.page_shift;
    if constexpr (F == kRows4) {
        w.k = a.kc + hk * a.kcs[1]; w.v = a.vc + hk * a.vcs[1];
        w.ks = a.ksc + hk * a.kss[1]; w.vs = a.vsc + hk * a.vss[1];
        w.k_lane = n16 * (unsigned)a.kcs[2] + g * (D / 8);
        w.v_lane = 4 * g * (unsigned)a.vcs[2] + n16 * (D / 32);
        w.ks_lane = n16 + (unsigned)(g * (D / 4) / kFp4Group) * (unsigned)a.kss[2];
        w.vs_lane = 4 * g + (unsigned)(n16 * (D / 16) / kFp4Group) * (unsigned)a.vss[2];
        w.v_row = a.vcs[2];
    } else {
        w.k = a.kc + hk * a.kcs[1] * item; w.v = a.vc + hk * a.vcs[1] * item;
        w.k_lane = n16 * (unsigned)(a.kcs[2] * item) + 16 * g;
        w.v_lane = 4 * g * (unsigned)(a.vcs[2] * item) + n16 * (D / 16 * item);
        w.v_row = a.vcs[2] * item;
    }

    // tiles of the chunk go to the waves in turn; two in registers, one loading while the other is attended
    int key = lo + wave * TK;
    if (key < hi) {
        Tile<F, D> t0, t1;
        load_tile<F, D>(a, w, key, t0);
        for (;;) {
            const int k1 = key + kWaves * TK;
            load_tile<F, D>(a, w, k1 < hi ? k1 : key, t1);
            attend_tile<F, D, NT>(p, t0, hi, wp.see_first, r);
            if (k1 >= hi) break;
            key = k1 + kWaves * TK;
            load_tile<F, D>(a, w, key < hi ? key : k1, t0);
            attend_tile<F, D, NT>(p, t1, hi, wp.see_first, r);
            if (key >= hi) break;
        }
    }

    // the waves' rows together, 16 at a time
    const int x = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * (D / 16);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float l = r.l[n];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (n) __syncthreads();
        if (g == 0) { s_m[wave][n16] = r.m[n]; s_l[wave][n16] = l; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) s_o[wave][n16][(D / 16) * (4 * g + i) + j] = r.o[n][j][i];
        __syncthreads();
        const int row = r0 + 16 * n + x;
        if (row >= rows) continue;
        float m = -INFINITY, sum = 0.f, acc[D / 16] = {};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) m = fmaxf(m, s_m[k][x]);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float f = exp2f(s_m[k][x] - ref);
            sum += f * s_l[k][x];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc[j] += f * s_o[k][x][c0 + j];
        }
        const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
        if (p.splits > 1) {
            const long long at = share_of(p, wp, row);
            float* o = p.ws + at * D + c0;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] = acc[j];
            if (c0 == 0) {
                float* ml = share_sums(p, D) + at * 2;
                ml[0] = m; ml[1] = sum;
            }
        } else {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T* o = (T*)p.out + kv_row(a, a.os, b, sq.row0, i, h) + c0;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] = (T)(acc[j] * inv);
            if (p.lse && c0 == 0)
                p.lse[lse_of(a, sq, b, h, i)] =
                    sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
        }
    }
}

// The shares of a row together: one work-group a row, a wave takes every fourth share.
template <class T, int D>
__global__ __launch_bounds__(256) void kv_join_kernel(AttnArgs p) {
    __shared__ float s_o[4][D];
    __shared__ float s_m[4], s_l[4];
    const KvArgs& a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.y;
    const unsigned row = p.by_hkv.div(blockIdx.x), hk = blockIdx.x - row * a.Hkv;
    const KvSeq sq = kv_seq(a, b);
    const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
    if (i >= sq.n) return;
    // a share wrote this row if its keys begin before those that the row's tile of rows sees end; before those of the row is enough
    const int see = seen(a, a.kv_len[b], sq.n, i);
    int parts = (see + p.chunk - 1) / p.chunk;
    parts = parts > p.splits ? p.splits : parts < 1 ? 1 : parts;
    const long long at = (((long long)b * a.Hkv + hk) * p.rows + row) * p.splits;
    const float* o = p.ws + at * D;
    const float* ml = share_sums(p, D) + at * 2;
    constexpr int E = (D + 63) / 64;
    float m = -INFINITY, l = 0.f, acc[E] = {};
    for (int s = wave; s < parts; s += 4) {
        const float ms = ml[2 * s], top = fmaxf(m, ms), ref = top == -INFINITY ? 0.f : top;
        const float down = exp2f(m - ref), up = exp2f(ms - ref);
        l = l * down + up * ml[2 * s + 1];
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (D >= 64 || lane < D) acc[e] = acc[e] * down + up * o[(long long)s * D + lane * E + e];
        m = top;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (D >= 64 || lane < D) s_o[wave][lane * E + e] = acc[e];
    if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= D) return;
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, x = 0.f;
    for (int k = 0; k < 4; ++k) {
        const float f = exp2f(s_m[k] - ref);
        sum += f * s_l[k];
        x += f * s_o[k][c];
    }
    ((T*)p.out)[kv_row(a, a.os, b, sq.row0, i, h) + c] = (T)(sum == 0.f ? 0.f : x / sum);
    if (p.lse && c == 0)
        p.lse[lse_of(a, sq, b, h, i)] = sum == 0.f ? -INFINITY : top * kLn2 + logf(sum);
}

// Rows of a work-group.  Beyond 64 rows with d = 128 and bf16 products: 128 through LDS.
int tile_rows(long long rows, int d, int dtype) {
    if (rows > 64 && d == 128 && dtype != 0) return kChunkRows;
    return rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
}

template <int F, int D>
int run(const AttnArgs& p, int R, hipStream_t st) {
    using T = typename RowType<F>::type;
    const long long x = (long long)p.a.Hkv * p.tiles * p.splits, rows = (long long)p.a.Hkv * p.rows;
    if (x > 0x7fffffffll || (p.splits > 1 && rows > 0x7fffffffll)) return -1;
    const dim3 grid((unsigned)x, p.a.B), block(64 * kWaves);
    int e;
    if (R == 16) e = (int)launch_kernel(kv_attn_kernel<F, D, 1>, grid, block, 0, st, p);
    else if (R == 32) e = (int)launch_kernel(kv_attn_kernel<F, D, 2>, grid, block, 0, st, p);
    else if (R == 64) e = (int)launch_kernel(kv_attn_kernel<F, D, 4>, grid, block, 0, st, p);
    else e = launch_kv_chunk(p, F == kRows4, grid, st);
    if (e != (int)hipSuccess || p.splits == 1) return e;
    return (int)launch_kernel(kv_join_kernel<T, D>, dim3((unsigned)rows, p.a.B), dim3(256), 0, st, p);
}

}  // namespace

KvSplit kv_split(int B, int Hq, int Hkv, int N, int d, int dtype, long long longest) {
    const long long rows = (long long)N * (Hq / Hkv), R = tile_rows(rows, d, dtype), tiles = (rows + R - 1) / R;
    const long long groups = tiles * B * Hkv;
    long long splits = (1024 + groups - 1) / groups;
    if (tiles == 1 && splits < (longest + 2047) / 2048) splits = (longest + 2047) / 2048;
    if (splits > (longest + 255) / 256) splits = (longest + 255) / 256;
    if (splits < 1) splits = 1;
    const long long chunk = ((longest + splits - 1) / splits + 127) / 128 * 128;
    splits = (longest + chunk - 1) / chunk;
    KvSplit s;
    s.splits = splits < 1 ? 1 : (int)splits;
    s.chunk = chunk < 128 ? 128 : chunk > (1 << 30) ? 1 << 30 : (int)chunk;
    s.ws_bytes = s.splits == 1 ? 0 : (size_t)B * Hkv * rows * s.splits * (d + 2) * 4;
    return s;
}

int launch_kv_attn(const KvArgs& a, int dtype, int format, int d, const KvSplit& sp, const void* q, void* out, float* lse, float* ws,
                   hipStream_t st) {
    AttnArgs p;
    p.a = a;
    p.q = q; p.out = out; p.lse = lse; p.ws = ws;
    p.splits = sp.splits; p.chunk = sp.chunk;
    p.rows = a.N * a.grp;
    const int R = tile_rows(p.rows, d, dtype);
    p.tiles = (p.rows + R - 1) / R;
    p.c = a.sigma * kLog2e;
    p.by_hkv.set(a.Hkv); p.by_splits.set(sp.splits); p.by_grp.set(a.grp);
    if (dtype == 0) return d == 32 ? run<kRows32, 32>(p, R, st) : d == 64 ? run<kRows32, 64>(p, R, st) : d == 128 ? run<kRows32, 128>(p, R, st) : -1;
    if (format) return d == 64 ? run<kRows4, 64>(p, R, st) : d == 128 ? run<kRows4, 128>(p, R, st) : -1;
    return d == 64 ? run<kRows16, 64>(p, R, st) : d == 128 ? run<kRows16, 128>(p, R, st) : -1;
}

}  // namespace aa
