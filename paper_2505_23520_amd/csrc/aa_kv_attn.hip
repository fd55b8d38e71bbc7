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
//
// Roundings to bf16: the weights (2^-8 each at most, as the matrix instruction takes them; their sum l is of the unrounded ones) and the
// result.  Codes of 4 bits are bf16 numbers exactly.  Float caches stay 32 bits throughout.
// Bound by memory for few rows: one token over 131072 keys of 8 heads, d = 128, bf16 537 MB in 92 us, 5.8 TB/s (a pure read of 4 GB by the
// library's sum: 4.0); 32 sequences of 200 .. 16000 in 134 us, 5.6; 64 sequences in 4 bits 552 MB in 109 us, 5.1, where the conversion of the
// codes takes a third of the vector unit's time beside it.  1000 keys: 6.4 us and the join 3, both latency.
#include "aa_kv_attn.h"

namespace aa {
namespace {

using u32x2 = __attribute__((ext_vector_type(2))) unsigned;
using u32x4 = __attribute__((ext_vector_type(4))) unsigned;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x2 = __attribute__((ext_vector_type(2))) float;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;

constexpr int kWaves = 4;

enum { kRows32, kRows16, kRows4 };  // cached rows: float, bf16, 4 bits

template <int F> struct RowType { using type = __bf16; };
template <> struct RowType<kRows32> { using type = float; };

// One tile of keys in registers: TT halves of 16 keys, of which the first rows[h] exist and are seen by some row.
template <int F, int D> struct Tile;
template <int D> struct Tile<kRows16, D> {
    static constexpr int TT = 2, words = D / 32;
    u32x4 k[TT][D / 32];
    unsigned v[TT][4][words];
    int key, rows[TT];
};
template <int D> struct Tile<kRows4, D> {
    static constexpr int TT = 2, words = 1;
    unsigned k[TT][D / 32];
    unsigned v[TT][4][words];
    unsigned ks[TT], vs[TT];
    int key, rows[TT];
};
template <int D> struct Tile<kRows32, D> {
    static constexpr int TT = 1, words = D / 16;
    u32x4 k[TT][D / 16];
    unsigned v[TT][4][words];
    int key, rows[TT];
};

// Waves of a SIMD that a kernel's registers allow, and so work-groups of a CU.
template <int F, int D, int NT> constexpr int kOccupancy = NT == 1 ? (D == 128 ? (F == kRows4 ? 3 : 2) : D == 64 ? 3 : 4) : NT == 2 && (D < 128 || F == kRows4) ? 2 : 1;

// What a wave needs to find a tile: its sequence's pages, the pools from its head on, and a lane's place in 16 keys (bytes).
struct Where {
    const_int* table;
    long long room;
    int shift, n_pages;
    const char *k, *v;
    const unsigned char *ks, *vs;
    long long k_page, v_page, k_row, v_row, ks_page, vs_page;
    int k_lane, v_lane[4], ks_lane, vs_lane, k_end, v_end;     // *_end: where the last row's bytes end, from the row's start
};

// The pages of a tile; -1: none.  Pages of 32 tokens and more hold both halves of one.
template <int TT> struct Pages { int p[TT]; };
template <int TT> __device__ __forceinline__ Pages<TT> pages_of(const Where& w, int key) {
    Pages<TT> x;
    x.p[0] = key < w.room ? w.table[key >> w.shift] : -1;
    if constexpr (TT == 2) {
        x.p[1] = x.p[0];
        if (__builtin_expect(w.shift == 4, 0)) x.p[1] = key + 16 < w.room ? w.table[(key >> 4) + 1] : -1;
    }
    return x;
}

// `bytes` bytes from x on, what is read behind them is 0.  Both are the same for the whole wave and said to be so: the compiler would
// otherwise take each load through a loop over the lanes' descriptors.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const void* x, int bytes) {
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)x), hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)x >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)((uintptr_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
// n rows, `row` bytes apart, of which the last ends `end` bytes from its start.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const char* x, int n, long long row, int end) {
    const int bytes = n * (int)row - ((int)row - end);
    return bytes_at(x, n > 0 ? bytes : 0);
}

template <int N> __device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t rs, int at, unsigned* x) {
    static_assert(N == 1 || N == 2 || N % 4 == 0, "");
    if constexpr (N == 1) {
        x[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, at, 0, 0);
    } else if constexpr (N == 2) {
        const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0);
        x[0] = u[0]; x[1] = u[1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(rs, at + 4 * i, 0, 0);
            x[i] = u[0]; x[i + 1] = u[1]; x[i + 2] = u[2]; x[i + 3] = u[3];
        }
    }
}

// Requests a tile, of which keys below hi count.  Rows that do not exist cost no memory traffic and come as zeros: a last tile's values behind
// the last key, whose weight is 0, may have any bits.
template <int F, int D>
__device__ __forceinline__ void load_tile(const Where& w, int key, int hi, const Pages<Tile<F, D>::TT>& pages, Tile<F, D>& t) {
    t.key = key;
    constexpr int TT = Tile<F, D>::TT;
    const char *k[TT], *v[TT];
    const unsigned char *ks[TT], *vs[TT];
#pragma unroll
    for (int h = 0; h < TT; ++h) {
        const bool there = (unsigned)pages.p[h] < (unsigned)w.n_pages;
        const int n = hi - (key + 16 * h);
        t.rows[h] = !there ? 0 : n < 16 ? n : 16;            // 0 and less: none
        if (h && __builtin_expect(w.shift > 4, 1)) {
            k[h] = k[0] + 16 * (int)w.k_row; v[h] = v[0] + 16 * (int)w.v_row;
            if constexpr (F == kRows4) { ks[h] = ks[0] + 16; vs[h] = vs[0] + 16; }
        } else {
            const long long pg = there ? pages.p[h] : 0;
            const int in = (key + 16 * h) & ((1 << w.shift) - 1);      // a page's rows span less than 2^31 bytes
            k[h] = w.k + pg * w.k_page + in * (int)w.k_row; v[h] = w.v + pg * w.v_page + in * (int)w.v_row;
            if constexpr (F == kRows4) { ks[h] = w.ks + pg * w.ks_page + in; vs[h] = w.vs + pg * w.vs_page + in; }
        }
    }
#pragma unroll
    for (int h = 0; h < TT; ++h) {
        const auto rs = rows_at(k[h], t.rows[h], w.k_row, w.k_end);
        if constexpr (F == kRows4) {
            load_words<D / 32>(rs, w.k_lane, t.k[h]);
            t.ks[h] = __builtin_amdgcn_raw_buffer_load_b8(bytes_at(ks[h], t.rows[h] > 0 ? 0x7fffffff : 0), w.ks_lane, 0, 0);
        } else {
#pragma unroll
            for (int s = 0; s < (F == kRows32 ? D / 16 : D / 32); ++s) t.k[h][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, w.k_lane + 64 * s, 0, 0);
        }
    }
#pragma unroll
    for (int h = 0; h < TT; ++h) {
        const auto rs = rows_at(v[h], t.rows[h], w.v_row, w.v_end);
        if constexpr (F == kRows4)
            t.vs[h] = __builtin_amdgcn_raw_buffer_load_b32(bytes_at(vs[h], t.rows[h] > 0 ? 0x7fffffff : 0), w.vs_lane, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F == kRows4 && D == 64) t.v[h][i][0] = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rs, w.v_lane[i], 0, 0);
            else load_words<Tile<F, D>::words>(rs, w.v_lane[i], t.v[h][i]);
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
    float m[NT], l[NT];              // m: before the scale; l: this lane's keys alone
    int see[NT];                     // keys that the lane's row sees
};

// What is not finite among a tile's values, 0 in its place: the rows that see it are marked in LDS, a byte for each row and channel (1: +infinity
// or NaN, 2: -infinity or NaN), and get it when the waves' rows come together.  (Added to the accumulators here it costs registers of the
// loop: d = 64, 64 rows, 1000 tokens over 16000 keys 288 -> 333 us.)
template <int F, int D, int NT>
__device__ __forceinline__ void set_apart(Tile<F, D>& t, Rows<F, D, NT>& r, unsigned* marks, bool& marked) {
    constexpr int TT = Tile<F, D>::TT, PER = D / 16;                     // channels that a lane has of a key
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                       // nothing of this before the branch that leads here
    const int n16 = lane & 15, g = lane >> 4;
    if (!marked) {
#pragma unroll 1
        for (int i = lane; i < 4 * NT * D; i += 64) marks[i] = 0;
    }
    marked = true;
#pragma unroll
    for (int h = 0; h < TT; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_sched_barrier(0);           // one key's after the other's: few registers
            unsigned w[(PER + 3) / 4] = {};
            if constexpr (F == kRows4) {
                const bool bad = (t.vs[h] >> (8 * i) & 255u) == 255u;
#pragma unroll
                for (int j = 0; j < PER / 4; ++j) w[j] = bad ? 0x03030303u : 0u;
                t.v[h][i][0] = bad ? 0u : t.v[h][i][0];
                t.vs[h] = bad ? (t.vs[h] & ~(255u << (8 * i))) | (127u << (8 * i)) : t.vs[h];
            } else {
#pragma unroll
                for (int c = 0; c < Tile<F, D>::words; ++c) {
                    const unsigned u = t.v[h][i][c];
                    if constexpr (F == kRows32) {
                        const unsigned bad = ((u & 0x7f800000u) + 0x00800000u) >> 31, nan = ((u & 0x7fffffu) + 0x7fffffu) >> 23, below = u >> 31;
                        w[c / 4] |= bad * ((nan | (1 - below)) + 2 * (nan | below)) << (8 * (c & 3));
                        t.v[h][i][c] = u & (bad - 1);
                    } else {                             // bits 15 and 31: not finite; NaN or of the sign
                        const unsigned bad = not_finite(u), nan = ((u & 0x007f007fu) + 0x007f007fu) << 8;
                        const unsigned m = (bad & (nan | ~u)) >> 15 | (bad & (nan | u)) >> 14;
                        w[c / 2] |= ((m & 3u) | (m >> 8 & 0x300u)) << (16 * (c & 1));
                        t.v[h][i][c] = finite(u);
                    }
                }
                if (PER == 2) w[0] <<= 16 * (n16 & 1);
            }
            const int key = t.key + 16 * h + 4 * g + i;
            unsigned any = 0;
#pragma unroll
            for (int j = 0; j < (PER + 3) / 4; ++j) any |= w[j];
            if (!__any(any != 0)) continue;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll 1
                for (int row = 0; row < 16; ++row) {
                    const int see = __builtin_amdgcn_readlane(r.see[n], row);        // (by all lanes: a lane that is off may hold anything)
                    if (!any || key >= see) continue;
#pragma unroll
                    for (int j = 0; j < (PER + 3) / 4; ++j) atomicOr(marks + (16 * n + row) * (D / 4) + PER * n16 / 4 + j, w[j]);
                }
        }
}

template <int F, int D, int NT>
__device__ __forceinline__ void attend_tile(const AttnArgs& p, Tile<F, D>& t, int see_all, int see_some, Rows<F, D, NT>& r, unsigned* marks, bool& marked) {
    constexpr int TT = Tile<F, D>::TT;
    const int g = (threadIdx.x & 63) >> 4;
    bool whole = true;
#pragma unroll
    for (int h = 0; h < TT; ++h) whole = whole && t.rows[h] == 16;
    if constexpr (F == kRows4) {
        if (!whole) {                // codes behind the last row are 0, their scales may be NaN
#pragma unroll
            for (int h = 0; h < TT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (4 * g + i >= t.rows[h]) t.vs[h] = (t.vs[h] & ~(255u << (8 * i))) | (127u << (8 * i));
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
                union { u32x4 u; f32x4 f; } q, k;
                q.u = r.q[n][c];
                k.u = t.k[0][c];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.f[e], q.f[e], s[n][0], 0, 0, 0);
            }
        }
        // Ten wait states until a result may be read: the compiler counts none for a read behind the branch below.
#pragma unroll
        for (int n = 0; n < NT; ++n) asm volatile("s_nop 9" : "+v"(s[n][0]));
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
    // weights (scores and references before the scale c: one multiply-add makes the exponent of both)
    if (__builtin_expect(!(whole && t.key + 16 * TT <= see_all), 0)) {
        int base = 4 * g;
        asm volatile("" : "+v"(base));                   // else 50 instructions of this stand in every tile's way
        if (see_all < see_some && t.key + 16 * TT > see_all) {       // a row may see more than another: 0 times what is not finite must not reach that
            unsigned bad = 0;
#pragma unroll
            for (int h = 0; h < TT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (F == kRows4) {
                        bad |= ((t.vs[h] >> (8 * i) & 255u) + 1) & 256u;
                    } else {
#pragma unroll
                        for (int j = 0; j < Tile<F, D>::words; ++j)
                            bad |= F == kRows32 ? ((t.v[h][i][j] & 0x7f800000u) + 0x00800000u) & 0x80000000u : not_finite(t.v[h][i][j]);
                    }
                }
            if (__any(bad != 0)) {
                set_apart<F, D, NT>(t, r, marks, marked);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < TT; ++h) {
                const int left = r.see[n] - t.key - 16 * h, lim = left < t.rows[h] ? left : t.rows[h];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][h][i] = base + i < lim ? s[n][h][i] : -INFINITY;
            }
    }
    union { bf16x8 b; __bf16 e[8]; } pb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float top = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3]));
        if constexpr (TT == 2) top = fmaxf(top, fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3])));
        if (__builtin_expect(__any(top > r.m[n] + p.slack), 0)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m = fmaxf(top, r.m[n]);
            const float down = m == -INFINITY || m == r.m[n] ? 1.f : exp2f((r.m[n] - m) * p.c);
            r.m[n] = m;
            r.l[n] *= down;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) r.o[n][j] *= down;
        }
        const float ref = r.m[n] == -INFINITY ? 0.f : r.m[n] * p.c;
#pragma unroll
        for (int h = 0; h < TT; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][h][i] = __builtin_amdgcn_exp2f(fmaf(s[n][h][i], p.c, -ref));
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
                    r.o[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[0][i][j]), s[n][0][i], r.o[n][j], 0, 0, 0);
    } else {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {              // two channels at a time
            unsigned x[TT][4];
#pragma unroll
            for (int h = 0; h < TT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (F == kRows4) x[h][i] = fp4_pair(t.v[h][i][0], __uint_as_float(((t.vs[h] >> (8 * i)) & 255u) << 23), c);
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

// A sequence as a work-group's stretch meets it.
struct Part { int b, len, units, tiles; KvSeq sq; };
template <int R> __device__ __forceinline__ Part part_of(const AttnArgs& p, int b) {
    Part x;
    x.b = b;
    x.sq = kv_seq(p.a, b);
    x.len = p.a.kv_len[b];
    x.units = p.whole ? x.sq.n > 0 : deal_units(seen(p.a, x.len, x.sq.n, x.sq.n - 1), x.sq.n);
    x.tiles = (x.sq.n * p.a.grp + R - 1) / R;
    return x;
}

// Sums of the lanes up to each lane: within 16, then over the rows of 16 before.
__device__ __forceinline__ unsigned wave_scan(unsigned x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast 15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// The line of units (see aa_kv_deal.h) as a wave works it out alone, 64 sequences at a time: units of one KV head, and the sequence that
// holds unit `at` of a head with the units before it.
template <int R> struct Line {
    const AttnArgs& p;
    Part y;                                                  // the lane's sequence
    unsigned x, upto;                                        // its units; with those before in the same 64
    __device__ __forceinline__ Line(const AttnArgs& args) : p(args) {}
    __device__ __forceinline__ void load(int first) {
        const int b = first + (threadIdx.x & 63);
        x = 0;
        if (b < p.a.B) {
            y = part_of<R>(p, b);
            x = (unsigned)y.units * y.tiles;
        }
        upto = wave_scan(x);
    }
    __device__ __forceinline__ unsigned units() {
        unsigned sum = 0;
        for (int first = 0; first < p.a.B; first += 64) {
            load(first);
            sum += __builtin_amdgcn_readlane(upto, 63);
        }
        return sum;
    }
    // after units()
    __device__ __forceinline__ Part find(unsigned at, unsigned* before) {
        unsigned base = 0;
        for (int first = 0; first < p.a.B; first += 64) {
            if (p.a.B > 64) load(first);
            const unsigned long long after = __ballot(base + upto > at);
            if (after) {
                const int l = __ffsll(after) - 1;
                *before = base + __builtin_amdgcn_readlane(upto - x, l);
                Part s;
                s.b = first + l;
                s.len = __builtin_amdgcn_readlane(y.len, l);
                s.units = __builtin_amdgcn_readlane(y.units, l);
                s.tiles = __builtin_amdgcn_readlane(y.tiles, l);
                s.sq.n = __builtin_amdgcn_readlane(y.sq.n, l);
                s.sq.row0 = (long long)(unsigned)__builtin_amdgcn_readlane((int)y.sq.row0, l);     // rows are counted in 31 bits
                return s;
            }
            base += __builtin_amdgcn_readlane(upto, 63);
        }
        return part_of<R>(p, 0);                             // not reached: `at` is below units()
    }
};

__device__ __forceinline__ Deal deal_of(const AttnArgs& p, unsigned total) {
    Deal d;
    d.each = p.by_groups.div(total);
    d.more = total - d.each * p.groups;
    return d;
}

// What the joining kernel is told by the work-group that ends inside a tile which it has begun (the first of those that share it).
struct Shared { int b, hk, r0, count; };
__device__ __forceinline__ Shared* shared_tiles(const AttnArgs& p, int R, int D) { return (Shared*)(p.ws + 2ll * p.groups * R * (D + 2)); }

template <int F, int D, int NT>
__global__ __launch_bounds__(64 * kWaves, (kOccupancy<F, D, NT>)) void kv_attn_kernel(AttnArgs p) {
    using T = typename RowType<F>::type;
    constexpr int item = sizeof(T), TT = Tile<F, D>::TT, TK = 16 * TT, R = 16 * NT, P = D + 4;
    static_assert(kUnitKeys % (kWaves * TK) == 0, "a unit is whole rounds of the waves");
    __shared__ float s_o[kWaves][16][P];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ unsigned s_marks[kWaves][R * D / 4];      // see set_apart
    __shared__ bool s_marked[kWaves];
    const KvArgs& a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    // this work-group's stretch, and where it begins
    unsigned head_units, before = 0;
    Part s = part_of<R>(p, 0);
    Line<R> line(p);
    if (a.B == 1) head_units = (unsigned)s.units * s.tiles;
    else head_units = line.units();
    Shared* const told = p.tell ? shared_tiles(p, R, D) + blockIdx.x : nullptr;
    if (told && threadIdx.x == 0) told->count = 0;
    const unsigned total = head_units * a.Hkv;
    const Deal deal = deal_of(p, total);
    unsigned at = deal_start(deal, blockIdx.x);
    const unsigned end = deal_start(deal, blockIdx.x + 1);
    if (at >= end) return;
    int hk = (int)(at / head_units);
    const unsigned in_head = at - hk * head_units;
    if (a.B > 1) s = line.find(in_head, &before);
    int tile_no = p.tiles == 1 ? 0 : (int)((in_head - before) / s.units);
    int t = (int)(in_head - before) - tile_no * s.units;

    Where w;
    w.room = (long long)a.max_pages << a.page_shift;
    w.shift = a.page_shift;
    w.n_pages = a.n_pages;
    constexpr int unit = F == kRows4 ? 1 : item, row_bytes = F == kRows4 ? D / 2 : D * item;
    w.k_page = a.kcs[0] * unit; w.v_page = a.vcs[0] * unit;
    w.k_row = a.kcs[2] * unit; w.v_row = a.vcs[2] * unit;
    w.k_end = w.v_end = row_bytes;
    w.k_lane = n16 * (int)w.k_row + g * (F == kRows4 ? D / 8 : 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) w.v_lane[i] = (4 * g + i) * (int)w.v_row + n16 * (row_bytes / 16);
    if constexpr (F == kRows4) {
        w.ks_page = a.kss[0]; w.vs_page = a.vss[0];
        w.ks_lane = n16 + g * (D / 4) / kFp4Group * (int)a.kss[2];
        w.vs_lane = 4 * g + n16 * (D / 16) / kFp4Group * (int)a.vss[2];
    }

    for (;;) {                                           // over the row tiles that the stretch touches
        bool marked = false;
        const int stop = s.units - t < (int)(end - at) ? s.units : t + (int)(end - at);
        const int r0 = tile_no * R, rows = s.sq.n * a.grp, last = r0 + R < rows ? r0 + R - 1 : rows - 1;
        const int see_first = seen(a, s.len, s.sq.n, (int)p.by_grp.div(r0)), see_last = seen(a, s.len, s.sq.n, (int)p.by_grp.div(last));
        const int hi = !p.whole && stop * kUnitKeys < see_last ? stop * kUnitKeys : see_last;
        w.table = (const_int*)(a.table + s.b * a.table_stride);
        w.k = a.kc + hk * a.kcs[1] * unit; w.v = a.vc + hk * a.vcs[1] * unit;
        if constexpr (F == kRows4) { w.ks = a.ksc + hk * a.kss[1]; w.vs = a.vsc + hk * a.vss[1]; }
        // tiles of keys go to the waves in turn
        int key = t * kUnitKeys + wave * TK;
        Pages<TT> pages = pages_of<TT>(w, key);
        Tile<F, D> t0, t1;
        load_tile<F, D>(w, key, hi, pages, t0);
        pages = pages_of<TT>(w, key + kWaves * TK);

        Rows<F, D, NT> r;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = r0 + 16 * n + n16 < rows ? r0 + 16 * n + n16 : rows - 1;
            const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
            r.see[n] = seen(a, s.len, s.sq.n, i);
            r.m[n] = -INFINITY;
            r.l[n] = 0.f;
            const char* q = (const char*)p.q + kv_row(a, a.qs, s.b, s.sq.row0, i, h) * item;
#pragma unroll
            for (int c = 0; c < Rows<F, D, NT>::Q; ++c)
                r.q[n][c] = *(const u32x4*)(q + (F == kRows4 ? (D / 2) * g + 16 * c : 64 * c + 16 * g));
#pragma unroll
            for (int j = 0; j < D / 16; ++j) r.o[n][j] = f32x4{0, 0, 0, 0};
        }

        // Two tiles in registers, one loading while the other is attended.  Behind the last one a tile without rows is loaded, so that every
        // path has as much in flight.  (Three or four tiles for 4 bits: slower, 131 / 133 / 153 us for 64 sequences, 0.5 M keys.)
        if (key < hi) {
            for (;;) {
                key += kWaves * TK;
                load_tile<F, D>(w, key, hi, pages, t1);
                pages = pages_of<TT>(w, key + kWaves * TK);
                attend_tile<F, D, NT>(p, t0, see_first, see_last, r, s_marks[wave], marked);
                if (key >= hi) break;
                key += kWaves * TK;
                load_tile<F, D>(w, key, hi, pages, t0);
                pages = pages_of<TT>(w, key + kWaves * TK);
                attend_tile<F, D, NT>(p, t1, see_first, see_last, r, s_marks[wave], marked);
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
            __syncthreads();                             // the last rows have been read
            if (g == 0) { s_m[wave][n16] = r.m[n] * p.c; s_l[wave][n16] = l; }
            if (n == 0 && lane == 0) s_marked[wave] = marked;
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
                if (s_marked[k]) {
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        const unsigned m = s_marks[k][(16 * n + x) * (D / 4) + (c0 + j) / 4] >> (8 * ((c0 + j) & 3));
                        acc[j] += (m & 1 ? INFINITY : 0.f) - (m & 2 ? INFINITY : 0.f);
                    }
                }
            }
            if (t > 0 || stop < s.units) {
                const long long place = (long long)deal_place(blockIdx.x, t) * R + 16 * n + x;
                float* o = p.ws + place * D + c0;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[j] = acc[j];
                if (c0 == 0) {
                    float* ml = p.ws + 2ll * p.groups * R * D + place * 2;
                    ml[0] = m; ml[1] = sum;
                }
            } else {
                const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                T* o = (T*)p.out + kv_row(a, a.os, s.b, s.sq.row0, i, h) + c0;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[j] = (T)(acc[j] * inv);
                if (p.lse && c0 == 0) p.lse[lse_of(a, s.sq, s.b, h, i)] = sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
            }
        }

        if (told && t == 0 && stop < s.units && threadIdx.x == 0) {
            const int shares = (int)(deal_group(deal, at + s.units - 1) - blockIdx.x) + 1, left = p.groups - (int)blockIdx.x;
            *told = Shared{s.b, hk, r0, shares < left ? shares : left};      // (more only if cu_seqlens does not ascend)
        }

        // the next row tile
        at += stop - t;
        if (at >= end) return;
        if (s_marked[0] | s_marked[1] | s_marked[2] | s_marked[3]) __syncthreads();         // the marks have been read
        t = 0;
        if (++tile_no == s.tiles) {
            tile_no = 0;
            int b = s.b;
            do {                                         // (units are left; if lengths change under a call it ends here)
                if (++b == a.B) { b = 0; if (++hk == a.Hkv) return; }
                s = part_of<R>(p, b);
            } while (s.units == 0);
        }
    }
}

// The shares of a row together, a wave a row or (TEAM = 4) a work-group a row: their maxima and sums, a share a lane, leave a weight for
// each in LDS; D / 4 lanes take a share, 16 bytes of its row each, 256 / D shares a wave at once and two or eight (BATCH) times as many on
// their way, the first of them before the weights are known (1000 keys: 9.8 -> 9.2 us with the kernel before).
// place(s): where share s stands; o, ml: the first place's values, and maximum and sum.
// mine: maximum and sum of share `lane`, requested ahead (of a share beyond count: anything).
constexpr int kMaxShares = 1024;
template <class T, int D, int TEAM, int BATCH, class Place>
__device__ __forceinline__ void join_batches(const AttnArgs& p, int count, const float* o, const float* ml, Place place, f32x2 mine,
                                         float* weights, f32x4* part, T* out, float* lse) {
    constexpr int L = D / 4, S = 64 / L;
    const int lane = threadIdx.x & 63, wave = TEAM == 1 ? 0 : threadIdx.x >> 6, c = lane % L;
    // a batch's requests at a time, also of the last ones (again, and not added); the first before the weights are known
    f32x4 v[BATCH];
    auto load = [&](int s0) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) v[k] = *(const f32x4*)(o + place(s0 + k * TEAM * S < count ? s0 + k * TEAM * S : count - 1) * D + 4 * c);
    };
    int s0 = wave * S + lane / L;
    load(s0);
    if (lane >= count) mine = f32x2{-INFINITY, 0.f};
    float m = mine[0];
    for (int s = lane + 64; s < count; s += 64) m = fmaxf(m, ml[2 * place(s)]);
#pragma unroll
    for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    const float ref = m == -INFINITY ? 0.f : m;
    float l = exp2f(mine[0] - ref) * mine[1];
    weights[lane] = exp2f(mine[0] - ref);                    // every wave its own: LDS keeps a wave's order
    for (int s = lane + 64; s < count; s += 64) {
        const float f = exp2f(ml[2 * place(s)] - ref);
        weights[s] = f;
        l += f * ml[2 * place(s) + 1];
    }
#pragma unroll
    for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
    f32x4 acc = {0, 0, 0, 0};
    for (;;) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const bool more = s0 + k * TEAM * S < count;
            const float f = weights[more ? s0 + k * TEAM * S : 0];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = more ? fmaf(f, v[k][e], acc[e]) : acc[e];
        }
        s0 += BATCH * TEAM * S;
        if (s0 >= count) break;
        load(s0);
    }
#pragma unroll
    for (int x = L; x < 64; x *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], x);
    if constexpr (TEAM > 1) {
        if (lane < L) part[wave * L + c] = acc;
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int k = 1; k < TEAM; ++k) acc += part[k * L + c];
    }
    if (lane >= L) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[4 * c + e] = (T)(l == 0.f ? 0.f : acc[e] / l);
    if (lse && c == 0) *lse = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

template <class T, int D, int TEAM, class Place>
__device__ __forceinline__ void join_row(const AttnArgs& p, int count, const float* o, const float* ml, Place place, f32x2 mine,
                                         float* weights, f32x4* part, T* out, float* lse) {
    if (count <= 2 * TEAM * (256 / D)) join_batches<T, D, TEAM, 2>(p, count, o, ml, place, mine, weights, part, out, lse);
    else join_batches<T, D, TEAM, 8>(p, count, o, ml, place, mine, weights, part, out, lse);
}

// The chunk kernel's shares, which stand row by row: a work-group for four rows of a KV head.
template <class T, int D>
__global__ __launch_bounds__(256) void kv_join_rows_kernel(AttnArgs p) {
    __shared__ float s_w[4][kMaxShares];
    const KvArgs& a = p.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int b = blockIdx.y, four = (int)p.by_hkv.div(blockIdx.x), hk = (int)blockIdx.x - four * a.Hkv, row = 4 * four + wave;
    const KvSeq sq = kv_seq(a, b);
    const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
    if (i >= sq.n) return;
    // a share wrote this row if its keys begin before those that the row's tile of rows sees end; before those of the row is enough
    const int len = a.kv_len[b], keys = share_keys(p, len, sq.n);
    int parts = (seen(a, len, sq.n, i) + keys - 1) / keys;
    parts = parts > p.splits ? p.splits : parts < 1 ? 1 : parts;
    const long long at = (((long long)b * a.Hkv + hk) * p.rows + row) * p.splits;
    const float* ml = share_sums(p, D);
    join_row<T, D, 1>(p, parts, p.ws, ml, [=](int s) { return at + s; }, *(const f32x2*)(ml + 2 * (at + (lane < parts ? lane : 0))), s_w[wave],
                      nullptr, (T*)p.out + kv_row(a, a.os, b, sq.row0, i, h), p.lse ? p.lse + lse_of(a, sq, b, h, i) : nullptr);
}

// kv_attn_kernel's shares of many row tiles: its work-groups tell which tiles are shared; a work-group for four rows of each.
template <class T, int D, int R>
__global__ __launch_bounds__(256) void kv_join_kernel(AttnArgs p) {
    __shared__ float s_w[4][kMaxShares];
    const KvArgs& a = p.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int group = blockIdx.x, r = 4 * blockIdx.y + wave;
    auto place = [=](int s) { return (long long)deal_place(group + s, s) * R + r; };
    const float* ml = p.ws + 2ll * p.groups * R * D;
    const f32x2 mine = *(const f32x2*)(ml + 2 * place(group + lane < p.groups ? lane : 0));      // some place's: on its way with what is told
    const Shared told = shared_tiles(p, R, D)[group];
    if (!told.count) return;
    const KvSeq sq = kv_seq(a, told.b);
    const int row = told.r0 + r, i = (int)p.by_grp.div(row), h = told.hk * a.grp + row - i * a.grp;
    if (r >= R || i >= sq.n) return;
    join_row<T, D, 1>(p, told.count, p.ws, ml, place, mine, s_w[wave], nullptr, (T*)p.out + kv_row(a, a.os, told.b, sq.row0, i, h),
                      p.lse ? p.lse + lse_of(a, sq, told.b, h, i) : nullptr);
}

// Of one sequence with few row tiles: where a tile's units are dealt to is known without being told, and it has many shares; a
// work-group a row.
template <class T, int D, int R>
__global__ __launch_bounds__(256) void kv_join_one_kernel(AttnArgs p) {
    __shared__ float s_w[4][kMaxShares];
    __shared__ f32x4 s_o[D];
    const KvArgs& a = p.a;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int row = (int)p.by_hkv.div(blockIdx.x), hk = (int)blockIdx.x - row * a.Hkv, i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
    const Part s = part_of<R>(p, 0);
    if (i >= s.sq.n) return;
    const Deal deal = deal_of(p, (unsigned)s.units * s.tiles * a.Hkv);
    const unsigned first = ((unsigned)hk * s.tiles + row / R) * s.units;
    const int group = (int)deal_group(deal, first), count = (int)deal_group(deal, first + s.units - 1) - group + 1;
    if (count == 1) return;                                  // finished where it was computed
    auto place = [=](int k) { return (long long)deal_place(group + k, k) * R + row % R; };
    const float* ml = p.ws + 2ll * p.groups * R * D;
    join_row<T, D, 4>(p, count, p.ws, ml, place, *(const f32x2*)(ml + 2 * place(lane < count ? lane : 0)), s_w[wave], s_o,
                      (T*)p.out + kv_row(a, a.os, 0, s.sq.row0, i, h), p.lse ? p.lse + lse_of(a, s.sq, 0, h, i) : nullptr);
}

// Rows of a work-group.  More rows share a key that is read once, but take registers from the tiles in flight; 128 share it through LDS.
// 32 / 8 heads, d = 128, rows of a KV head and us with 16 / 32 / 128 rows a work-group:
//   32 sequences, 0.24 M keys, bf16   4: 141 / 144 / 169   16: 148 / 149 / 173   20: 232 / 153 / 177   36: 334 / 252 / 186
//   2 sequences, 25000 keys, bf16     4: 25.8 / 27.5 / 24.9   20: 40.5 / 30.3 / 25.8   64: 67.6 / 43.8 / 30.9
//   64 sequences, 0.53 M keys, 4 bits   8: 125 / 147 / 478   32: 202 / 151 / 485   36: 279 / 252 / 503   64: 371 / 256 / 511
//   1 sequence, 30000 keys, 4 bits    120: 51.4 / 42.6 / 43.1
// (LDS: the conversion of 4 bits and the matrix products of 128 rows take their time however few rows there are.)  d = 64, 4 x 8000 keys:
// 2000 rows, 16 / 32 / 64 rows 195 / 153 / 92.  Float has no kernel through LDS.
int tile_rows(long long rows, int d, int dtype, int format) {
    if (rows <= 16) return 16;
    if (rows <= 32 || (d == 128 && dtype == 0) || (d == 128 && format && rows <= 64)) return 32;
    return d == 128 ? kChunkRows : 64;
}

constexpr long long kMaxGrid = 1ll << 24;     // work-groups of 256 threads: a launch counts its threads in 32 bits

template <int F, int D, int NT>
int run_registers(const AttnArgs& p, hipStream_t st) {
    using T = typename RowType<F>::type;
    int e = (int)launch_kernel(kv_attn_kernel<F, D, NT>, dim3(p.groups), dim3(64 * kWaves), 0, st, p);
    if (e != (int)hipSuccess || !p.ws) return e;
    if (!p.tell) return (int)launch_kernel(kv_join_one_kernel<T, D, 16 * NT>, dim3((unsigned)p.a.Hkv * p.rows), dim3(256), 0, st, p);
    return (int)launch_kernel(kv_join_kernel<T, D, 16 * NT>, dim3(p.groups, ((p.rows < 16 * NT ? p.rows : 16 * NT) + 3) / 4), dim3(256), 0, st, p);
}

template <int F, int D>
int run(const AttnArgs& p, int R, hipStream_t st) {
    using T = typename RowType<F>::type;
    if (R == 16) return run_registers<F, D, 1>(p, st);
    if (R == 32) return run_registers<F, D, 2>(p, st);
    if constexpr (D < 128) return run_registers<F, D, 4>(p, st);
    const int e = launch_kv_chunk(p, F == kRows4, dim3((unsigned)(p.a.Hkv * p.tiles * p.splits), p.a.B), st);
    if (e != (int)hipSuccess || p.splits == 1) return e;
    return (int)launch_kernel(kv_join_rows_kernel<T, D>, dim3((unsigned)(p.a.Hkv * ((p.rows + 3) / 4)), p.a.B), dim3(256), 0, st, p);
}

template <int F, int D> int occupancy(int R) { return R == 16 ? kOccupancy<F, D, 1> : R == 32 ? kOccupancy<F, D, 2> : kOccupancy<F, D, 4>; }

constexpr int kCUs = 256;

}  // namespace

KvSplit kv_split(int B, int Hq, int Hkv, int N, long long total, int d, int dtype, int format, long long longest, long long room) {
    const long long grp = Hq / Hkv, rows = N * grp, R = tile_rows(rows, d, dtype, format), tiles = (rows + R - 1) / R;
    const long long items = tiles * B * Hkv;
    KvSplit s = {0, 1, 0, 0, rows < (1ll << 30)};
    if (R < kChunkRows) {
        // Units are counted in 32 bits, all rows' together: of a packed call the tiles that its rows can fill, not N for every sequence.
        // Where that could be too many, a tile is one unit.
        const long long line = Hkv * (total * grp / R + B < tiles * B ? total * grp / R + B : tiles * B);
        s.fits = s.fits && line < (1ll << 31);
        // as many work-groups as run at once, or as there are units
        const int o = dtype == 0 ? (d == 32 ? occupancy<kRows32, 32>(R) : d == 64 ? occupancy<kRows32, 64>(R) : occupancy<kRows32, 128>(R))
                    : format ? (d == 64 ? occupancy<kRows4, 64>(R) : occupancy<kRows4, 128>(R))
                             : d == 64 ? occupancy<kRows16, 64>(R) : occupancy<kRows16, 128>(R);
        // Short sequences whole, without shares and the kernel that joins them (3 us, and its launch): a unit more costs a work-group
        // 0.7 us, and takes longer than the join from five units on, unless there are enough tiles to fill the chip.  32 / 8 heads,
        // bf16, shared / whole, us: 1 x 512 keys 9.4 / 9.1, 1 x 1000 9.6 / 13.4, 8 x 1000 15.9 / 14.6, 16 x 2000 28.2 / 24.7,
        // 32 x 100 .. 1991 31.7 / 29.6, 64 x 512 26.3 / 24.1.
        const int tile_units = deal_units((int)longest, 1);
        s.whole = tile_units <= 4 || (tile_units <= 16 && items >= 8 * tile_units) || line * deal_units((int)room, 1) >= (1ll << 31);
        const long long units = items * (s.whole ? 1 : tile_units);
        s.groups = (int)(units < kCUs * o ? units : kCUs * o);
        if (!s.whole && room > kUnitKeys) s.ws_bytes = 2ull * s.groups * R * (d + 2) * 4 + s.groups * sizeof(Shared);
        return s;
    }
    // Row tiles through LDS: all tiles of a KV head begin their keys together, which is what lets an XCD's L2 serve them (dealt evenly like
    // the others, 2048 and 1000 new tokens over 30011 and 8192 took 1148 us instead of 996).  Keys are split until there are as
    // many work-groups as run at once, three a CU, or shares of 256 keys, and up to twice as often where the fullest CU then has
    // less to do: a CU takes 16.5 us for 1000 keys of a tile however many work-groups bring them, a share of 128 rows 0.027 us of the
    // chip's memory time.  32 / 8 heads, 1 / 2 / 3 / 4 / 6 shares: 2 x 800 tokens over 20000 keys 559 / 671 / 563 / 590 / 574 us; 512 over 32768
    // 754 / 423 / 322 / 290 / 288; 1024 and 403 over 16384 and 5003 in 4 bits 496 / 382 / 379 / 383 / 386.
    long long splits = (kCUs * 3 + items - 1) / items;
    if (splits > (longest + 255) / 256) splits = (longest + 255) / 256;
    auto cost = [&](long long n) {
        return 16.5e-3 * (double)((items * n + kCUs - 1) / kCUs) * (double)((longest + n - 1) / n) + (n > 1 ? 4 + 0.027 * (double)(items * n) : 0.);
    };
    for (long long n = splits, most = 2 * splits + 2; n <= most && n * 512 <= longest; ++n)
        if (cost(n) < cost(splits)) splits = n;
    if (splits > kMaxShares) splits = kMaxShares;
    if (Hkv * tiles * splits >= kMaxGrid || Hkv * ((rows + 3) / 4) >= kMaxGrid) splits = 1;
    s.fits = s.fits && Hkv * tiles < kMaxGrid;
    s.splits = (int)splits;
    if (s.splits > 1) s.ws_bytes = (size_t)B * Hkv * rows * s.splits * (d + 2) * 4;
    return s;
}

int launch_kv_attn(const KvArgs& a, int dtype, int format, int d, const KvSplit& sp, const void* q, void* out, float* lse, float* ws,
                   hipStream_t st) {
    AttnArgs p;
    p.a = a;
    p.q = q; p.out = out; p.lse = lse;
    p.ws = sp.ws_bytes ? ws : nullptr;
    p.groups = sp.groups; p.whole = sp.whole; p.splits = sp.splits;
    p.rows = a.N * a.grp;
    const int R = tile_rows(p.rows, d, dtype, format);
    p.tiles = (p.rows + R - 1) / R;
    // Being told costs one sequence with few tiles more than it saves; 16000 keys of 8 KV heads, d = 64, 13 / 63 tiles, untold / told
    // 82 / 80, 308 / 292 us; 2 tiles of 30000 keys in 4 bits 29 / 32, 8 of 8000 in float 36.5 / 39.6.
    p.tell = p.ws && (a.B > 1 || p.tiles > 8 || (long long)a.Hkv * p.rows >= kMaxGrid);
    p.c = a.sigma * kLog2e;
    p.slack = fminf(8.f / p.c, 3.402823466e38f);
    p.by_hkv.set(a.Hkv); p.by_splits.set(sp.splits); p.by_grp.set(a.grp); p.by_groups.set(sp.groups ? sp.groups : 1);
    if (dtype == 0) return d == 32 ? run<kRows32, 32>(p, R, st) : d == 64 ? run<kRows32, 64>(p, R, st) : d == 128 ? run<kRows32, 128>(p, R, st) : -1;
    if (format) return d == 64 ? run<kRows4, 64>(p, R, st) : d == 128 ? run<kRows4, 128>(p, R, st) : -1;
    return d == 64 ? run<kRows16, 64>(p, R, st) : d == 128 ? run<kRows16, 128>(p, R, st) : -1;
}

}  // namespace aa
