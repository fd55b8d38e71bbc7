// kv_attn for many rows (chunks of a prompt): the tile loop of engine_bf16_kernel on pages.
//
//   work-group = 128 rows of one KV head (row r = token * grp + head: all query heads of the KV head read one tile) = 4 waves x 32
//   rows, three work-groups per CU; tiles of 64 keys, two K stages and one V stage in LDS;
//   S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16, a lane owning one row (see aa_engine_bf16_common.h).
// A tile's keys come from up to four pages, 16 from each at least: wave w fetches keys 16 w .. 16 w + 15, which lie in one page, so the
// address is scalar but for a lane's constant place.  A 1 KB group of LDS then holds four consecutive keys (key kk in group kk / 4, row
// kk % 4); the operand reads see the same groups and rows as there, so only the masks know that the keys stand in another order:
// row m of the score tile's half kb is key 4 (m % 16) + 2 kb + m / 16.
// 4-bit pages: a lane loads 32 channels of a key (16 bytes and a scale), converts them (exactly: bf16 holds every code's value) and
// writes them where a direct load would have put them; K of the next tile while the P V products run, V at the next tile's start.
// Rows of values behind the last key, or without storage, are cleared in LDS: their weight is 0, their bits may be anything.  What is not
// finite in a tile that some row does not see whole is added to the rows that see it, and cleared before the product.
// Bound by the matrix pipe and a wave's own chain, as that engine: 2048 and 1000 new tokens over 30011 and 8192, 32 / 8 heads, bf16 1.10 TFLOP
// in 986 to 1058 us by card, 1.04 to 1.11 PFLOP/s (a large matrix product: 1.26); 1024 and 403 over 16384 and 5003 in 4 bits 0.30 TFLOP in 354
// to 371 us with the join (6144 over 16384, three work-groups a CU and no join: 1.04).
#include "aa_engine_bf16_common.h"
#include "aa_kv_attn.h"

namespace aa {

using namespace eng;

namespace {

using u32x4 = __attribute__((ext_vector_type(4))) unsigned;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;

__device__ __forceinline__ void chunk_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Whether a V tile holds what is not finite: the whole tile, so that all lanes agree.
__device__ __forceinline__ bool values_not_finite(const char* Vs) {
    unsigned bad = 0;
    const char* at = Vs + 16 * counted_lane();
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const u32x4 x = *(const u32x4*)(at + i * VGRP);
        bad |= not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3]);
    }
    return __any(bad != 0);
}

// What is not finite in a V tile goes to the rows that see it, key by key (lim: keys of the tile that the lane's row sees).  `place`: 4 KB of the wave,
// where 16 of a lane's channels stand meanwhile, as registers for this would be taken from the tiles.
__device__ __forceinline__ void add_not_finite(const char* Vs, char* place, int lim, floatx16 (&o)[4]) {
    const int ln = counted_lane();
    float* mine = (float*)place + ln;
#pragma unroll
    for (int db = 0; db < 4; ++db) {
#pragma unroll
        for (int v = 0; v < 16; ++v) mine[64 * v] = o[db][v];
#pragma unroll 1
        for (int kk = 0; kk < TK; ++kk) {
            const char* row = Vs + (kk >> 2) * VGRP + (kk & 3) * 256;
            if (!__any(not_finite(*(const unsigned*)(row + 4 * ln)) != 0)) continue;
#pragma unroll 1
            for (int v = 0; v < 16; ++v) {
                const unsigned u = (unsigned)*(const unsigned short*)(row + 64 * db + 16 * (v >> 2) + 8 * (ln >> 5) + 2 * (v & 3)) << 16;
                if ((u & 0x7f800000u) == 0x7f800000u && kk < lim) mine[64 * v] += __uint_as_float(u);
            }
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] = mine[64 * v];
    }
}

template <bool FP4>
__global__ __launch_bounds__(256, 3) void kv_chunk_kernel(AttnArgs p) {
    __shared__ __attribute__((aligned(16))) char Ks0[KBYTES], Ks1[KBYTES], Vs0[VBYTES];
    const KvArgs& a = p.a;
    int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int n = lane & 31, hf = lane >> 5;
    AttnPart w;
    if (!attn_part<kChunkRows>(p, w)) return;
    __builtin_amdgcn_s_setprio(2);                   // against the softmax of the SIMD's other waves
    const int nT = (w.hi - w.lo + TK - 1) / TK;
    const int rw = w.r0 + 32 * wave;                 // the wave's first row; rows past the end repeat the last one and are not stored
    const int row = rw + n < w.rows ? rw + n : w.rows - 1;
    const int wave_first = rw < w.rows ? rw : w.rows - 1;
    const int see_wave = seen(a, w.len, w.sq.n, (int)p.by_grp.div(wave_first));
    const int wave_last = rw + 31 < w.rows ? rw + 31 : w.rows - 1;
    const int see_wave_last = seen(a, w.len, w.sq.n, (int)p.by_grp.div(wave_last));

    // ---- loader role: keys 16 wave .. 16 wave + 15 of a tile
    const_int* table = (const_int*)(a.table + w.b * a.table_stride);
    const long long room = (long long)a.max_pages << a.page_shift;
    // Pages of a tile: the wave's own, and which of the four groups of 16 keys have one.  The entries are requested two tiles ahead, in the
    // softmax, where nothing else is in flight in the scalar and LDS units: a scalar load on its way while operands are read from
    // LDS would turn every wait for one of them into a wait for all (looked up at the tile's start: 1032 us for 1014 us here).
    struct Entries { int x[4]; };
    struct Pages { int own; unsigned there; };
    auto entries_of = [&](int t) -> Entries {
        Entries e;
        const int j = w.lo + TK * t;
        e.x[0] = j < room ? table[j >> a.page_shift] : -1;
        e.x[1] = e.x[2] = e.x[3] = e.x[0];
        if (__builtin_expect(a.page_shift < 6, 0)) {
#pragma unroll
            for (int i = 1; i < 4; ++i) e.x[i] = j + 16 * i < room ? table[(j + 16 * i) >> a.page_shift] : -1;
        }
        return e;
    };
    auto pages_of = [&](const Entries& e) -> Pages {
        Pages g;
        g.there = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) g.there |= (unsigned)((unsigned)e.x[i] < (unsigned)a.n_pages) << i;
        const int x = wave == 0 ? e.x[0] : wave == 1 ? e.x[1] : wave == 2 ? e.x[2] : e.x[3];
        g.own = g.there >> wave & 1 ? x : -1;
        return g;
    };
    auto key_of = [&](int t) -> int { return w.lo + TK * t + 16 * wave; };
    const char* const k0 = a.kc + w.hk * a.kcs[1] * (FP4 ? 1 : 2);
    const char* const v0 = a.vc + w.hk * a.vcs[1] * (FP4 ? 1 : 2);
    const unsigned kstb = (unsigned)a.kcs[2] * (FP4 ? 1 : 2), vstb = (unsigned)a.vcs[2] * (FP4 ? 1 : 2);
    auto base_of = [&](const char* x0, const long long* st, int j, int page) -> const char* {
        return x0 + ((page < 0 ? 0 : page) * st[0] + (j & ((1 << a.page_shift) - 1)) * st[2]) * (FP4 ? 1 : 2);
    };
    auto rows_load = [&](const char* base, unsigned stb, char* dst, int pitch) {
        const int ln = counted_lane();
        const unsigned at = (ln >> 4) * stb + 16 * (ln & 15);
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)(15u * stb + 2u * D), 0x00020000);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(dst + (4 * wave + i) * pitch), 16, (int)at, (int)(4u * i * stb), 0, 0);
    };
    struct Codes { u32x4 x; unsigned byte; };
    auto rsrc_of = [&](const void* x) -> __amdgpu_buffer_rsrc_t {        // (scalar, and said to be)
        const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)x), hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)x >> 32));
        return __builtin_amdgcn_make_buffer_rsrc((void*)((uintptr_t)hi << 32 | lo), 0, 0x7fffffff, 0x00020000);
    };
    auto codes_load = [&](const char* base, unsigned stb, const unsigned char* sc, const long long* ss, int j, int page) -> Codes {
        const int ln = counted_lane();
        Codes c;
        c.x = __builtin_amdgcn_raw_buffer_load_b128(rsrc_of(base), (int)((ln >> 2) * stb + 16 * (ln & 3)), 0, 0);
        const unsigned char* s = sc + w.hk * ss[1] + (page < 0 ? 0 : page) * ss[0] + (j & ((1 << a.page_shift) - 1));
        c.byte = __builtin_amdgcn_raw_buffer_load_b8(rsrc_of(s), (ln >> 2) + (ln & 3) * (int)ss[2], 0, 0);
        return c;
    };
    // piece e of lane 4 key + c goes out in step (e - key) % 4, so that 16 lanes write to all banks
    auto codes_store = [&](const Codes& c, char* stage, int pitch) {
        const int ln = counted_lane(), key = ln >> 2;
        char* dst = stage + (4 * wave + (key >> 2)) * pitch + (key & 3) * 256 + 64 * (ln & 3);
        const float scale = __uint_as_float(c.byte << 23);
        u32x4 x, y;
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] = key & 1 ? c.x[(s + 1) & 3] : c.x[s];
#pragma unroll
        for (int s = 0; s < 4; ++s) y[s] = key & 2 ? x[(s + 2) & 3] : x[s];         // piece (s + key) % 4
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            union { u32x4 u; bf16x2 b[4]; } v;
            v.b[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y[s], scale, 0);
            v.b[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y[s], scale, 1);
            v.b[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y[s], scale, 2);
            v.b[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y[s], scale, 3);
            *(u32x4*)(dst + 16 * ((s + key) & 3)) = v.u;
        }
    };

    // ---- Q fragments (B operand of S^T = K Q^T): lane (n, hf) holds channels 16 ks + 8 hf .. + 8 of its row
    const int qi = (int)p.by_grp.div(row), qh = w.hk * a.grp + row - qi * a.grp;
    bf16x8 qf[8];
    {
        const __bf16* src = (const __bf16*)p.q + kv_row(a, a.qs, w.b, w.sq.row0, qi, qh);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const bf16x8*)(src + 16 * ks + 8 * hf);
    }
    const int see = seen(a, w.len, w.sq.n, qi);
    const float c2 = p.c, gap = rescale_limit(c2);
    float mref, mtrue, l;
    floatx16 o[4];
    init_state(mref, mtrue, l, o);

    const int koff = (n & 15) * KGRP + (n >> 4) * 256 + 16 * hf;
    const int ls = lane & 15, lg = lane >> 4;
    const int voff = (4 * hf + (ls >> 2)) * VGRP + 32 * (lg & 1) + 8 * (ls & 3);

    Pages now = pages_of(entries_of(0)), next = pages_of(entries_of(1));
    const int pg = now.own;
    Codes kc, vc;
    if (nT > 0) {
        if constexpr (FP4) {
            kc = codes_load(base_of(k0, a.kcs, key_of(0), pg), kstb, a.ksc, a.kss, key_of(0), pg);
            vc = codes_load(base_of(v0, a.vcs, key_of(0), pg), vstb, a.vsc, a.vss, key_of(0), pg);
            codes_store(kc, Ks0, KGRP);
            __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
        } else {
            rows_load(base_of(k0, a.kcs, key_of(0), pg), kstb, Ks0, KGRP);
        }
    }
    wait_vmem();
    chunk_barrier();

    auto tile_step = [&](int t, const char* Kcur, char* Knext) __attribute__((always_inline)) {
        const int t0 = w.lo + TK * t, j = key_of(t);
        if constexpr (FP4) codes_store(vc, Vs0, VGRP);
        else rows_load(base_of(v0, a.vcs, j, now.own), vstb, Vs0, VGRP);
        __builtin_amdgcn_sched_barrier(0);
        const unsigned there = now.there;
        const bool whole = there == 15 && t0 + TK <= w.hi;
        const bool on = t0 < see_wave_last && rw < w.rows;
        const char* Kb = Kcur + koff;
        const char* Vb = Vs0 + voff;
        bf16x8 pf[2][2];
        floatx16 s[2];
        if (on) {
            {
                bf16x8 kf[16];
                auto read_k = [&](int i) { kf[i] = *(const bf16x8*)(Kb + 512 * (i & 1) + 32 * (i >> 1)); };
#pragma unroll
                for (int i = 0; i < 4; ++i) read_k(i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i >> 1], i < 2 ? kZero16 : s[i & 1], 0, 0, 0);
                    if (i + 4 < 16) read_k(i + 4);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (__builtin_expect(!(whole && t0 + TK <= see_wave), 0)) {
                const int h = counted_lane() >> 5, lim = (see < w.hi ? see : w.hi) - t0 - 16 * h;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int kk = 32 * ((v >> 2) & 1) + 4 * (v & 3) + 2 * kb + (v >> 3);
                        const bool ok = kk < lim && (there >> (2 * ((v >> 2) & 1) + h) & 1);
                        s[kb][v] = ok ? s[kb][v] : -INFINITY;
                    }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const Entries ahead = entries_of(t + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (on) {
            __builtin_amdgcn_s_setprio(0);
            softmax_tile(s, pf, c2, gap, mref, mtrue, l, o);
            __builtin_amdgcn_s_setprio(2);
        }
        __builtin_amdgcn_sched_barrier(0);
        // the next K tile (past the end the last one again, into a stage that nobody reads)
        const int u = t + 1 < nT ? t + 1 : t, ju = key_of(u), pu = t + 1 < nT ? next.own : now.own;
        if constexpr (FP4) {
            kc = codes_load(base_of(k0, a.kcs, ju, pu), kstb, a.ksc, a.kss, ju, pu);
            vc = codes_load(base_of(v0, a.vcs, ju, pu), vstb, a.vsc, a.vss, ju, pu);
        } else {
            rows_load(base_of(k0, a.kcs, ju, pu), kstb, Knext, KGRP);
        }
        __builtin_amdgcn_sched_barrier(0);
        // V tile t has landed: the four loads of the next K tile are younger
        if constexpr (!FP4) __builtin_amdgcn_s_waitcnt(0x0F74);
        if (__builtin_expect(!whole, 0)) {           // each wave its own 16 rows
            const u32x4 zero = {0, 0, 0, 0};
            const int ln = counted_lane();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int kk = 4 * i + (ln >> 4);
                if (!(there >> wave & 1) || j + kk >= w.hi) *(u32x4*)(Vs0 + (4 * wave + i) * VGRP + 16 * ln) = zero;
            }
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0)
        chunk_barrier();
        if (__builtin_expect(t0 + TK > w.see_first, 0) && values_not_finite(Vs0)) {
            // some row does not see all keys, and 0 times what is not finite must not reach it (all waves are here, the tile of keys is free)
            add_not_finite(Vs0, (char*)Kcur + 4096 * wave, see - t0, o);
            chunk_barrier();
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                u32x4* x = (u32x4*)(Vs0 + (4 * wave + i) * VGRP + 16 * counted_lane());
                u32x4 y = *x;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = finite(y[e]);
                *x = y;
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
            chunk_barrier();
        }
        if (on) {
            shortx4 vlo[16], vhi[16];
            auto read_v = [&](int i) {
                vlo[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) shortx4*)(Vb + (i >> 2) * 256 + 64 * (i & 3)));
                vhi[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) shortx4*)(Vb + 8 * VGRP + (i >> 2) * 256 + 64 * (i & 3)));
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) read_v(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const shortx8 vv = __builtin_shufflevector(vlo[i], vhi[i], 0, 1, 2, 3, 4, 5, 6, 7);
                const int sg = i >> 2, db = i & 3;
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vv), pf[sg >> 1][sg & 1], o[db], 0, 0, 0);
                if (i + 4 < 16) read_v(i + 4);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (FP4) {
            codes_store(kc, Knext, KGRP);
            __builtin_amdgcn_s_waitcnt(0xC07F);
        } else {
            wait_vmem();                             // the next K tile has landed
        }
        chunk_barrier();
        now = next;
        next = pages_of(ahead);
    };
    for (int t = 0; t < nT; t += 2) {
        tile_step(t, Ks0, Ks1);
        if (t + 1 < nT) tile_step(t + 1, Ks1, Ks0);
    }

    // ---- epilogue (no lane's value but addresses lives through the loop)
    const float lt = row_sum(l);
    lane = counted_lane();
    n = lane & 31; hf = lane >> 5;
    if (rw >= w.rows) return;
    if (p.splits > 1) {
        if (rw + n >= w.rows) return;
        const long long at = share_of(p, w, rw + n);
        float* ws = p.ws + at * D;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                *(floatx4*)(ws + 32 * db + 8 * v4 + 4 * hf) =
                    floatx4{o[db][4 * v4], o[db][4 * v4 + 1], o[db][4 * v4 + 2], o[db][4 * v4 + 3]};
        if (hf == 0) {
            float* ml = share_sums(p, D) + at * 2;
            ml[0] = mref * c2;
            ml[1] = lt;
        }
        return;
    }
    // 16 lanes write a row of 256 bytes: the rows through the wave's own piece of the stages, which are free now
    char* const stg = wave == 0 ? Ks0 : wave == 1 ? Ks1 : Vs0 + (wave - 2) * kOutStageBytes;
    static_assert(KBYTES >= kOutStageBytes && VBYTES >= 2 * kOutStageBytes, "staging areas of the output rows");
    unsigned short* sb = (unsigned short*)stg;
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
            const floatx4 x = {o[db][4 * v4] * inv, o[db][4 * v4 + 1] * inv, o[db][4 * v4 + 2] * inv, o[db][4 * v4 + 3] * inv};
            *(bf16x4*)(sb + n * kOutPitch + 32 * db + 8 * v4 + 4 * hf) = __builtin_convertvector(x, bf16x4);
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 4), c = lane & 15;
        const intx4 x = *(const intx4*)(sb + r * kOutPitch + 8 * c);
        if (rw + r < w.rows) {
            const int ti = (int)p.by_grp.div(rw + r), h = w.hk * a.grp + rw + r - ti * a.grp;
            *(intx4*)((unsigned short*)p.out + kv_row(a, a.os, w.b, w.sq.row0, ti, h) + 8 * c) = x;
        }
    }
    if (!p.lse || hf || rw + n >= w.rows) return;
    const int ti = (int)p.by_grp.div(rw + n), th = w.hk * a.grp + rw + n - ti * a.grp;
    p.lse[lse_of(a, w.sq, w.b, th, ti)] = lt == 0.f ? -INFINITY : mref * c2 * kLn2 + logf(lt);
}

}  // namespace

int launch_kv_chunk(const AttnArgs& p, int format, dim3 grid, hipStream_t st) {
    if (format) return (int)launch_kernel(kv_chunk_kernel<true>, grid, dim3(256), 0, st, p);
    return (int)launch_kernel(kv_chunk_kernel<false>, grid, dim3(256), 0, st, p);
}

}  // namespace aa
