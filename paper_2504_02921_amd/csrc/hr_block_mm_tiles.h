// Products of 8-bit matrices through LDS (hr_block_matmul): the kernel, for the files that compile it.
//
// y^T is what the matrix instructions compute, w's rows by a's: a lane then has four neighbouring columns of one row of y and one factor a.scale for all of its
// values of a row of blocks.  A block of 128 columns is summed from zero (one 8-bit instruction of 16 x 16 x 128, or four of halves), scaled by
// a.scale w.scale and added in fp32: one fused multiply-add a value and block, beside the matrix pipe.
//
// 8-bit instruction or halves: of random normal codes the 8-bit instruction reaches 3.4 PFLOP/s from registers with the fused multiply-adds (4.1 without),
// halves 1.97.  But it adds groups of eight neighbouring products after cutting each at 2^-13 of the group's largest, which moves a sum by 1.4e-5 of the row's rms; sums of halves
// are off by 1e-8.  Behind bf16's rounding of a typical value that is little, but where large terms cancel it is more than what is left.  So every kind of result
// takes halves, unless the caller asks for speed (12800 x 4096 x 14336 into bf16 1180 to 1240 us, with the 8-bit instruction 700 to 730).
//
// What bounds it: 8192 x 8192 x 8192 into bf16 by the 8-bit instruction takes 467 us (2.35 PFLOP/s; on another card 493; a library product of the same codes with a single scale 371), with the matrix pipe 65 %
// busy at 1.69 GHz; the same without any load in the loop is 70 % at 1.79.  The clock is what power allows: the products themselves draw most of it (zeros run
// 1.3 times as fast as normal deviates), the fused multiply-adds of the blocks' scales the next part.  Halves: 820 us into bf16 (1.34 PFLOP/s), 843 into
// fp32 (a library product of matrices in half 734).
//
// How: tiles of codes and scales go straight from memory to LDS, rows of 128 bytes whose 16-byte chunks are exchanged by (row / 2) % 8, so that the reads of a
// fragment (16 rows, two chunks a lane) fall on all banks.  Which tiles a call takes goes by what each shape costs (matmul_plan).  Workgroups that share rows of w are
// on one XCD, eight rows of tiles at a time (4, 6 and 16 are within 3 %).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "hr_block_mm.h"

namespace hr {

namespace {

typedef __attribute__((ext_vector_type(8))) int mm_i8;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
constexpr int kNoLoad = 0x7FF00000;      // a vector offset past every range: nothing is fetched, zero arrives

#ifdef __HIP_DEVICE_COMPILE__            // the host pass does not know the descriptor type
typedef __amdgpu_buffer_rsrc_t rsrc_t;
#else
typedef int rsrc_t;
#endif
__device__ __forceinline__ rsrc_t make_rsrc(const void* p, int64_t bytes) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00020000);
#else
    return 0;
#endif
}
// 16 or 4 bytes a lane, straight to LDS: lane l's behind lane l - 1's from a wave-uniform address on
__device__ __forceinline__ void load_lds16(rsrc_t r, void* lds, int voff, int soff) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)lds, 16, voff, soff, 0, 0);
#endif
}
__device__ __forceinline__ void load_lds4(rsrc_t r, void* lds, int voff, int soff) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)lds, 4, voff, soff, 0, 0);
#endif
}

// BM rows x BN rows of w by WM x WN wavefronts, KG groups of which take turns along k, each with NS stages: where there are few tiles, a compute unit's loads are
// what counts (65 x 896 x 4864, 8-bit instruction: 70 tiles of 16 x 64 by four groups 9.6 us, 140 of 16 x 32 by eight 6.9; halves 7.5).  With a gate a wavefront's rows of w are half
// gate rows, half the rows that they multiply.
template <int BM, int BN, int WM, int WN, int NS, int KG, bool EIGHT, bool GATE, typename OUT, bool CODES>
__global__ void __launch_bounds__(WM * WN * KG * 64, WM * WN * KG == 4 ? 2 : 1) block_mm_tile_kernel(MatmulArgs a) {
    constexpr int NWAVE = WM * WN, NT = NWAVE * 64, BK = kBlockCols;       // of a group
    constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
    constexpr int H = GATE ? 2 : 1, BNY = BN / H, TNY = TN / H;            // columns of y
    // The next block's fragments are read under this one's last instructions.  With halves, two rows a wavefront and others that have the same rows of w it
    // lost: 64 x 64 and 64 x 128 tiles 7 to 9 % slower (8-bit instruction: up to 30 % faster)
    constexpr bool PIPE = MI % 2 == 0 && (EIGHT || MI >= 4 || WM == 1);
    constexpr int RPP = NT / 8, PA = (BM + RPP - 1) / RPP, PB = BN / RPP;  // rows a pass of 16-byte loads brings, passes
    constexpr bool SHORT = BM < RPP;                                       // the first wavefronts bring all rows of a
    constexpr int SW = (BM + 63) / 64;                                     // wavefronts that bring the rows' scales
    constexpr int STAGE = (BM + BN) * BK + NT * 4;
    static_assert((SHORT ? BM % 8 : BM % RPP) == 0 && BN % RPP == 0 && SW + H <= NWAVE && (!CODES || BNY % kBlockCols == 0) && TNY <= kBlockCols, "loader shape");
    extern __shared__ __attribute__((aligned(16))) char smem[];

    const int tiles_m = (int)((a.M + BM - 1) / BM), tiles_n = (a.N + BNY - 1) / BNY;
    unsigned pid = blockIdx.x;
    TileCoord tc = map_tile((int)pid, tiles_m, tiles_n);
    if (!tc.valid) return;
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = all / NWAVE, wave = all % NWAVE;
    const int tid = KG > 1 ? (int)threadIdx.x - group * NT : (int)threadIdx.x;
    const int wm = wave / WN, wn = wave % WN, r = lane & 15, fq = lane >> 4;
    const int nk = (int)blocks_of(a.K), turns = (nk + KG - 1) / KG;       // blocks of k; block kt is group kt % KG's in turn kt / KG

    // ---- loads: a wavefront's load brings eight rows of 128 codes
    // which half of w a pass brings goes by the wavefront (a pass has every wavefront's rows) or by the pass
    constexpr bool BY_WAVE = GATE && RPP % TN == 0;
    static_assert(!GATE || NI % 2 == 0, "whole blocks of 16 of either half");
    static_assert(!GATE || BY_WAVE || TNY % RPP == 0, "a load lies in one half");
    // A lane's place in its wavefront's loads: of a and w, kNoLoad behind the last column, and of the scales.  Beside the largest tile's halves there is no
    // register to keep them in (a reload from memory would stand in front of every block's first loads): they are computed when they are used
    constexpr bool CROWDED = PIPE && !EIGHT && MI * NI >= 32;
    auto places = [&](int kt, int& xa, int& xw) {
        int l = lane;
        if constexpr (CROWDED) asm volatile("" : "+v"(l));
        const int lrow = l >> 3, column = ((l & 7) ^ ((wave * 8 + lrow) >> 1 & 7)) * 16;
        const int left = kt < nk ? a.K - kt * BK : 0, in_a = lrow * (int)a.a_stride + column, in_w = lrow * (int)a.w_stride + column;
        xa = column < left ? in_a : kNoLoad;
        xw = column < left ? in_w : kNoLoad;
    };
    const int swave = wave - SW, scale_row = swave < 0 ? wave * 64 : 0, scale_step = (int)(swave < 0 ? a.a_scale_stride : a.w_scale_stride) * 4;
    auto scale_place = [&](int kt) {
        int l = lane;
        if constexpr (CROWDED) asm volatile("" : "+v"(l));
        return (scale_row + l) * scale_step | (kt < nk ? 0 : kNoLoad);
    };
    const int64_t first_half = BY_WAVE && wave * 8 % TN >= TNY ? a.half : 0;
    int64_t m0;
    int n0, pass_a[PA], pass_w[PB];
    rsrc_t ra, rw0, rw1, rs;
    auto set_tile = [&](const TileCoord& t) {
        m0 = (int64_t)t.tm * BM;
        n0 = t.tn * BNY;
        const int rows_a = (int)min((int64_t)BM, a.M - m0), rows_w = min(BNY, a.N - n0);
        ra = make_rsrc(a.a + m0 * a.a_stride, rows_a * a.a_stride);
        rw0 = make_rsrc(a.w + (n0 + first_half) * a.w_stride, rows_w * a.w_stride);
        rw1 = make_rsrc(a.w + (n0 + (int64_t)a.half) * a.w_stride, rows_w * a.w_stride);
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int row = p * RPP + wave * 8;
            pass_a[p] = row < rows_a ? row * (int)a.a_stride : 0;          // a pass of rows that there are not: other rows, not stored
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int row = p * RPP + wave * 8, f = GATE ? row / TN * TNY + row % TNY : row;
            pass_w[p] = f < rows_w ? f * (int)a.w_stride : 0;
        }
        // scales: the first SW wavefronts bring those of the rows, the next one (two) those of w's blocks, the others none
        const int sblocks = swave < H ? (int)blocks_of(rows_w) : 0;
        rs = swave < 0 ? make_rsrc(a.a_scales + m0 * a.a_scale_stride, rows_a * a.a_scale_stride * 4)
                       : make_rsrc(a.w_scales + ((int64_t)n0 + (swave == 1 ? (int64_t)a.half : 0)) / kBlockCols * a.w_scale_stride, sblocks * a.w_scale_stride * 4);
    };
    set_tile(tc);
    auto stage = [&](int s) { return smem + (group * NS + s) * STAGE; };
    constexpr int LPS = PA + PB + 1;                     // loads of a wavefront and block
    // load q of the LPS of a turn's block into stage s; a block past the end fetches nothing, and its zeros add nothing
    auto request_one = [&](int q, int turn, int s, int xa, int xw) {
        char* to = stage(s);
        const int kt = turn * KG + group, at = kt < nk ? kt * BK : 0;
        if (SHORT && q == 0 && wave * 8 >= BM) return;   // goes by the wavefront
        if (q < PA) load_lds16(ra, to + (q * RPP + wave * 8) * BK, xa, pass_a[q < PA ? q : 0] + at);
        else if (q < PA + PB) {
            const int p = q - PA < PB ? q - PA : 0;
            load_lds16(GATE && !BY_WAVE && p * RPP % TN >= TNY ? rw1 : rw0, to + (BM + p * RPP + wave * 8) * BK, xw, pass_w[p] + at);
        } else load_lds4(rs, to + (BM + BN) * BK + wave * 256, scale_place(kt), kt < nk ? kt * 4 : 0);
    };
    auto request = [&](int turn, int s) {
        int xa, xw;
        places(turn * KG + group, xa, xw);
#pragma unroll
        for (int q = 0; q < LPS; ++q) request_one(q, turn, s, xa, xw);
    };
    // the chunk that the rows end in, in the last turn, if they end inside one
    auto mend_end = [&](char* in) {
        for (int row = tid; row < BM + BN && (nk - 1) % KG == group; row += NT) {
            mm_i4* c = (mm_i4*)(in + row * BK + ((a.K % BK / 16) ^ (row >> 1 & 7)) * 16);
            *c = first_codes(*c, a.K % 16);
        }
        __syncthreads();
    };
    // All but the loads of BLOCKS blocks have landed (of which a wavefront that brings no rows of a has one less each)
    auto landed = [&](auto blocks) {
        constexpr int V = decltype(blocks)::value * LPS, V1 = decltype(blocks)::value * (LPS - 1);
        static_assert(V < 64, "the load counter has six bits");
        asm volatile("" ::: "memory");
        if (SHORT && wave * 8 >= BM) __builtin_amdgcn_s_waitcnt((V1 & 15) | ((V1 >> 4) << 14) | 0x0F70);
        else __builtin_amdgcn_s_waitcnt((V & 15) | ((V >> 4) << 14) | 0x0F70);
        asm volatile("" ::: "memory");
    };
    // Everybody is here, and what they wrote to LDS too
    auto meet = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    using std::integral_constant;
    // ... of what a wavefront's own loads brought, which have landed
    auto mend_own = [&](char* in) {
        for (int p = lane >> 3; p < PA + PB && (nk - 1) % KG == group; p += 8) {
            if (SHORT && p == 0 && wave * 8 >= BM) continue;         // others' rows
            const int row = (p < PA ? p * RPP : BM + (p - PA) * RPP) + wave * 8 + (lane & 7);
            mm_i4* c = (mm_i4*)(in + row * BK + ((a.K % BK / 16) ^ (row >> 1 & 7)) * 16);
            *c = first_codes(*c, a.K % 16);
        }
    };

    mm_f4 acc[MI][NI];
    const int sw = r >> 1;
    const int at_a = (wm * TM + r) * BK, at_w = (BM + wn * TN + r) * BK, c0 = (fq ^ sw) * 16, c1 = ((4 + fq) ^ sw) * 16;

    // A workgroup of the large tiles takes one after another and requests the first block of the next before it stores what it has (a tile's
    // start waits for memory for 2 to 3 us): 8-bit instruction, 8192 x 8192 x 8192 2.31 to 2.35 PFLOP/s, 12800 x 28672 x 4096 gated 1404 to 1344 us
    constexpr bool PERSIST = PIPE && KG == 1 && MI >= 4 && NS == 2;
    if constexpr (PERSIST) request(0, 0);
    for (;;) {                                           // one pass unless PERSIST
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mm_f4{0.f, 0.f, 0.f, 0.f};
    if constexpr (PIPE) {
        // A block is MI rows of NI sums; a row's sums are scaled and added while the next row's are computed.  A's fragments are
        // read two rows ahead and w's replaced behind their last use, so that the block's one barrier, in front of its last row but one, finds
        // all of the stage read: what is requested behind it has a whole block's time to land.
        mm_i8 af[2], w8[EIGHT ? NI : 1];
        mm_h8 wh[EIGHT ? 1 : NI][4];
        float as[2], ws[H], sc[2][H];
        mm_f4 part[NI];
        auto fragment = [&](const char* at) {
            const mm_i4 lo = *(const mm_i4*)(at + c0), hi = *(const mm_i4*)(at + c1);
            return mm_i8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        auto read_a = [&](const char* in, int i) {
            af[i & 1] = fragment(in + at_a + i * 16 * BK);
            as[i & 1] = ((const float*)(in + (BM + BN) * BK))[wm * TM + i * 16 + r];
        };
        auto read_w = [&](const char* in, int j) {
            const mm_i8 w = fragment(in + at_w + j * 16 * BK);
            if constexpr (EIGHT) w8[j] = w;
            else {
#pragma unroll
                for (int s = 0; s < 4; ++s) wh[j][s] = halves(w[2 * s], w[2 * s + 1]);
            }
        };
        auto read_ws = [&](const char* in) {
#pragma unroll
            for (int h = 0; h < H; ++h) ws[h] = ((const float*)(in + (BM + BN) * BK))[SW * 64 + h * 64 + wn * TNY / kBlockCols];
        };
        if constexpr (PERSIST) {
            landed(integral_constant<int, 0>{});
        } else {
#pragma unroll
            for (int s = 0; s < NS; ++s) request(s, s);
            landed(integral_constant<int, NS - 1>{});
        }
        if (turns == 1 && a.K % 16 != 0) mend_own(stage(0));
        meet();
        if constexpr (PERSIST) request(1, 1);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            read_w(stage(0), j);
            part[j] = mm_f4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int h = 0; h < H; ++h) sc[1][h] = 0.0f;
        read_ws(stage(0));
        read_a(stage(0), 0);
        read_a(stage(0), 1);
        // Two wavefronts share a SIMD: where one goes first, they do not wait for the same unit at the same time
        if (all >= NWAVE * KG / 2) __builtin_amdgcn_s_setprio(1);
        int slot = 0;
        for (int turn = 0; turn < turns; ++turn) {       // no branch further down: it would keep the compiler from the order there
            if (turn == turns - 2 && a.K % 16 != 0) {
                landed(integral_constant<int, 0>{});
                mend_own(stage(slot + 1 == NS ? 0 : slot + 1));
            }
            int xa = kNoLoad, xw = kNoLoad;
            const int here = slot, ahead = slot + 1 == NS ? 0 : slot + 1, behind = slot == 0 ? NS - 1 : slot - 1;
            char *from = stage(here), *next = stage(ahead);
            slot = ahead;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int cur = i & 1, old = cur ^ 1, iold = i == 0 ? MI - 1 : i - 1;
                if (i == MI - 2) {
                    landed(integral_constant<int, NS - 2>{});      // the next block; those behind it may be on their way
                    meet();
                    places((turn + NS) * KG + group, xa, xw);
                }
#pragma unroll
                for (int h = 0; h < H; ++h) sc[cur][h] = as[cur] * ws[h];
                auto add_old = [&](int j) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[iold][j][e] = fmaf(part[j][e], sc[old][GATE && j >= NI / 2 ? 1 : 0], acc[iold][j][e]);
                };
                auto ask = [&](int j) {                  // a load behind each of the first instructions behind the barrier
                    constexpr int EACH = MI > 2 ? 1 : (LPS + 2 * NI - 1) / (2 * NI);
#pragma unroll
                    for (int e = 0; e < EACH; ++e) {
                        const int q = ((i + 2) % MI * NI + j) * EACH + e;
                        if (q < LPS) request_one(q, i >= MI - 2 ? turn + NS : turn + NS - 1, i >= MI - 2 ? here : behind, xa, xw);
                    }
                };
                static_assert(MI == 2 || PA + PB <= 2 * NI, "codes are requested in the two rows behind the barrier, scales there or behind them");
                if constexpr (EIGHT) {
#pragma unroll
                    for (int j = 0; j < NI; ++j) {
                        add_old(j);
                        part[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8[j], af[cur], mm_f4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
                        if (i == MI - 1) read_w(next, j);
                        ask(j);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const mm_h8 ah = halves(af[cur][2 * s], af[cur][2 * s + 1]);
#pragma unroll
                        for (int j = 0; j < NI; ++j) {
                            if (s == 0) add_old(j);
                            part[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh[j][s], ah, s == 0 ? mm_f4{0.f, 0.f, 0.f, 0.f} : part[j], 0, 0, 0);
                            if (s == 1) ask(j);
                        }
                        if (s % 2 == 1) __builtin_amdgcn_sched_barrier(0);
                    }
                    if (i == MI - 1) {
#pragma unroll
                        for (int j = 0; j < NI; ++j) {
                            read_w(next, j);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
                if (i == MI - 1) read_ws(next);
                read_a(i < MI - 2 ? from : next, i < MI - 2 ? i + 2 : i + 2 - MI);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[MI - 1][j][e] = fmaf(part[j][e], sc[1][GATE && j >= NI / 2 ? 1 : 0], acc[MI - 1][j][e]);
    } else {
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) request(s, s);
        int slot = 0;
        for (int turn = 0; turn < turns; ++turn) {
            landed(integral_constant<int, NS - 2>{});
            meet();                                      // this block has landed, and nobody reads the one before
            const int before = slot == 0 ? NS - 1 : slot - 1;
            request(turn + NS - 1, before);
            char* from = stage(slot);
            if (turn == turns - 1 && a.K % 16 != 0) mend_end(from);
            const float* scales = (const float*)(from + (BM + BN) * BK);
            float ws[H];
#pragma unroll
            for (int h = 0; h < H; ++h) ws[h] = scales[SW * 64 + h * 64 + wn * TNY / kBlockCols];
            mm_i8 w8[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const mm_i4 lo = *(const mm_i4*)(from + at_w + j * 16 * BK + c0), hi = *(const mm_i4*)(from + at_w + j * 16 * BK + c1);
                w8[j] = mm_i8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            }
            mm_h8 wh[EIGHT ? 1 : NI][4];
            if constexpr (!EIGHT) {
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int s = 0; s < 4; ++s) wh[j][s] = halves(w8[j][2 * s], w8[j][2 * s + 1]);
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const float as = scales[wm * TM + i * 16 + r];
                const mm_i4 lo = *(const mm_i4*)(from + at_a + i * 16 * BK + c0), hi = *(const mm_i4*)(from + at_a + i * 16 * BK + c1);
                mm_f4 part[NI];
                if constexpr (EIGHT) {
                    const mm_i8 a8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
                    for (int j = 0; j < NI; ++j) part[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8[j], a8, mm_f4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const mm_h8 ah = s < 2 ? halves(lo[2 * s % 4], lo[2 * s % 4 + 1]) : halves(hi[2 * s % 4], hi[2 * s % 4 + 1]);
#pragma unroll
                        for (int j = 0; j < NI; ++j)
                            part[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh[j][s], ah, s == 0 ? mm_f4{0.f, 0.f, 0.f, 0.f} : part[j], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    const float scale = as * ws[GATE && j >= NI / 2 ? 1 : 0];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(part[j][e], scale, acc[i][j][e]);
                }
            }
            slot = slot + 1 == NS ? 0 : slot + 1;
        }
    }
    const int64_t tile_m0 = m0;
    const int tile_n0 = n0;
    bool another = false;
    if constexpr (PERSIST) {
        pid += gridDim.x;
        if (pid / kXcds < (unsigned)(tiles_m * tiles_n)) tc = map_tile((int)pid, tiles_m, tiles_n);
        else tc.valid = false;
        another = tc.valid;
        // into stage 0, where nobody reads any more what counts: the last block's fragments were read in front of its barrier
        if (another) {
            set_tile(tc);
            request(0, 0);
        }
    }
    if constexpr (KG > 1) {
        // the groups' sums meet in LDS, as many rows at a time as it holds, and leave it in rows
        constexpr int PITCH = BN + 4, SLABS = MI >= 4 ? 4 : MI, IS = MI / SLABS, SR = WM * IS * 16;       // rows of a slab: IS blocks of every wavefront
        float* sums = (float*)smem;
        __builtin_amdgcn_s_waitcnt(0x0F70);              // nothing is on its way into LDS
#pragma unroll
        for (int slab = 0; slab < SLABS; ++slab) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < IS; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
                    *(mm_f4*)(sums + ((group * WM + wm) * IS * 16 + i * 16 + r) * PITCH + wn * TN + j * 16 + 4 * fq) = acc[slab * IS + i][j];
            __syncthreads();
            constexpr int Q = BNY / 4;
            for (int u = threadIdx.x; u < SR * Q; u += NT * KG) {
                const int row = u / Q, col = u % Q * 4;
                const int64_t m = tile_m0 + row / (IS * 16) * TM + slab * IS * 16 + row % (IS * 16);
                const int at = GATE ? col / TNY * TN + col % TNY : col;
                mm_f4 c = *(const mm_f4*)(sums + row * PITCH + at), up = GATE ? *(const mm_f4*)(sums + row * PITCH + at + TNY) : c;
#pragma unroll
                for (int g = 1; g < KG; ++g) {
                    c += *(const mm_f4*)(sums + (g * SR + row) * PITCH + at);
                    if (GATE) up += *(const mm_f4*)(sums + (g * SR + row) * PITCH + at + TNY);
                }
                const mm_f4 y = finish4<GATE>(a, tile_n0 + col, c, up);
                if constexpr (CODES) store_block4(a, m, tile_n0 + col, y, m < a.M);
                else if (m < a.M && tile_n0 + col < a.N) store4<OUT>(a, m, tile_n0 + col, y);
            }
        }
    } else {
        // From registers: a lane has four columns of a row in each block of 16 x 16
        constexpr int NY = NI / H;
        const int64_t row0 = tile_m0 + wm * TM + r;
        const int col0 = tile_n0 + wn * TNY;
        float bias[H][NY][4];
        if (a.bias) {
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int j = 0; j < NY; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int n = col0 + j * 16 + 4 * fq + e;
                        bias[h][j][e] = n < a.N ? a.bias[n + h * a.half] : 0.0f;
                    }
        }
        auto finish = [&](int i) {
            if (a.bias) {
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] += bias[j / NY][j % NY][e];
            }
            if constexpr (GATE) {
#pragma unroll
                for (int j = 0; j < NY; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = gated(acc[i][j][e], acc[i][NY + j][e], a.gate);
            }
        };
        if constexpr (CODES) {
            // a row's largest value over its 128 columns: over a wavefront's by lane swaps, then over the wavefronts that share the block through LDS,
            // in stage 1
            constexpr int SHARE = kBlockCols / TNY;
            float* tops = (float*)(smem + (PERSIST ? STAGE : 0));            // [BM][WN]
            if constexpr (PERSIST) {
                if (another) landed(integral_constant<int, 1>{});      // all but the next tile's block
                else landed(integral_constant<int, 0>{});
            } else {
                landed(integral_constant<int, 0>{});
            }
            meet();
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                finish(i);
                float v[NY * 4];
#pragma unroll
                for (int q = 0; q < NY * 4; ++q) {
                    if (col0 + q / 4 * 16 + 4 * fq + q % 4 >= a.N) acc[i][q / 4][q % 4] = 0.0f;
                    v[q] = acc[i][q / 4][q % 4];
                }
                const float top = max_over_fq(finite_top(v));
                if (fq == 0) tops[(wm * TM + i * 16 + r) * WN + wn] = top;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                float top = 0.0f;
#pragma unroll
                for (int q = 0; q < SHARE; ++q) top = fmaxf(top, tops[(wm * TM + i * 16 + r) * WN + wn / SHARE * SHARE + q]);
                const float scale = scale_of(top), by = 1.0f / scale;
                const int64_t m = row0 + i * 16;
                if (wn % SHARE == 0 && fq == 0 && m < a.M && col0 < a.N) a.scales[m * a.scale_stride + col0 / kBlockCols] = scale;
                uint32_t w[NY];
#pragma unroll
                for (int j = 0; j < NY; ++j) w[j] = codes4(acc[i][j][0] * by, acc[i][j][1] * by, acc[i][j][2] * by, acc[i][j][3] * by);
                store_codes<NY>(a, m, col0, fq, w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                finish(i);
                const int64_t m = row0 + i * 16;
                if constexpr (sizeof(OUT) == 2 && NY % 2 == 0) {
                    // of two blocks side by side a lane takes eight neighbouring columns of one
#pragma unroll
                    for (int j = 0; j < NY; j += 2) {
                        mm_f4 lo, hi;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][j][e]), __float_as_uint(acc[i][j + 1][e]), false, false);
                            lo[e] = __uint_as_float(x[0]);
                            hi[e] = __uint_as_float(x[1]);
                        }
                        const int n = col0 + (j + (fq & 1)) * 16 + (fq >> 1) * 8;
                        if (m < a.M) store8<OUT>(a, m, n, lo, hi);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < NY; ++j) {
                        const int n = col0 + j * 16 + 4 * fq;
                        if (m < a.M && n < a.N) store4<OUT>(a, m, n, acc[i][j]);
                    }
                }
            }
        }
    }
    if (!another) break;
    }
}

template <int BM, int BN, int WM, int WN, int NS, int KG, bool EIGHT, bool GATE, typename OUT, bool CODES>
hipError_t launch_tile(const MatmulArgs& a, hipStream_t st) {
    constexpr size_t stages = (size_t)KG * NS * ((BM + BN) * kBlockCols + WM * WN * 256);
    constexpr size_t slab = KG > 1 ? (size_t)KG * (BM >= 64 * WM ? BM / 4 : WM * 16) * (BN + 4) * sizeof(float) : 0;
    constexpr size_t lds = stages > slab ? stages : slab;
    constexpr bool persist = BM / WM >= 64 && NS == 2 && KG == 1;
    static_assert(lds <= 160 * 1024, "LDS of a CU");
    const auto kernel = block_mm_tile_kernel<BM, BN, WM, WN, NS, KG, EIGHT, GATE, OUT, CODES>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    constexpr int BNY = GATE ? BN / 2 : BN;
    const int64_t tiles = (a.M + BM - 1) / BM * ((a.N + BNY - 1) / BNY);
    const int64_t groups = (tiles + kXcds - 1) / kXcds * kXcds, held = kCus * (WM * WN == 4 ? 2 : 1);
    kernel<<<(unsigned)(persist && groups > held ? held : groups), WM * WN * KG * 64, lds, st>>>(a);
    return hipGetLastError();
}

// DEPTH: stages; TURNS: groups along k
template <bool EIGHT, typename OUT, int BM, int BN, int WM, int WN, int DEPTH, int TURNS>
hipError_t launch_out(const MatmulArgs& a, hipStream_t st) {
    if constexpr (BN / WN < 32) {                    // a wavefront has no 16 columns of either half
        if (a.half > 0) return hipErrorInvalidValue;
    } else {
        if (a.half > 0) return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, EIGHT, true, OUT, false>(a, st);
    }
    return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, EIGHT, false, OUT, false>(a, st);
}
template <bool EIGHT, typename OUT>
hipError_t launch_out_shape(const MatmulArgs& a, int shape, hipStream_t st) {
    switch (shape) {
        case MM_16x32_8: return launch_out<EIGHT, OUT, 16, 32, 1, 2, 3, 8>(a, st);
        case MM_32x32_8: return launch_out<EIGHT, OUT, 32, 32, 1, 2, 2, 8>(a, st);
        case MM_16x64_4: return launch_out<EIGHT, OUT, 16, 64, 1, 4, 3, 4>(a, st);
        case MM_32x64_2: return launch_out<EIGHT, OUT, 32, 64, 2, 2, 3, 2>(a, st);
        case MM_64x64: return launch_out<EIGHT, OUT, 64, 64, 2, 2, 4, 1>(a, st);
        case MM_64x64_2: return launch_out<EIGHT, OUT, 64, 64, 2, 2, 4, 2>(a, st);
        case MM_64x128: return launch_out<EIGHT, OUT, 64, 128, 2, 2, 3, 1>(a, st);
        case MM_64x128_2: return launch_out<EIGHT, OUT, 64, 128, 2, 2, 3, 2>(a, st);
        case MM_64x256: return launch_out<EIGHT, OUT, 64, 256, 2, 4, 3, 1>(a, st);
        case MM_128x128: return launch_out<EIGHT, OUT, 128, 128, 2, 2, 2, 1>(a, st);
        case MM_128x128_2: return launch_out<EIGHT, OUT, 128, 128, 2, 2, 2, 2>(a, st);
        case MM_128x256: return launch_out<EIGHT, OUT, 128, 256, 2, 4, 3, 1>(a, st);
        case MM_256x256: return launch_out<EIGHT, OUT, 256, 256, 2, 4, 2, 1>(a, st);
        default: return hipErrorInvalidValue;
    }
}

// Into codes: tiles with whole blocks of 128 columns of y
template <bool EIGHT, int BM, int BN, int WM, int WN, int DEPTH, int TURNS>
hipError_t launch_codes(const MatmulArgs& a, hipStream_t st) {
    if constexpr (BN >= 2 * kBlockCols) {
        if (a.half > 0) return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, EIGHT, true, float, true>(a, st);
    }
    if constexpr (BN == kBlockCols || BM >= 64) {
        if (a.half == 0) return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, EIGHT, false, float, true>(a, st);
    }
    return hipErrorInvalidValue;
}
template <bool EIGHT>
hipError_t launch_codes_shape(const MatmulArgs& a, int shape, hipStream_t st) {
    switch (shape) {
        case MM_16x128_4: return launch_codes<EIGHT, 16, 128, 1, 4, 2, 4>(a, st);
        case MM_32x128_2: return launch_codes<EIGHT, 32, 128, 1, 4, 3, 2>(a, st);
        case MM_16x256: return launch_codes<EIGHT, 16, 256, 1, 8, 4, 1>(a, st);
        case MM_32x256: return launch_codes<EIGHT, 32, 256, 1, 8, 4, 1>(a, st);
        case MM_64x128: return launch_codes<EIGHT, 64, 128, 2, 2, 3, 1>(a, st);
        case MM_64x128_2: return launch_codes<EIGHT, 64, 128, 2, 2, 3, 2>(a, st);
        case MM_64x256: return launch_codes<EIGHT, 64, 256, 2, 4, 3, 1>(a, st);
        case MM_128x128: return launch_codes<EIGHT, 128, 128, 2, 2, 2, 1>(a, st);
        case MM_128x128_2: return launch_codes<EIGHT, 128, 128, 2, 2, 2, 2>(a, st);
        case MM_128x256: return launch_codes<EIGHT, 128, 256, 2, 4, 3, 1>(a, st);
        case MM_256x256: return launch_codes<EIGHT, 256, 256, 2, 4, 2, 1>(a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

}  // namespace hr
