// Products with block-scaled weights for many rows: rows travel memory -> LDS in a ring of stages, weights memory ->
// registers, both as the matrix instruction takes them.
#include <type_traits>
#include "async_lds.h"
#include "mx_gemm.h"

namespace fate {

constexpr int kTileStages = 4;

// 16 bytes per lane from the lane's own address to lds + lane * 16.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_load16_at(uint32_t lds, const void* vaddr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds), "v"(vaddr) : "memory", "m0");
}
#pragma clang diagnostic pop

// A workgroup of four waves multiplies up to RT rows with 256 rows of weights, 64 (four tile rows) per wave; UP: 32 of W1
// and the same 32 of W3, so that a wave holds what SwiGLU and the block's scale need.
// Rows lie in LDS as [RT][8 pieces of 16 columns], piece c of row r at place c ^ (r & 7): the 16 lanes that read one
// piece of 16 rows at a time find them on different banks.
template <int RT, bool UP, int BITS>
__device__ __forceinline__ void tile_body(const MxArgs& a, const MxItem& it, const MxMatrix& m, uint8_t* lds) {
    constexpr int NT = RT / 16;                                   // row tiles of 16
    constexpr int NL = RT >= 32 ? RT / 32 : 1;                    // loads of rows per wave and stage
    constexpr int LPS = NL + 1;
    constexpr int D = RT >= 128 || BITS == 8 ? 2 : 4;             // weight tiles in flight per tile row
    const int lane = (int)(threadIdx.x & 63), g = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const bool shared = it.group >= a.E;
    const int Kp = shared ? a.Kp_s : a.Kp_r, KT = m.KT;
    const long long out0 = shared ? (long long)(it.group - a.E) * a.N + it.row0 : it.row0;
    uint8_t* xl = lds;                                            // [stages][RT * 128]
    uint8_t* sl = lds + kTileStages * RT * kMxStep;               // [stages][RT * 4]
    auto source = [&](int r) -> long long {
        r = r < it.rows ? r : 0;
        if (shared) return a.gather ? it.row0 + r : out0 + r;
        return a.gather ? a.perm[it.row0 + r] / a.k : it.row0 + r;
    };
    const uint8_t* xp[NL];
    constexpr int kPer = RT * 8 / 4;                              // pieces per wave
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int q = wave * kPer + i * 64 + (lane < kPer ? lane : 0);
        const int r = q >> 3, c = (q & 7) ^ (r & 7);
        xp[i] = (shared ? a.x_s : a.x_r) + source(r) * Kp + c * 16;
    }
    const uint8_t* sp = (shared ? a.xs_s : a.xs_r) + source(wave * (RT / 4) + (lane & (RT / 4 - 1))) * (Kp / 32);
    const uint32_t xl0 = lds_offset(xl) + wave * kPer * 16, sl0 = lds_offset(sl) + wave * RT;
    auto issue = [&](int s) {
        const uint32_t st = (uint32_t)(s & (kTileStages - 1));
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (kPer >= 64 || lane < kPer) lds_load16_at(xl0 + st * (RT * kMxStep) + i * 1024, xp[i] + s * kMxStep);
        }
        if (lane < RT / 4) lds_load4(sl0 + st * (RT * 4), sp + s * 4);
    };
    issue(0);
    if (KT > 1) issue(1);
    if (KT > 2) issue(2);

    const int last = mx_row_tiles(m.rows) - 1;
    const uint8_t* w[4];
    const uint32_t* ws[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int rb = UP ? it.col * 8 + wave * 2 + (i & 1) : it.col * 16 + wave * 4 + i;
        rb = rb < last ? rb : last;
        w[i] = (UP && i >= 2 ? m.w3 : m.w) + (long long)rb * KT * MxWTile<BITS>::kBytes;
        ws[i] = reinterpret_cast<const uint32_t*>((UP && i >= 2 ? m.s3 : m.s) + (long long)rb * m.KG * 256) + lane;
    }
    MxWTile<BITS> wt[D][4];
    uint32_t sc[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sn[i] = ws[i][0];
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            wt[d][i].load(w[i] + (long long)(d < KT ? d : KT - 1) * MxWTile<BITS>::kBytes, lane);

    v4f acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    const uint8_t* xr = xl + (lane & 15) * kMxStep;
    const int c0 = (g ^ (lane & 7)) * 16, c1 = ((4 + g) ^ (lane & 7)) * 16;
    const uint8_t* sr = sl + (lane & 15) * 4 + g;

    for (int kg = 0; kg < m.KG; ++kg) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sc[i] = sn[i];
            sn[i] = ws[i][(kg + 1 < m.KG ? kg + 1 : kg) * 64];
        }
        auto step = [&](auto J) {
            constexpr int j = decltype(J)::value;
            const int s = kg * 4 + j;
            if (s < KT) {
                wait_stages<LPS, 2>(KT - 1 - s);                  // stage s has landed (this wave's part of it)
                lds_only_barrier();                               // everyone's part; stage s - 1 is read
                if (s + 3 < KT) issue(s + 3);
                const uint8_t* xs = xr + j * (RT * kMxStep);
                const uint8_t* ss = sr + j * (RT * 4);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const v4i lo = *reinterpret_cast<const v4i*>(xs + t * 16 * kMxStep + c0);
                    const v4i hi = *reinterpret_cast<const v4i*>(xs + t * 16 * kMxStep + c1);
                    const v8i x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    const uint32_t e = ss[t * 64];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][i] = wt[j % D][i].template mfma<j>(sc[i], x, e, acc[t][i]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    wt[j % D][i].load(w[i] + (long long)(s + D < KT ? s + D : KT - 1) * MxWTile<BITS>::kBytes, lane);
            }
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    }

    const long long ld = shared ? a.ld_s : a.ld_r;
    if constexpr (UP) {
        const int n0 = it.col * 128 + wave * 32;
        const bool zero = n0 >= m.rows;                           // padding columns of h
        uint8_t* y = static_cast<uint8_t*>(shared ? a.y_s : a.y_r);
        uint8_t* ys = shared ? a.ys_s : a.ys_r;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = t * 16 + (lane & 15);
            v4f h0, h1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h0[i] = zero ? 0.0f : mx_swiglu(acc[t][0][i], acc[t][2][i]);
                h1[i] = zero ? 0.0f : mx_swiglu(acc[t][1][i], acc[t][3][i]);
            }
            const long long row = out0 + r;
            mx_store_h(h0, h1, r < it.rows, y + row * ld + n0, ys + row * (ld / 32) + n0 / 32);
        }
    } else {
        const int cols = shared ? a.cols_s : a.cols_r;
        void* y = shared ? a.y_s : a.y_r;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = t * 16 + (lane & 15);
            if (r < it.rows) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r0 = (it.col * 16 + wave * 4 + i) * 16 + 4 * g;
                    if (r0 < cols) {
                        v4f v = acc[t][i];
                        if (a.bias != nullptr) {
#pragma unroll
                            for (int b = 0; b < 4; ++b) v[b] += r0 + b < cols ? a.bias[r0 + b] : 0.0f;
                        }
                        mx_store_y(a, y, (out0 + r) * ld + r0, cols - r0, v);
                    }
                }
            }
        }
    }
}

// A group's last tile, and small groups, take the body for as many rows as they have.
template <int RT, bool UP, int BITS>
__device__ __forceinline__ void tile_by_rows(const MxArgs& a, const MxItem& it, const MxMatrix& m, uint8_t* lds) {
    if constexpr (RT > 16) {
        if (it.rows <= RT / 2) {
            tile_by_rows<RT / 2, UP, BITS>(a, it, m, lds);
            return;
        }
    }
    tile_body<RT, UP, BITS>(a, it, m, lds);
}

template <int RT, bool UP>
__global__ __launch_bounds__(256, 2) void mx_tile_kernel(MxArgs a, int cb_r, int cb_s) {
    extern __shared__ __align__(16) uint8_t lds[];
    const MxItem it = mx_find_item<RT, true>(a, cb_r, cb_s, (int)blockIdx.x);
    if (it.group < 0) return;
    MxMatrix m;
    if (!mx_matrix<UP>(a, it.group, &m)) {
        if constexpr (!UP) {                                      // an expert that cannot be used adds nothing
            const bool shared = it.group >= a.E;
            const int cols = shared ? a.cols_s : a.cols_r;
            const long long out0 = shared ? (long long)(it.group - a.E) * a.N + it.row0 : it.row0;
            for (int q = (int)threadIdx.x; q < it.rows * 64; q += 256) {
                const int r = q >> 6, r0 = it.col * 256 + (q & 63) * 4;
                if (r0 < cols)
                    mx_store_y(a, shared ? a.y_s : a.y_r, (out0 + r) * (shared ? a.ld_s : a.ld_r) + r0, cols - r0,
                               v4f{0.0f, 0.0f, 0.0f, 0.0f});
            }
        }
        return;
    }
    if (m.bits == 4) tile_by_rows<RT, UP, 4>(a, it, m, lds);
    else tile_by_rows<RT, UP, 8>(a, it, m, lds);
}

long long mx_max_tiles(const MxArgs& a, int RT);

template <int RT, bool UP>
static fate_status launch_tile(hipStream_t st, const MxArgs& a) {
    constexpr int width = UP ? 128 : 256;
    const int cb_r = (a.cols_r + width - 1) / width, cb_s = (a.cols_s + width - 1) / width;
    const long long items = mx_max_tiles(a, RT) * cb_r + (long long)a.n_shared * ((a.N + RT - 1) / RT) * cb_s;
    const long long grid = (items + 7) / 8 * 8;
    if (grid > 0x7fffffffLL) FATE_FAIL(FATE_ESHAPE, "too many workgroups (%lld)", grid);
    const size_t lds = (size_t)kTileStages * RT * (kMxStep + 4);
    if (lds > 64 * 1024)
        FATE_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(mx_tile_kernel<RT, UP>),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    mx_tile_kernel<RT, UP><<<(unsigned)grid, 256, lds, st>>>(a, cb_r, cb_s);
    FATE_HIP(hipGetLastError());
    return FATE_OK;
}

// rows: of an average group.
template <bool UP>
static fate_status launch_by_rows(hipStream_t st, const MxArgs& a, long long rows) {
    if (rows <= 16) return launch_tile<16, UP>(st, a);
    if (rows <= 32) return launch_tile<32, UP>(st, a);
    if (rows <= 64) return launch_tile<64, UP>(st, a);
    return launch_tile<128, UP>(st, a);
}

fate_status launch_mx_tile(hipStream_t st, const MxArgs& a, bool up, long long rows) {
    return up ? launch_by_rows<true>(st, a, rows) : launch_by_rows<false>(st, a, rows);
}

}  // namespace fate
