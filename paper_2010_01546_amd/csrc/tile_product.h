#pragma once
// Products of two matrices on the matrix cores, for bfloat16 entries (float32 sums) and 8-bit integers (32-bit integer sums), with an
// epilogue of the caller's:  C[r][c] = sum_k A[r][k] B[c][k].
//
// A workgroup of four wavefronts owns a tile of 64 NRT x 64 NCT results, a wavefront 32 NRT x 32 NCT of them in accumulation registers
// (v_mfma_f32_32x32x16_bf16 or v_mfma_i32_32x32x32_i8).  The contraction goes by in stages of 64 bytes of every row of the two
// panels; a ring of stages lies in LDS, filled by loads that go there directly, one barrier per stage, and the fragment reads of the next
// stage and the loads of a later one are placed between the matrix instructions of this one.
//
// An operand lies in memory in one of two ways.
//   Rows along the contraction (k contiguous): a stage holds 64 bytes of each row, four chunks of 16; chunk c of row r lies at
//     c ^ (r / 4 % 4), which spreads the 16 lanes that read together over all banks.
//   Contraction-major (bfloat16; a row of memory is one k): a stage holds 32 k of all the panel's columns and is turned as it is read
//     (ds_read_b64_tr_b16: 16 lanes get 4 k of a column each out of 4 x 16 entries).  The chunks of row k are permuted by 4 (k % 4) (panels
//     of 64 columns: 4 (k / 2 % 2)), so that the four rows read together fall into different banks.  No transposed copy is made.
// Where the contraction ends inside a stage, the loads past the end fetch a zero (in both operands: 0 x NaN is NaN).  Rows or columns past
// the edge are clamped; they feed results that the epilogue does not store.
//
// Few tiles: the contraction is cut into runs over more workgroups; these leave their sums in a workspace, in the order of the accumulation
// registers, and a second launch adds them in order and applies the epilogue.
#include "fw_internal.h"
#include <type_traits>

namespace fw {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

static __device__ uint4 tile_zero;          // 16 bytes of zeros, never written

struct TileProduct {
    const char *a, *b0, *b1;      // operands; b1: a second matrix, of the same tile's other columns (PAIR) or of the contraction's second part
    long long apitch, bpitch;     // bytes between rows in memory
    int R, C;                     // results; PAIR: C columns of each matrix
    int chunks;                   // 16-byte chunks of a row (operands along the contraction)
    int klen;                     // k of a part (contraction-major operands)
    int part, stages;             // stages of the first part, stages in all
    int nrb, ncb, tiles, runs, spr;
    int nrt, nct;                 // tile shape
    void* partial;
};

// Tiles in bands of eight rows of tiles, column by column inside a band: the 32 tiles that an XCD works on at a time share eight row
// panels and four column panels.
__device__ __forceinline__ void tile_at(const TileProduct& g, int tile, int& I, int& J) {
    const int band = tile / (8 * g.ncb), h = min(8, g.nrb - 8 * band), in = tile - band * 8 * g.ncb;
    J = in / h;
    I = 8 * band + in - J * h;
}

template <int I, int N, class F> __device__ __forceinline__ void static_for(const F& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        static_for<I + 1, N>(f);
    }
}

template <int NRT, int NCT> constexpr int tile_stages() { return NRT + NCT >= 8 ? 5 : NRT + NCT == 6 ? 3 : 4; }

// PAIR: the panel of B holds columns of b0 and the same columns of b1; tiles tb and tb + NCT / 2 of a wavefront belong together.
template <bool I8, int NRT, int NCT, bool AKM, bool BKM, bool PAIR, class Epi>
__global__ __launch_bounds__(256, NRT + NCT >= 8 ? 1 : 2) void tile_product_kernel(TileProduct g, Epi epi) {
    constexpr int NST = tile_stages<NRT, NCT>(), NF = NRT + NCT, STAGE = 4096 * NF, NM = NRT * NCT;
    using Acc = typename std::conditional<I8, intx16, floatx16>::type;
    __shared__ __align__(1024) char lds[NST][STAGE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave >> 1, wj = wave & 1;
    const int half = lane >> 5, l32 = lane & 31;
    // workgroups go to the 8 XCDs in turn: each XCD gets a contiguous run of tiles
    const int total = g.tiles * g.runs, per_xcd = (total + 7) / 8;
    int tile = ((int)blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3);
    if (tile >= total || ((int)blockIdx.x >> 3) >= per_xcd) return;
    const int run = __builtin_amdgcn_readfirstlane(tile / g.tiles);
    tile -= run * g.tiles;
    int I, J;
    tile_at(g, tile, I, J);
    I = __builtin_amdgcn_readfirstlane(I); J = __builtin_amdgcn_readfirstlane(J);
    const int c0 = run * g.spr, cend = min(c0 + g.spr, g.stages);

    // what this lane brings: of each panel a wavefront loads 1 KB pieces wave, wave + 4, ...
    const char* src[NF];
    int lim[NF];                               // stages (of a part) below which the chunk lies inside the contraction
    auto along = [&](const char* base, long long pitch, int row, int rows, int k) {
        const int c = (lane & 3) ^ ((lane >> 4) & 3);
        src[k] = base + (long long)min(row, rows - 1) * pitch + 16 * c;
        lim[k] = (g.chunks - c + 3) >> 2;
    };
    auto major = [&](auto NT, const char* base, long long pitch, int tile0, int cols, int piece, int k) {
        constexpr int CH = 8 * decltype(NT)::value;              // chunks of a row of the panel
        const int kr = piece * (64 / CH) + lane / CH, p = lane % CH;
        const int c = p ^ (CH > 8 ? 4 * (kr & 3) : 4 * ((kr >> 1) & 1));
        src[k] = base + kr * pitch + 16ll * min(tile0 * CH + c, (cols + 7) / 8 - 1);
        lim[k] = (g.klen - kr + 31) >> 5;
    };
#pragma unroll
    for (int k = 0; k < NRT; ++k) {
        const int piece = wave + 4 * k;
        if constexpr (AKM) major(std::integral_constant<int, NRT>(), g.a, g.apitch, I, g.R, piece, k);
        else along(g.a, g.apitch, I * 64 * NRT + 16 * piece + (lane >> 2), g.R, k);
    }
#pragma unroll
    for (int k = 0; k < NCT; ++k) {
        const int piece = wave + 4 * k;
        if constexpr (BKM) major(std::integral_constant<int, NCT>(), g.b0, g.bpitch, J, g.C, piece, NRT + k);
        else if constexpr (PAIR) {
            const int pr = 16 * piece, w = pr % (32 * NCT);
            const int col = J * 32 * NCT + pr / (32 * NCT) * 16 * NCT + w % (16 * NCT) + (lane >> 2);
            along(w >= 16 * NCT ? g.b1 : g.b0, g.bpitch, col, g.C, NRT + k);
        } else along(g.b0, g.bpitch, J * 64 * NCT + 16 * piece + (lane >> 2), g.C, NRT + k);
    }
    const long long second = BKM ? g.b1 - g.b0 : 0;
    auto load_one = [&](int buf, int c, int k) {                 // k is a constant after unrolling
        const bool two = BKM && c >= g.part;
        const int cc = two ? c - g.part : c;
        long long off;
        if (k < NRT) off = AKM ? (long long)c * 32 * g.apitch : (long long)c * 64;
        else off = BKM ? (long long)cc * 32 * g.bpitch + (two ? second : 0) : (long long)c * 64;
        const bool inside = c < cend && ((k < NRT && !AKM) || !BKM ? c : cc) < lim[k];
        const void* from = inside ? (const void*)(src[k] + off) : (const void*)&tile_zero;
        dma16(from, &lds[buf][1024 * (wave + 4 * (k < NRT ? k : k - NRT)) + (k < NRT ? 0 : 4096 * NRT)]);
    };

    Acc acc[NRT][NCT];
#pragma unroll
    for (int a = 0; a < NRT; ++a)
#pragma unroll
        for (int b = 0; b < NCT; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0;

    // fragments of a stage: f = kk NF + (tile of A, then tile of B), kk the half of the stage's contraction
    intx4 fr[2][2 * NF];
    const int at = l32 * 64, sw = (l32 >> 2) & 3, j = lane & 15;
    const int small = 2 * ((lane >> 4) & 1) + ((j >> 1) & 1);
    auto read_one = [&](int buf, int set, int f) {
        const int kk = f / NF, r = f % NF;
        const bool isa = r < NRT;
        const int t = isa ? wi * NRT + r : wj * NCT + r - NRT;
        const char* panel = &lds[buf][isa ? 0 : 4096 * NRT];
        if (isa ? AKM : BKM) {
            const int nt = isa ? NRT : NCT, rowb = 128 * nt;
            const int ch = 4 * (nt > 1 ? t ^ (j >> 2) : t ^ (j >> 3)) + small;
            const char* p = panel + (16 * kk + 8 * half + (j >> 2)) * rowb + 16 * ch + 8 * (j & 1);
            typedef __attribute__((address_space(3))) shortx4* lp;
            union { shortx4 h[2]; intx4 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * rowb));
            fr[set][f] = u.v;
        } else {
            fr[set][f] = *reinterpret_cast<const intx4*>(panel + t * 2048 + at + 16 * ((2 * kk + half) ^ sw));
        }
    };
    auto multiply_one = [&](int set, int m) {
        const int kk = m / NM, ta = (m % NM) / NCT, tb = m % NCT;
        if constexpr (I8)
            acc[ta][tb] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fr[set][kk * NF + ta], fr[set][kk * NF + NRT + tb], acc[ta][tb], 0, 0, 0);
        else
            acc[ta][tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fr[set][kk * NF + ta]),
                                                                  __builtin_bit_cast(bf16x8, fr[set][kk * NF + NRT + tb]), acc[ta][tb], 0, 0, 0);
    };

    // The loads of a wavefront complete in order: "at most those of NST - 2 stages outstanding" means that the stage before them has
    // landed for it, the barrier extends that to all four.  At the barrier of a stage every wavefront holds that stage's fragments in
    // registers, so its buffer is free for the stage NST further on.  Every turn issues the same number of loads (past the end they fetch
    // zeros), which keeps the count valid.
#pragma unroll
    for (int i = 0; i < NST - 1; ++i)
#pragma unroll
        for (int k = 0; k < NF; ++k) load_one(i, c0 + i, k);
    FW_WAIT_VM((NST - 2) * NF);
    __builtin_amdgcn_s_barrier();
    FW_COMPILER_FENCE();
#pragma unroll
    for (int k = 0; k < NF; ++k) load_one(NST - 1, c0 + NST - 1, k);
#pragma unroll
    for (int f = 0; f < 2 * NF; ++f) read_one(0, 0, f);
    int sc = 0;
    auto turn = [&](int c, auto SET) {
        constexpr int set = decltype(SET)::value;
        const int sn = sc == NST - 1 ? 0 : sc + 1;
        FW_WAIT_LGKM0();
        FW_WAIT_VM((NST - 2) * NF);
        __builtin_amdgcn_s_barrier();
        FW_COMPILER_FENCE();
        // reads of the next stage first, then the loads, spread over the matrix instructions
        constexpr int OPS = 3 * NF;
#pragma unroll
        for (int m = 0; m < 2 * NM; ++m) {
#pragma unroll
            for (int o = m * OPS / (2 * NM); o < (m + 1) * OPS / (2 * NM); ++o) {
                if (o < 2 * NF) read_one(sn, set ^ 1, o);
                else load_one(sc, c + NST, o - 2 * NF);
            }
            multiply_one(set, m);
            __builtin_amdgcn_sched_barrier(0);
        }
        sc = sn;
    };
    int c = c0;
    for (; c + 1 < cend; c += 2) {
        turn(c, std::integral_constant<int, 0>());
        turn(c + 1, std::integral_constant<int, 1>());
    }
    if (c < cend) turn(c, std::integral_constant<int, 0>());
    FW_WAIT_VM(0);
    FW_WAIT_LGKM0();

    if (g.runs > 1) {
        typedef typename std::conditional<I8, int4, float4>::type Quad;
        Quad* out = reinterpret_cast<Quad*>(g.partial) + ((size_t)run * g.tiles + tile) * (NM * 4 * 256) + tid;
#pragma unroll
        for (int ta = 0; ta < NRT; ++ta)
#pragma unroll
            for (int tb = 0; tb < NCT; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    Quad q = {acc[ta][tb][4 * i], acc[ta][tb][4 * i + 1], acc[ta][tb][4 * i + 2], acc[ta][tb][4 * i + 3]};
                    out[((ta * NCT + tb) * 4 + i) * 256] = q;
                }
        return;
    }
    const int col = PAIR ? J * 32 * NCT + 16 * NCT * wj : J * 64 * NCT + 32 * NCT * wj;
    static_for<0, NRT>([&](auto TA) {
        constexpr int ta = decltype(TA)::value;
        epi.template apply<NCT>(I * 64 * NRT + 32 * NRT * wi + 32 * ta + 4 * half, col + l32, acc[ta]);
    });
}

// adds the runs of a tile's row of 32 x 32 results, in order, and applies the epilogue
template <bool I8, int NRT, int NCT, bool PAIR, class Epi>
__global__ __launch_bounds__(256) void tile_runs_kernel(TileProduct g, Epi epi) {
    using Acc = typename std::conditional<I8, intx16, floatx16>::type;
    typedef typename std::conditional<I8, int4, float4>::type Quad;
    const int tile = blockIdx.x / NRT, ta = blockIdx.x % NRT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wi = wave >> 1, wj = wave & 1, half = lane >> 5, l32 = lane & 31;
    int I, J;
    tile_at(g, tile, I, J);
    Acc acc[NCT];
    const Quad* in = reinterpret_cast<const Quad*>(g.partial) + (size_t)tile * (NRT * NCT * 4 * 256) + (size_t)ta * NCT * 4 * 256 + tid;
    for (int z = 0; z < g.runs; ++z) {
#pragma unroll
        for (int tb = 0; tb < NCT; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Quad q = in[(size_t)z * g.tiles * (NRT * NCT * 4 * 256) + (tb * 4 + i) * 256];
                if (z == 0) { acc[tb][4 * i] = q.x; acc[tb][4 * i + 1] = q.y; acc[tb][4 * i + 2] = q.z; acc[tb][4 * i + 3] = q.w; }
                else { acc[tb][4 * i] += q.x; acc[tb][4 * i + 1] += q.y; acc[tb][4 * i + 2] += q.z; acc[tb][4 * i + 3] += q.w; }
            }
    }
    const int col = PAIR ? J * 32 * NCT + 16 * NCT * wj : J * 64 * NCT + 32 * NCT * wj;
    epi.template apply<NCT>(I * 64 * NRT + 32 * NRT * wi + 32 * ta + 4 * half, col + l32, acc);
}

// row of accumulation register i, for the first row that `apply` is given
__device__ __forceinline__ int tile_row(int row0, int i) { return row0 + 8 * (i >> 2) + (i & 3); }

// Tile shape and runs of the least estimated time in cycles: rounds of 256 workgroups x (stages of a run + filling the ring) x the longer
// of a stage's matrix instructions (32 cycles each) and its loads (about 40 bytes per cycle and compute unit), plus the pass that adds
// the runs.  A run keeps at least 8 stages.
inline void tile_plan(TileProduct& g, bool pair) {
    static const int shapes[][2] = {{4, 4}, {2, 4}, {2, 2}, {1, 4}, {1, 2}};
    double best = 1e300;
    for (const auto& s : shapes) {
        const int nrt = s[0], nct = s[1], tc = pair ? 32 * nct : 64 * nct;
        const int nrb = (g.R + 64 * nrt - 1) / (64 * nrt), ncb = (g.C + tc - 1) / tc;
        const long long tiles = (long long)nrb * ncb;
        const double t_mfma = 64.0 * nrt * nct + 40.0, t_load = (nrt + nct) * 4096.0 / 40.0, t_stage = t_mfma > t_load ? t_mfma : t_load;
        for (int runs = 1; runs <= 32 && (runs == 1 || (tiles * runs <= 512 && g.stages / runs >= 8)); ++runs) {
            const int spr = (g.stages + runs - 1) / runs, n = (g.stages + spr - 1) / spr;
            double cost = (double)((tiles * n + 255) / 256) * (spr + 6.0) * t_stage;
            if (n > 1) cost += 6000.0 + 2.0 * n * tiles * (nrt * nct * 16384.0) / 4e12 * 2.1e9;
            if (cost < best * 0.999) {
                best = cost;
                g.nrt = nrt; g.nct = nct; g.nrb = nrb; g.ncb = ncb; g.tiles = (int)tiles; g.runs = n; g.spr = spr;
            }
        }
    }
}
inline size_t tile_partial_bytes(const TileProduct& g) {
    return g.runs > 1 ? align_up((size_t)g.runs * g.tiles * g.nrt * g.nct * 16384, 256) : 0;
}

template <bool I8, int NRT, int NCT, bool AKM, bool BKM, bool PAIR, class Epi>
fw_status tile_launch(const TileProduct& g, const Epi& epi, hipStream_t st) {
    const long long total = (long long)g.tiles * g.runs;
    if (total > (1 << 30)) return FW_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((tile_product_kernel<I8, NRT, NCT, AKM, BKM, PAIR, Epi>), dim3((unsigned)((total + 7) / 8 * 8)), dim3(256), 0, st, g, epi);
    FW_LAUNCH_CHECK();
    if (g.runs > 1) {
        hipLaunchKernelGGL((tile_runs_kernel<I8, NRT, NCT, PAIR, Epi>), dim3((unsigned)(g.tiles * NRT)), dim3(256), 0, st, g, epi);
        FW_LAUNCH_CHECK();
    }
    return FW_OK;
}

template <bool I8, bool AKM, bool BKM, bool PAIR, class Epi>
fw_status tile_product(const TileProduct& g, const Epi& epi, hipStream_t st) {
    if (g.nrt == 4) return tile_launch<I8, 4, 4, AKM, BKM, PAIR>(g, epi, st);
    if (g.nrt == 2 && g.nct == 4) return tile_launch<I8, 2, 4, AKM, BKM, PAIR>(g, epi, st);
    if (g.nrt == 2) return tile_launch<I8, 2, 2, AKM, BKM, PAIR>(g, epi, st);
    if (g.nct == 4) return tile_launch<I8, 1, 4, AKM, BKM, PAIR>(g, epi, st);
    return tile_launch<I8, 1, 2, AKM, BKM, PAIR>(g, epi, st);
}

}  // namespace fw
