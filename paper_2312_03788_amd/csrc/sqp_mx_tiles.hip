// Microscaled product in tiles: 32x32x64 scaled matrix instructions on operands that lie in shared memory as they do in memory.
// Bound: the matrix cores.
//
// A workgroup of W = 4 or 8 waves takes BM rows x BN columns, a wave 32 RT x 32 CT of them (weights are the instruction's rows, activations
// its columns, so that a lane's results are neighbouring columns of y).  K goes in stages of 128 bytes of activations (256 k of e2m1, 128 of
// e4m3) through SLOTS slots, filled by direct loads into shared memory ahead of time; pieces of 16 bytes change places within 256 bytes, so
// that the sixteen rows that are read at once lie in different banks (operands are read without a conflict; the conflicts that the counters show, 27 to
// 31 % of the shared memory's cycles, are those of the scales, a word or less each from rows 16 or 32 bytes apart: without these reads they are 3 to
// 6 %, the results' way out, and a launch takes the same time).  Stages of 64 bytes of a row are slower (2048 x 8192 x 8192, e2m1, four
// slots: 89 us instead of 76): every load asks for twice as many lines, and asking for them is what the loads take.
// The order of blocks within a stage is free as long as both operands and their scales have the same: lane half h takes blocks
// STEPS h + s in step s, so that its scales lie together.  Of e4m3 activations a lane's first 16 values belong to the lower half's block and the
// others to the upper half's (the instruction's order).
// Scales come 16 (512 k) of a row at a time, by direct loads too where rows of them begin at words, else through registers.  Every row's are a
// line of their own: 4 % of the bytes, but a third of the lines asked for (256 x 256).  Where shared memory has room for it they come 32 at a
// time: per 512 k the 256 x 256 tile (e2m1) takes 3.4 us instead of 3.5, 64 x 8192 x 8192 (e4m3) 24.9 us instead of 26.6, 32 x 8192 x 8192 (e2m1) 19.0
// instead of 21.3.
//
// Measured: 2048 x 8192 x 8192 in whole rounds of 256 x 256, 62.5 us with e2m1 activations (4.4 PFLOP/s; a loop of the instruction alone
// reaches 7.2), 94 with e4m3 (2.9; 4.3).  What is left out of a 512 k step of 3.45 us shows what it waits for: without the copies of codes 2.76,
// without those of scales 3.17, all tiles from the same rows, so that every line is in the caches, 3.46: it is the copies' way through the
// compute unit, not memory.  128 x 128 (e4m3), in the same order: 1.81, 1.31, 1.56, 1.86; a slot more 1.85, stages of twice the length 1.80,
// operands fetched as early as can be the same.  Between idle gaps the same code is 15 % quicker: the power limit has its part.
#include <algorithm>
#include <type_traits>

#include "sqp_mx_gemm.h"

namespace {

typedef int rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ rsrc_t buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return rsrc_t{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)bytes, 0x00020000};
}

// 16 bytes per lane from base + (lane_offset | past) + offset to shared memory at dst + 16 lane; beyond the buffer: zeros.  In assembly, since
// the compiler would wait for it at the next read of shared memory; the kernel waits itself.  (The address is put together between the write of
// m0 and the load, which have to be an instruction apart.)  STREAM: with the hint for data that is read once.
template <bool STREAM>
__device__ __forceinline__ void copy_piece(rsrc_t base, uint32_t lane_offset, uint32_t past, uint32_t offset, uint32_t dst, uint32_t dst_more)
{
    uint32_t at;
#define SQP_COPY_PIECE(hint)                                                                                                        \
    asm volatile("s_add_u32 m0, %1, %2\n\tv_or_b32 %0, %3, %4\n\tbuffer_load_dwordx4 %0, %5, %6 offen " hint "lds"                \
                 : "=&v"(at)                                                                                                        \
                 : "s"(dst), "i"(dst_more), "v"(lane_offset), "v"(past), "s"(base), "s"(offset)                                    \
                 : "memory", "scc")
    if constexpr (STREAM) SQP_COPY_PIECE("nt ");
    else SQP_COPY_PIECE("");
#undef SQP_COPY_PIECE
}

constexpr int XCDS = 8;

// Workgroup w of `total`: its place when every XCD has one run of consecutive places.
__device__ __forceinline__ uint32_t xcd_run(uint32_t w, uint32_t total)
{
    const uint32_t xcd = w % XCDS, len = total / XCDS, more = total % XCDS;
    return xcd * len + (xcd < more ? xcd : more) + w / XCDS;
}

template <int XT, int RT, int CT, int WM, int WN, int BLK, int SLOTS, int SC>
struct Tile {
    static constexpr bool FOUR = XT == SQP_E2M1;
    static constexpr int BM = 32 * RT * WM, BN = 32 * CT * WN, W = WM * WN, THREADS = 64 * W;
    static constexpr int BLOCKS = BLK, STEPS = BLOCKS / 2;              // of 32 k per stage, of two blocks
    static constexpr int SPC = 16 / BLOCKS;                             // stages per chunk of 16 scales
    static constexpr int XB = (FOUR ? 16 : 32) * BLOCKS, WB = 16 * BLOCKS;  // bytes of a row per stage
    static constexpr int XCOPIES = BM * XB / 1024, COPIES = XCOPIES + BN * WB / 1024;  // of 1 KB per stage
    static constexpr int PER = (COPIES + W - 1) / W;                    // per wave
    static constexpr int SBM = (BM + 63) / 64 * 64;                     // rows of activations' scales (copies are of 64 rows or 32)
    static constexpr int HALVES = SC == 32 ? 2 : 1, SROW = 16 * HALVES; // chunks of 512 k, and bytes of a row, that scales are loaded for at once
    static constexpr int STAGE = COPIES * 1024, SCALES = (SBM + BN) * SROW;
    static constexpr int SCOPIES = SCALES / 1024, SPER = (SCOPIES + W * HALVES - 1) / (W * HALVES);  // of scales, per wave and 512 k (SC != 0)
    static constexpr int YOUNGER = (SPC - 1) * PER;                     // copies of codes, at least, that are issued between scales and the meeting before their use
    static constexpr int LDS = SLOTS * STAGE + 2 * SCALES;
    static_assert(LDS <= 160 * 1024 && (XB < 256 || (COPIES % 4 == 0 && XCOPIES % 4 == 0 && W % 4 == 0)), "shared memory; the same piece in all of a wave's copies");
};

template <int XT, int RT, int CT, int WM, int WN, int BLK, int SLOTS, int SC>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(WM * WN == 8 || RT * CT < 8 ? 2 : 1)))
mx_tiles_kernel(const SqpMxGemm a, int tiles_m, int tiles_n, int group_m, int chunks_per_part)
{
    typedef Tile<XT, RT, CT, WM, WN, BLK, SLOTS, SC> T;
    constexpr bool FOUR = T::FOUR, DIRECT = SC != 0;
    constexpr int XFMT = FOUR ? 4 : 0, BM = T::BM, BN = T::BN, XB = T::XB, WB = T::WB, STEPS = T::STEPS, BLOCKS = T::BLOCKS, SPC = T::SPC;
    constexpr int AHEAD = (SLOTS - 2) * T::PER;     // copies that may be under way when the waves meet
    constexpr int W = T::W, SROWS = (BM + BN + T::THREADS - 1) / T::THREADS;  // waves; rows of scales per thread
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::LDS];

    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    const int blocks = a.K / SQP_MX_BLOCK;
    // the tile: groups of group_m rows of tiles, row index fastest
    int m0, n0;
    {
        const uint32_t i = xcd_run(blockIdx.x, gridDim.x), g = i / (uint32_t)(group_m * tiles_n), in = i - g * (uint32_t)(group_m * tiles_n);
        const uint32_t rows = min((uint32_t)group_m, (uint32_t)tiles_m - g * group_m), col = in / rows;
        m0 = (int)(g * group_m + in - col * rows) * BM;
        n0 = a.first_col + (int)col * BN;
    }
    const int first = blockIdx.y * chunks_per_part, end = min((blocks + 15) / 16, first + chunks_per_part);  // chunks of 512 k

    const uint32_t x_row = (uint32_t)a.K / (FOUR ? 2 : 1), w_row = (uint32_t)a.K / 2;
    const rsrc_t xbuf = buffer_of(a.x, (uint32_t)a.M * x_row), wbuf = buffer_of(a.w, (uint32_t)a.N * w_row);
    const uint32_t base = (uint32_t)(size_t)&lds[0];
    // A wave's copies: every W-th of a stage's, the activations' first (where they are no whole number of W, some are made
    // twice, so that every wave has as many to wait for).  A copy is 4 rows of 256 bytes, 8 of 128 or 16 of 64: this lane's row and piece of it
    // (the same in all of a wave's copies, which are even numbers of copies apart, or fours).
    uint32_t off[T::PER];
    auto is_x = [&](int i) { return T::XCOPIES % W == 0 && T::COPIES % W == 0 ? W * i < T::XCOPIES : (wave + W * i) % T::COPIES < T::XCOPIES; };
    static_assert(T::XCOPIES % 2 == 0 && T::COPIES % 2 == 0, "copies of a wave are all even or all odd");
    auto piece_of = [&](int bytes) {  // a row's pieces change places so that 256 bytes of neighbouring rows hold one piece of sixteen rows
        return bytes == 256 ? (lane & 15) ^ (4 * (wave & 3) + (lane >> 4)) : bytes == 128 ? (lane & 7) ^ (4 * (wave & 1) + (lane >> 4)) : (lane & 3) ^ (lane >> 4);
    };
    const int xpiece = piece_of(XB), wpiece = piece_of(WB);
    constexpr int XLINE = XB / 16, WLINE = WB / 16;  // pieces of a row
#pragma unroll
    for (int i = 0; i < T::PER; i++) {
        const int c = (wave + W * i) % T::COPIES;
        if (is_x(i)) off[i] = (uint32_t)min(m0 + (64 * c + lane) / XLINE, a.M - 1) * x_row + 16u * (uint32_t)xpiece;
        else off[i] = (uint32_t)min(n0 + (64 * (c - T::XCOPIES) + lane) / WLINE, a.N - 1) * w_row + 16u * (uint32_t)wpiece;
    }
    // A stage's copies; pieces past the end of K are taken from beyond the buffer (no tensor has 2^31 bytes; the scalar offset stays within
    // the row, so that they are beyond it whether or not the hardware's check counts that offset).
    uint32_t xpast = 0, wpast = 0, at_stage = 0;
    const uint32_t last_stage = (uint32_t)(blocks - 1) / BLOCKS;
    auto aim = [&](int stage) {
        const int left = blocks - BLOCKS * stage;
        at_stage = min((uint32_t)stage, last_stage);
        xpast = xpiece < (FOUR ? left : 2 * left) ? 0u : 0x80000000u;
        wpast = FOUR ? xpast : wpiece < left ? 0u : 0x80000000u;
    };
    const uint32_t wave_base = __builtin_amdgcn_readfirstlane(base + 1024u * (uint32_t)wave);
    // Weights of calls of few rows are read by one workgroup each (64 x 44032 x 8192: 55.0 us, 52.6 with the hint); where a stage takes half of
    // a line, the other half would be fetched again (16 rows of e4m3: 52.1, 59.5 with the hint).
    constexpr bool STREAM = BM <= 64 && WB == 128;
    auto copy = [&](uint32_t slot, int i) {
        const bool x = is_x(i);
        const uint32_t offset = at_stage * (x ? XB : WB), past = x ? xpast : wpast;
        if constexpr (T::COPIES % W == 0 && T::XCOPIES % W == 0) {
            if (STREAM && !x) copy_piece<true>(wbuf, off[i], past, offset, wave_base + slot, 1024u * (uint32_t)(W * i));
            else copy_piece<false>(x ? xbuf : wbuf, off[i], past, offset, wave_base + slot, 1024u * (uint32_t)(W * i));
        } else {
            copy_piece<false>(x ? xbuf : wbuf, off[i], past, offset, __builtin_amdgcn_readfirstlane(base + slot + 1024u * (uint32_t)((wave + W * i) % T::COPIES)), 0u);
        }
    };

    // Scales, 16 blocks of every row a chunk.  A chunk that ends early is read up to its end: what is wanted lies `by` further on.
    uint8_t *const s_s = lds + SLOTS * T::STAGE;
    // DIRECT: copied as the codes are, since rows of them begin at words.
    const rsrc_t xsbuf = buffer_of(a.xs, (uint32_t)a.M * (uint32_t)blocks), wsbuf = buffer_of(a.ws, (uint32_t)a.N * (uint32_t)blocks);
    // SC = 32: those of two chunks at once, by two lanes a row, each kept inside the row by itself; one half of the copies is made in either
    // of the two chunks before.  Rows 8 to 15 of 16 have their two in the other order, so that 16 rows lie in different banks.
    uint32_t soff[DIRECT ? T::SPER : 1], smore[DIRECT ? T::SPER : 1];  // of the first half, and how much further those of the second are
    auto scopy = [&](int i) { return (wave + W * i) % T::SCOPIES; };
    const uint32_t second = T::HALVES == 2 && ((lane ^ lane >> 4) & 1) ? ~0u : 0u;
    auto copy_scales = [&](int c, int i, uint32_t row) {  // of chunk c (and the one behind it)
        const int start = 16 * c, at = min(start, blocks - 16), k = scopy(i);
        const uint32_t dst = __builtin_amdgcn_readfirstlane(base + SLOTS * T::STAGE + ((c - first) / T::HALVES & 1) * T::SCALES + 1024u * (uint32_t)k);
        if constexpr (T::HALVES == 2) row += second & (uint32_t)(min(start + 16, blocks - 16) - at);
        copy_piece<false>(k < T::SBM * T::SROW / 1024 ? xsbuf : wsbuf, row, 0u, (uint32_t)at, dst, 0u);
    };
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < T::SPER; i++) {
            auto offset = [&](int k) {
                const int row = 64 / T::HALVES * scopy(k) + lane / T::HALVES;
                return (uint32_t)(row < T::SBM ? min(m0 + row, a.M - 1) : min(n0 + row - T::SBM, a.N - 1)) * (uint32_t)blocks;
            };
            soff[i] = offset(i);
            smore[i] = T::HALVES == 2 ? offset(i + T::SPER) - soff[i] : 0u;
        }
    }
    // Else through registers, a row or two per thread.
    u32x4 sv[SROWS];
    auto scale_row = [&](int i) {
        const int row = (int)threadIdx.x + T::THREADS * i;
        return row < BM ? a.xs + (size_t)min(m0 + row, a.M - 1) * blocks : a.ws + (size_t)min(n0 + row - BM, a.N - 1) * blocks;
    };
    auto load_first_scales = [&] {
#pragma unroll
        for (int i = 0; i < SROWS; i++) sv[i] = sqp_mx_load_scales(scale_row(i) + 16 * first, blocks - 16 * first);
    };
    // The chunks behind, without branches.  (Behind the last one something is read that is not used: the row's end, or where no row
    // has 16 scales the activations' first bytes.)
    const bool one_chunk = blocks < 16;
    auto load_scales = [&](int chunk) {
        const int at = one_chunk ? 0 : min(16 * chunk, blocks - 16);
#pragma unroll
        for (int i = 0; i < SROWS; i++) {
            u32x4 v;
            __builtin_memcpy(&v, (one_chunk ? (const uint8_t *)a.x : scale_row(i)) + at, 16);
            sv[i] = v;
        }
        return 16 * chunk - at;
    };
    auto store_scales = [&](int chunk, int by) {
#pragma unroll
        for (int i = 0; i < SROWS; i++) {
            const int row = (int)threadIdx.x + T::THREADS * i;
            if (SROWS * T::THREADS == BM + BN || row < BM + BN) *(u32x4 *)&s_s[(chunk & 1) * T::SCALES + 16 * (row < BM ? row : row + T::SBM - BM)] = sqp_mx_shift_down(sv[i], by);
        }
    };

    f32x16 acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < CT; j++) acc[i][j] = (f32x16)(0.f);

    const int xr = 32 * RT * wm + l32, wr = 32 * CT * wn + l32;  // this lane's row of the wave's first tile
    u32x4 xf[2][RT][FOUR ? 1 : 2], wf[2][CT];
    uint32_t xsc[RT], wsc[CT], next_xsc[RT], next_wsc[CT];
    // Operand n of a step: the weights' first, then the activations' (e4m3: two each).
    constexpr int OPERANDS = CT + RT * (FOUR ? 1 : 2);
    auto fetch = [&](uint32_t slot, int s, int to, int n) {
        auto place = [](int row, int piece, int bytes) { return piece ^ (bytes == 256 ? row & 15 : bytes == 128 ? row >> 1 & 7 : row >> 2 & 3); };
        if (n < CT) {
            wf[to][n] = *(const u32x4 *)(lds + slot + T::XCOPIES * 1024 + (wr + 32 * n) * WB + 16 * place(wr, STEPS * h + s, WB));
        } else {
            const int i = FOUR ? n - CT : (n - CT) / 2, half = FOUR ? 0 : (n - CT) % 2;
            xf[to][i][half] = *(const u32x4 *)(lds + slot + (xr + 32 * i) * XB + 16 * place(xr, FOUR ? STEPS * h + s : 2 * (STEPS * half + s) + h, XB));
        }
    };
    auto fetch_scale = [&](int chunk, int u, int n) {  // of stage u of the chunk
        int at = u * BLOCKS + STEPS * h, buf = chunk & 1;
        // (a block past the end has zeros for codes, and some scale of its own row, so that no other row's NaN gets there)
        if constexpr (DIRECT) {
            at = min(at + max(16 * chunk - (blocks - 16), 0), 16 - STEPS);
            buf = (chunk - first) / T::HALVES & 1;
            if constexpr (T::HALVES == 2) at += 16 * (((chunk - first) ^ l32 >> 3) & 1);
        }
        const uint8_t *p = s_s + buf * T::SCALES + T::SROW * (n < CT ? T::SBM + wr + 32 * n : xr + 32 * (n - CT)) + at;
        const uint32_t v = STEPS == 4 ? *(const uint32_t *)p : *(const uint16_t *)p;
        if (n < CT) next_wsc[n] = v;
        else next_xsc[n - CT] = v;
    };

    // the first stages, and the first chunk's scales
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < T::SPER; i++) {
            copy_scales(first, i, soff[i]);
            if constexpr (T::HALVES == 2) copy_scales(first, i + T::SPER, soff[i] + smore[i]);
        }
    }
#pragma unroll
    for (int t = 0; t < SLOTS - 1; t++) {
        aim(first * SPC + t);
#pragma unroll
        for (int i = 0; i < T::PER; i++) copy(t * T::STAGE, i);
        if constexpr (!DIRECT)
            if (t == 0) {
                load_first_scales();
                store_scales(first, 0);
            }
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(AHEAD) : "memory");
#pragma unroll
    for (int n = 0; n < CT + RT; n++) fetch_scale(first, 0, n);
#pragma unroll
    for (int n = 0; n < OPERANDS; n++) fetch(0, 0, 0, n);
    constexpr int MEET = RT * CT >= 8 ? 1 : 0, LEFT = RT * CT - MEET;  // matrix instructions of a last step in front of the meeting, behind it
    constexpr int EARLY = LEFT * T::PER / (LEFT + RT * CT);            // copies issued behind the meeting
    aim(first * SPC + SLOTS - 1);
#pragma unroll
    for (int i = 0; i < EARLY; i++) copy((SLOTS - 1) * T::STAGE, i);

    // The order of instructions is fixed, and there are no branches (across one the compiler moves matrix instructions).  While a step's matrix
    // instructions run the next step's operands are fetched, and in a stage's first steps the copies of a stage to come are issued one by
    // one into the slot of the stage before: many at once would wait for each other, and the matrix instructions behind them.  In a
    // stage's last step, behind its first matrix instructions, the waves meet: then every read of this stage's slot has ended and the
    // next stage has landed.  (Behind the part's last stage copies and fetches are made all the same, and not used.)
    uint32_t slot = 0, free = (SLOTS - 1) * T::STAGE;
    for (int c = first; c < end; c++) {
        int by = 0;
        if constexpr (!DIRECT) by = load_scales(c + 1);
        auto stage = [&](auto u_) {
            constexpr int u = decltype(u_)::value;
            if constexpr (SLOTS == 2) {  // (known to the compiler)
                slot = u % 2 * T::STAGE;
                free = T::STAGE - slot;
            }
            const uint32_t next = slot == (SLOTS - 1) * T::STAGE ? 0u : slot + T::STAGE;
            // (the next chunk's scales: stored where few copies are under way, since the compiler waits for all of them)
            if constexpr (!DIRECT && SLOTS > 2 && u == SPC - 1) store_scales(c + 1, by);
#pragma unroll
            for (int i = 0; i < RT; i++) xsc[i] = next_xsc[i];
#pragma unroll
            for (int j = 0; j < CT; j++) wsc[j] = next_wsc[j];
            auto step = [&](auto s_) {
                constexpr int s = decltype(s_)::value;
                constexpr bool LAST = s + 1 == STEPS;
                constexpr int PF = (OPERANDS + (LAST ? LEFT : RT * CT) - 1) / (LAST ? LEFT : RT * CT);  // per matrix instruction: operands, scales
                constexpr int PS = (RT + CT + LEFT - 1) / LEFT;
                // (at a chunk's end the next one's scales have to be there too)
                constexpr int UNDER_WAY = DIRECT && u == SPC - 1 && AHEAD > T::YOUNGER ? T::YOUNGER : AHEAD;
                if constexpr (!DIRECT && SLOTS == 2 && LAST && u == SPC - 1) store_scales(c + 1, by);
                if constexpr (LAST) aim(c * SPC + u + SLOTS);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < RT * CT; q++) {
                    const int i = q / CT, j = q % CT;
                    i32x8 b;
                    if constexpr (FOUR) b = sqp_mx_operand(xf[s & 1][i][0]);
                    else b = sqp_mx_operand(xf[s & 1][i][0], xf[s & 1][i][FOUR ? 0 : 1]);
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(sqp_mx_operand(wf[s & 1][j]), b, acc[i][j], 4, XFMT, s, (int)wsc[j], s, (int)xsc[i]);
                    __builtin_amdgcn_sched_barrier(0);
                    const int at = LAST ? q - MEET : q;
                    if (LAST && q == MEET) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(UNDER_WAY) : "memory");
                    if (at >= 0) {
#pragma unroll
                        for (int n = at * PF; n < (at + 1) * PF; n++)
                            if (n < OPERANDS) fetch(LAST ? next : slot, LAST ? 0 : s + 1, (s + 1) & 1, n);
                        if constexpr (LAST) {
#pragma unroll
                            for (int n = at * PS; n < (at + 1) * PS; n++)
                                if (n < RT + CT) fetch_scale(u == SPC - 1 ? c + 1 : c, (u + 1) % SPC, n);
                        }
                    }
                    // the next chunk's scales
                    if constexpr (DIRECT && u == 0 && s == 0) {
#pragma unroll
                        for (int n = q; n < T::SPER; n += RT * CT) {
                            const int odd = T::HALVES == 2 ? (c - first) & 1 : 0;
                            copy_scales(c - odd + T::HALVES, n + T::SPER * odd, soff[n] + (smore[n] & (uint32_t)-odd));
                        }
                    }
                    // a stage's copies: behind the meeting before it, and in its first step
                    if constexpr (LAST || s == 0) {
                        constexpr int OVER = LEFT + RT * CT;
                        const int p = LAST ? at : LEFT + q;
                        if (p >= 0) {
#pragma unroll
                            for (int n = p * T::PER / OVER; n < (p + 1) * T::PER / OVER; n++) copy(LAST ? slot : free, n);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            step(std::integral_constant<int, 0>());
            step(std::integral_constant<int, 1>());
            if constexpr (STEPS > 2) {
                step(std::integral_constant<int, 2>());
                step(std::integral_constant<int, 3>());
            }
            free = slot;
            slot = next;
        };
        stage(std::integral_constant<int, 0>());
        stage(std::integral_constant<int, 1>());
        if constexpr (SPC > 2) {
            stage(std::integral_constant<int, 2>());
            stage(std::integral_constant<int, 3>());
        }
    }
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");  // (no copy may arrive any more: the slots are used again below)

    // result register r of tile (i, j): row 32 i + l32, columns 32 j + 8 (r >> 2) + 4 h + (r & 3)
    if (a.part) {
#pragma unroll
        for (int i = 0; i < RT; i++) {
            const int m = m0 + xr + 32 * i;
#pragma unroll
            for (int j = 0; j < CT; j++)
#pragma unroll
                for (int r4 = 0; r4 < 4; r4++) {
                    const int n = n0 + 32 * CT * wn + 32 * j + 8 * r4 + 4 * h;
                    if (m < a.M && n < a.N)
                        *(f32x4 *)(a.part + ((size_t)blockIdx.y * a.M + m) * a.N + n) = f32x4{acc[i][j][4 * r4], acc[i][j][4 * r4 + 1], acc[i][j][4 * r4 + 2], acc[i][j][4 * r4 + 3]};
                }
        }
        return;
    }
    // Through shared memory (a wave's own part of it), so that rows leave in pieces of 16 bytes side by side.
    const int cols = 32 * CT >> a.silu, pitch = 2 * 32 * CT + 16;
    uint8_t *const mine = lds + wave * 32 * pitch;
    const int out_n = a.N >> a.silu, n_first = (n0 + 32 * CT * wn) >> a.silu;
#pragma unroll
    for (int i = 0; i < RT; i++) {
#pragma unroll
        for (int j = 0; j < CT; j++)
#pragma unroll
            for (int r4 = 0; r4 < 4; r4++) {
                const f32x4 v = {acc[i][j][4 * r4], acc[i][j][4 * r4 + 1], acc[i][j][4 * r4 + 2], acc[i][j][4 * r4 + 3]};
                const int col = 32 * j + 8 * r4 + 4 * h;
                if (a.silu) *(uint32_t *)(mine + l32 * pitch + col) = sqp_half2(sqp_silu(v.x) * v.y, sqp_silu(v.z) * v.w);
                else *(uint2 *)(mine + l32 * pitch + 2 * col) = make_uint2(sqp_half2(v.x, v.y), sqp_half2(v.z, v.w));
            }
        for (int u = lane; u < 4 * cols; u += 64) {  // 32 rows of cols / 8 pieces
            const int row = u / (cols / 8), p = u % (cols / 8), m = m0 + 32 * RT * wm + 32 * i + row, n = n_first + 8 * p;
            const uint4 v = *(const uint4 *)(mine + row * pitch + 16 * p);
            if (m < a.M && n < out_n) *(uint4 *)(a.y + (size_t)m * out_n + n) = v;
        }
    }
}

// The K parts' sums joined, in their order.
__global__ void __launch_bounds__(256) mx_join_kernel(const SqpMxGemm a, int parts)
{
    const long n4 = a.N / 4, all = a.M * n4, i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    f32x4 s = ((const f32x4 *)a.part)[i];
    for (int p = 1; p < parts; p++) s += ((const f32x4 *)a.part)[i + p * all];
    sqp_mx_store4(a, (int)(i / n4), 4 * (int)(i % n4), s);
}

template <int XT, int RT, int CT, int WM, int WN, int BLK, int SLOTS, int SC>
int launch(const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t st)
{
    typedef Tile<XT, RT, CT, WM, WN, BLK, SLOTS, SC> T;
    if (SC != 0 && (a.K % 128 || a.K < 512)) return SQP_ERR_SHAPE;  // (the plan takes another tile)
    const int tm = (a.M + T::BM - 1) / T::BM, tn = (a.cols + T::BN - 1) / T::BN;
    const int chunks = (a.K + 511) / 512, per = (chunks + p.parts - 1) / p.parts, parts = (chunks + per - 1) / per;
    if ((long)tm * tn > 0x7fffffffL || parts > 65535) return SQP_ERR_SHAPE;
    SqpMxGemm b = a;
    if (parts == 1) b.part = nullptr;
    const dim3 grid((unsigned)(tm * tn), (unsigned)parts);
    mx_tiles_kernel<XT, RT, CT, WM, WN, BLK, SLOTS, SC><<<grid, T::THREADS, 0, st>>>(b, tm, tn, std::min(tm, 4), per);
    if (parts > 1) mx_join_kernel<<<(unsigned)(((long)a.M * (a.N / 4) + 255) / 256), 256, 0, st>>>(b, parts);
    return sqp_launch_status();
}

template <int XT>
int pick(const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t st)
{
    constexpr bool FOUR = XT == SQP_E2M1;
    // 256 x 256 asks for the fewest bytes per product, but fills the compute units only in whole rounds of 256; the plan knows what each costs.  Of 128 x 128
    // there are two: short slots with two workgroups per compute unit for many tiles (700 x 22016 x 4096, e4m3: 75.8 us, 82.1 deep), deep slots for
    // up to one round (512 x 8192 x 8192, e2m1: 23.7 us, 28.2).
    // (waves' tiles, waves; blocks per stage of e4m3 activations; slots, and scales of a row per copy, for either type)
#define TILE(i, RT, CT, WM, WN, BLK8, SLOTS4, SC4, SLOTS8, SC8)                                                                                            \
    static_assert(SQP_MX_TILE[i].rows == 32 * RT * WM && SQP_MX_TILE[i].cols == 32 * CT * WN && SQP_MX_TILE[i].direct == (SC4 != 0), "the tile's shape"); \
    if (p.tile == i) return launch<XT, RT, CT, WM, WN, FOUR ? 8 : BLK8, FOUR ? SLOTS4 : SLOTS8, FOUR ? SC4 : SC8>(p, a, st)
    TILE(0, 4, 2, 2, 4, 4, 2, 32, 3, 16);
    TILE(1, 2, 4, 2, 2, 4, 3, 16, 4, 32);
    TILE(2, 2, 2, 2, 2, 4, 2, 32, 3, 16);
    TILE(3, 2, 2, 2, 2, 4, 4, 32, 5, 32);
    TILE(4, 2, 1, 1, 4, 8, 3, 16, 4, 32);
    TILE(5, 1, 1, 1, 4, 8, 3, 32, 3, 16);
    TILE(6, 1, 1, 1, 2, 4, 3, 16, 3, 16);
    TILE(7, 2, 2, 2, 2, 4, 2, 0, 3, 0);
#undef TILE
    return SQP_ERR_SHAPE;
}

}  // namespace

int sqp_mx_tiles(int x_type, const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t st)
{
    return x_type == SQP_E2M1 ? pick<SQP_E2M1>(p, a, st) : pick<SQP_E4M3>(p, a, st);
}
