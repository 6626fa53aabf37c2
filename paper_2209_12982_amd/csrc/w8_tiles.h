// Many rows times 8-bit weights: tiles of outputs, operands through LDS.
//
// The matrix cores bound it.  Weights are the first operand of mfma 32x32x32 (the form that reaches their full rate), x the
// second; a wave has WN x WM blocks of 32 x 32.  Stages of BK bytes of k are copied from memory straight to LDS, STAGES - 1
// ahead; the copies fill LDS densely, so the 16-byte pieces of a row are exchanged (swap) such that sixteen rows' reads of
// the same piece fall into the sixteen columns of the 256-byte banks.  Within 32 rows of weights the copy puts row
// 16 h + 4 q + e where operand row 8 q + 4 h + e is read: a lane's sixteen sums are then neighbouring outputs of one row.
//
// Measured: 8192 rows by 16384 x 4096 480 to 490 us, 2.25 to 2.29 POP/s, at the 1.6 to 1.7 GHz that the load leaves of the
// clock, the matrix cores 58% of the cycles; 2048 by 4096 x 16384 133 to 137 us, 2.01 to 2.07 POP/s; 48 by 16384 x 4096 13.2 us,
// bound by the weights' bytes.
#pragma once
#include <type_traits>

#include "w8_device.h"

namespace w8 {

template <int N> using Int = std::integral_constant<int, N>;

template <int WN_, int WM_, int GN_, int GM_, int GK_, int BK_, int STAGES_> struct Tile {
    static constexpr int WN = WN_, WM = WM_, GN = GN_, GM = GM_, GK = GK_, BK = BK_, STAGES = STAGES_;
    static constexpr int kWaves = GN * GM * GK, kThreads = 64 * kWaves;
    static constexpr int kOuts = 32 * WN * GN, kRows = 32 * WM * GM;        // of a workgroup
    static constexpr int kRowPieces = BK / 16;
    static constexpr int kPiecesW = kOuts * kRowPieces / kThreads, kPiecesX = kRows * kRowPieces / kThreads;    // of a thread
    static constexpr int kBytesW = kOuts * BK, kBytes = kBytesW + kRows * BK;
    // The largest tiles leave a compute unit room for one workgroup: it takes tile after tile, and the next one's first stage
    // is on its way while results are stored.
    static constexpr bool kLoop = kOuts * kRows >= 65536;
    static constexpr int kSlots = 32;                       // compute units of an XCD
    static_assert(WN == 1 || WN == 2 || WN == 4, "rows of results are turned in whole sets of banks");
    static_assert(!kLoop || (STAGES == 2 && GK == 1), "results are turned in the second stage");
    static_assert(kOuts * kRowPieces % kThreads == 0 && kRows * kRowPieces % kThreads == 0, "whole copies");
    static __device__ int swap(int row) { return BK >= 256 ? row & 15 : (BK == 128 ? (row >> 1) & 7 : (row >> 2) & 3); }
};

// An address that all lanes have alike, in scalar registers.
__device__ inline const int8_t* uniform(const int8_t* p) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)p >> 32));
    return (const int8_t*)((uintptr_t)hi << 32 | lo);
}
// 16 bytes a lane from base + off to LDS at dst + 16 lane, which is on its way until vmcnt says otherwise; in assembly
// because the compiler would wait for all copies before each read of LDS.  A scalar base moves on from stage to stage
// without vector instructions, which take issue slots from the matrix products; that it is one is said here, where the
// instruction needs it, and not left to what the compiler makes of the additions before.
__device__ inline void copy16(const int8_t* base, uint32_t off, uint32_t dst) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(uniform(base)), "{m0}"(dst) : "memory");
}
__device__ inline void copy16_from(const void* from, uint32_t dst) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(dst) : "memory");
}

// The same value, which the compiler does not know to be so: what follows from it is worked out here, not kept in registers
// over the whole kernel.
__device__ inline int anew(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// A tile: its rows (experts: places in the order), outputs, expert, stages of k, and the place of its sums in a.tail, or -1.
struct Where {
    int m0, m1, n0, expert, first, last, slot;
};

// The tiles of rows of 64 experts from e0 on: where a lane's expert has its rows, how many tiles, and how many up to it.
template <int ROWS> __device__ inline void count_tiles(const Args& a, int e0, int& begin, int& end, int& count, int& upto) {
    const int lane = threadIdx.x & 63;
    begin = 0, end = 0;
    if (e0 + lane < a.experts) rows_of(a, e0 + lane, begin, end);
    count = (end - begin + ROWS - 1) / ROWS;
    upto = count;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int other = __shfl_up(upto, s);
        if (lane >= s) upto += other;
    }
}

// The tiles of one XCD (workgroup i runs on XCD i % 8): a piece of the list of all.  An expert's tiles stand together there,
// those of the same outputs next to each other, so that weights stay in the XCD's L2 for all rows that need them; dense ones
// eight rows of tiles at a time.  Items are what workgroups take: the whole tiles, and parts of the last ones.
struct List {
    int begin, length, whole, parts, items;     // whole: tiles that are not cut
};
// In how many parts of k the last `rest` tiles of an XCD are cut, where these would leave half of its compute units idle.
__host__ __device__ inline int tail_parts(int rest, int stages) {
    int parts = rest > 0 ? 32 / rest : 1;
    parts = parts > kMostParts ? kMostParts : parts;
    return parts > stages / 4 ? stages / 4 : parts;
}
template <class S, bool EXPERTS> __device__ inline List list_of(const Args& a, int xcd, int n_tiles, int m_tiles) {
    int tiles = n_tiles * m_tiles;
    if (EXPERTS) {
        tiles = 0;
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            int begin, end, count, upto;
            count_tiles<S::kRows>(a, e0, begin, end, count, upto);
            tiles += __builtin_amdgcn_readlane(upto, 63);
        }
        tiles = min(tiles, m_tiles) * n_tiles;              // more only where ends are not in order
    }
    const int each = (tiles + 7) / 8;
    List l;
    l.begin = xcd * each;
    l.length = max(0, min(each, tiles - l.begin));
    l.whole = l.length, l.parts = 1;
    if (S::kLoop && a.tail) {
        const int rest = l.length % S::kSlots, parts = tail_parts(rest, (a.k + S::BK - 1) / S::BK);
        if (parts > 1) l.whole -= rest, l.parts = parts;
    }
    l.items = l.whole + (l.length - l.whole) * l.parts;
    return l;
}
// Tile `index` of all.
template <class S, bool EXPERTS> __device__ inline void locate(const Args& a, int index, int n_tiles, int m_tiles, Where& t) {
    t.expert = 0;
    if (!EXPERTS) {
        const int set = 8 * n_tiles, g = index / set, high = min(8, m_tiles - 8 * g), in = index - g * set;
        t.m0 = (8 * g + in % high) * S::kRows;
        t.n0 = in / high * S::kOuts;
        t.m1 = a.m;
        return;
    }
    t.m0 = t.m1 = t.n0 = 0;
    int before = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        int begin, end, count, upto;
        count_tiles<S::kRows>(a, e0, begin, end, count, upto);
        const uint64_t here = __ballot(index < min(before + upto, m_tiles) * n_tiles);
        if (here) {
            const int l = __builtin_ctzll(here), tiles = __builtin_amdgcn_readlane(count, l);
            const int in = index - (before + __builtin_amdgcn_readlane(upto, l) - tiles) * n_tiles;
            t.expert = e0 + l;
            t.m0 = __builtin_amdgcn_readlane(begin, l) + in % tiles * S::kRows;
            t.m1 = __builtin_amdgcn_readlane(end, l);
            t.n0 = in / tiles * S::kOuts;
            return;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
}

// FAR: rows of x whose distance from the first of a tile (experts: of x) does not fit 32 bits.
template <int TYPE, class S, bool EXPERTS, bool FAR = false>
__global__ __launch_bounds__(S::kThreads) void w8_tiles_kernel(Args a, int n_tiles, int m_tiles) {
    typedef typename Half<TYPE>::type T;
    typedef __attribute__((ext_vector_type(8))) T T8;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::STAGES][S::kBytes];
    constexpr int kSets = S::kLoop ? 2 : 1;
    __shared__ __attribute__((aligned(16))) float w_scale[kSets][S::kOuts], bias[kSets][S::kOuts], x_scale[kSets][S::kRows];
    __shared__ int out_row[kSets][S::kRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, half = lane >> 5;

    const List list = list_of<S, EXPERTS>(a, blockIdx.x % 8, n_tiles, m_tiles);
    const int all = (a.k + S::BK - 1) / S::BK;
    auto where = [&](int turn, Where& t) {
        const int item = (int)(blockIdx.x / 8) + turn * (int)(gridDim.x / 8);
        if (item >= list.items) return false;
        const int cut = list.length - list.whole, part = item < list.whole ? 0 : (item - list.whole) / cut;
        locate<S, EXPERTS>(a, list.begin + item - part * cut, n_tiles, m_tiles, t);
        t.first = 0, t.last = all, t.slot = -1;
        if (item >= list.whole) {
            const int steps = (all + list.parts - 1) / list.parts;
            t.first = min(part * steps, all);
            t.last = min(t.first + steps, all);
            t.slot = (int)(blockIdx.x % 8) * S::kSlots + item - list.whole;
        } else if (!EXPERTS && a.part) {
            t.first = (int)blockIdx.y * a.steps;
            t.last = min(t.first + a.steps, all);
        }
        for (int* v : {&t.m0, &t.m1, &t.n0, &t.expert, &t.first, &t.last, &t.slot}) *v = __builtin_amdgcn_readfirstlane(*v);
        return true;
    };
    Where t;
    if (!where(0, t)) return;

    auto load_scales = [&](const Where& t, int set) {
        for (int o = threadIdx.x; o < S::kOuts; o += S::kThreads) {
            const int col = min(t.n0 + o, a.n - 1);
            w_scale[set][o] = a.w_scales[(int64_t)t.expert * a.n + col];
            bias[set][o] = !EXPERTS && a.bias ? (float)((const T*)a.bias)[col] : 0.f;
        }
        for (int o = threadIdx.x; o < S::kRows; o += S::kThreads) {
            const int at = min(t.m0 + o, t.m1 - 1), route = EXPERTS ? a.order[at] : at;
            x_scale[set][o] = a.x_scales[EXPERTS ? x_row(a, route) : route];
            out_row[set][o] = t.m0 + o < t.m1 && (!EXPERTS || (uint32_t)route < (uint32_t)a.routes) ? route : -1;
        }
    };

    // pieces that this thread copies: where they come from, relative to the tile's weights and to x
    uint32_t from_w[S::kPiecesW], from_x[S::kPiecesX];
    int lane_s = lane;
    auto place = [&](int p, int& row, int& piece) {
        row = p / S::kRowPieces;
        piece = (p % S::kRowPieces) ^ S::swap(row);
    };
    const int8_t *w_base, *x_base;
    auto prepare = [&](const Where& t) {
        const int lane = anew(threadIdx.x & 63);
#pragma unroll
        for (int i = 0; i < S::kPiecesW; ++i) {
            int row, piece;
            place((i * S::kWaves + wave) * 64 + lane, row, piece);
            const int w_row = (row & ~31) | (row >> 2 & 1) << 4 | (row >> 3 & 3) << 2 | (row & 3);
            from_w[i] = (uint32_t)(min(t.n0 + w_row, a.n - 1) - t.n0) * (uint32_t)a.k + 16 * piece;
        }
#pragma unroll
        for (int i = 0; i < S::kPiecesX; ++i) {
            int row, piece;
            place((i * S::kWaves + wave) * 64 + lane, row, piece);
            const int at = min(t.m0 + row, t.m1 - 1);
            const int64_t row_x = EXPERTS ? x_row(a, a.order[at]) : at - t.m0;
            from_x[i] = FAR ? (uint32_t)row_x : (uint32_t)(row_x * a.x_stride) + 16 * piece;
        }
        w_base = uniform(a.w + ((int64_t)t.expert * a.n + t.n0) * a.k);
        x_base = uniform(a.x + (EXPERTS ? 0 : t.m0 * a.x_stride));
    };
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds[0][0] + wave * 1024;
    // Piece i of stage s on its way.  cut: the end of k lies inside the stage, what is behind it becomes 0.
    auto copy_piece = [&](int s, int buf, int i, bool cut) {
        const bool is_w = i < S::kPiecesW;
        const int j = is_w ? i : i - S::kPiecesW;
        const int8_t* base = (is_w ? w_base : x_base) + (int64_t)s * S::BK;
        int row, piece;
        place((j * S::kWaves + wave) * 64 + lane, row, piece);
        const auto off = [&]() -> std::conditional_t<FAR, int64_t, uint32_t> {
            if (is_w) return from_w[j];
            if constexpr (FAR) return from_x[j] * a.x_stride + 16 * piece;
            return from_x[j];
        }();
        const uint32_t dst = to + buf * S::kBytes + (is_w ? 0 : S::kBytesW) + j * (1024 * S::kWaves);
        if (!cut) {
            if constexpr (FAR)
                copy16_from(base + off, dst);
            else
                copy16(base, off, dst);
        } else {
            copy16_from(s * S::BK + 16 * piece < a.k ? base + off : (const int8_t*)kZeros, dst);
        }
    };
    constexpr int kPieces = S::kPiecesW + S::kPiecesX;
    auto copy = [&](int s, int buf) {
        if ((s + 1) * S::BK <= a.k) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) copy_piece(s, buf, i, false);
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) copy_piece(s, buf, i, true);
        }
    };

    i32x16 acc[S::WN][S::WM];
    const int wn = wave % S::GN, wm = wave / S::GN % S::GM, wk = wave / (S::GN * S::GM);
    constexpr int kSteps = S::BK / 32 / S::GK;              // of a wave
    i32x4 w[2][S::WN], x[2][S::WM];                         // operands of a step of 32 of k, and of the next one
    auto read = [&](int buf, int t, int to) {
        const uint8_t* lw = lds[buf] + (32 * S::WN * wn + c) * S::BK;
        const uint8_t* lx = lds[buf] + S::kBytesW + (32 * S::WM * wm + c) * S::BK;
        const int at = ((2 * (kSteps * wk + t) + half) ^ S::swap(c)) * 16;
#pragma unroll
        for (int i = 0; i < S::WN; ++i) w[to][i] = *(const i32x4*)(lw + i * (32 * S::BK) + at);
#pragma unroll
        for (int j = 0; j < S::WM; ++j) x[to][j] = *(const i32x4*)(lx + j * (32 * S::BK) + at);
    };
    bool busy;                                              // whether the wave has results; else it only copies
    auto multiply = [&](int from, int i) {
#pragma unroll
        for (int j = 0; j < S::WM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[from][i], x[from][j], acc[i][j], 0, 0, 0);
    };
    int buf, s;
    // Takes stage s.  Before its last step the next one has to have arrived, for all waves, with no more than `later` stages
    // on their way; all reads of this stage are done by then, so its buffer is filled again (FILL 1; 2: with the end of k).
    auto stage = [&](auto fill, auto later) __attribute__((always_inline)) {
        constexpr int FILL = decltype(fill)::value, LATER = decltype(later)::value;
        const int after = buf + 1 == S::STAGES ? 0 : buf + 1;
#pragma unroll
        for (int t = 0; t < kSteps - 1; ++t) {
            if (!busy) break;
            read(buf, t + 1, (t + 1) & 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < S::WN; ++i) multiply(t & 1, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (LATER >= 0) {
            WINO_WAIT_VM_LDS(LATER * kPieces);
            winof4::ring_barrier();
            if (busy) read(after, 0, kSteps & 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < S::WN; ++i) {
            if (busy) multiply((kSteps - 1) & 1, i);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (FILL != 0) {
#pragma unroll
                for (int p = i * kPieces / S::WN; p < (i + 1) * kPieces / S::WN; ++p) copy_piece(s + S::STAGES, buf, p, FILL == 2);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (kSteps & 1) {                         // the next stage begins with the first of the two sets
#pragma unroll
            for (int i = 0; i < S::WN; ++i) w[0][i] = w[1][i];
#pragma unroll
            for (int j = 0; j < S::WM; ++j) x[0][j] = x[1][j];
        }
        buf = after;
        ++s;
    };
    // All stages of a tile, whose first ones are on their way.
    auto run = [&](const Where& t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::WN; ++i)
#pragma unroll
            for (int j = 0; j < S::WM; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
        busy = t.m0 + 32 * S::WM * wm < t.m1 && t.n0 + 32 * S::WN * wn < a.n;
        const int last = t.last;
        buf = 0, s = t.first;
        if (s >= last) return;
        if (last - s >= S::STAGES)
            WINO_WAIT_VM_LDS((S::STAGES - 1) * kPieces);
        else
            WINO_WAIT_VM_LDS(0);
        winof4::ring_barrier();
        read(0, 0, 0);
        const int whole = min(last, a.k / S::BK);           // stages without the end of k
        while (s + S::STAGES < whole) stage(Int<1>(), Int<S::STAGES - 2>());
        if (s + S::STAGES < last) stage(Int<2>(), Int<S::STAGES - 2>());
        while (s + 1 < last) stage(Int<0>(), Int<0>());
        stage(Int<0>(), Int<-1>());
    };
    // All waves have done what they do in LDS; copies and stores stay on their way.
    auto meet = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        winof4::ring_barrier();
    };

    // 32 rows at a time, each wave turns its own results in LDS, so that neighbouring lanes store neighbouring bytes: up to 256
    // of a row.  The 16-byte pieces of a row are exchanged by the row's number: both ways sixteen lanes meet sixteen columns of
    // the banks.
    constexpr int kParts = S::GK > 1 ? (S::GK - 1) * S::GN * S::GM * S::WN * S::WM * 4096 : 0;
    constexpr int kTurn = 32 * (S::WN == 1 ? 128 : 256);    // bytes of a wave
    static_assert((S::kLoop ? S::kBytes : kParts) + S::GN * S::GM * kTurn <= S::STAGES * S::kBytes, "room to turn");
    uint8_t* mine = &lds[0][0] + (S::kLoop ? S::kBytes : kParts) + wave * kTurn;
    // Stores rows of BLOCKS times 32 results of type E; put(block, piece) gives the 16-byte pieces of this lane's half of them.
    auto turned = [&](const Where& t, int set, int j, int i0, auto blocks, auto* out, int64_t stride, auto put) __attribute__((always_inline)) {
        const int col0 = t.n0 + 32 * (S::WN * wn + i0);
        if (col0 >= a.n) return;
        typedef std::remove_reference_t<decltype(*out)> E;
        const int lane = lane_s, c = lane & 31, half = lane >> 5;
        constexpr int BLOCKS = decltype(blocks)::value, kBlock = 32 * (int)sizeof(E), kRow = BLOCKS * kBlock;
        static_assert(32 * kRow <= kTurn, "room");
        auto at = [&](int row, int byte) {
            const int swap = kRow == 256 ? row & 15 : (kRow == 128 ? (row >> 1) & 7 : (row >> 2) & 3);
            return mine + row * kRow + 16 * ((byte >> 4) ^ swap) + (byte & 15);
        };
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int p = 0; p < kBlock / 32; ++p) *(u32x4*)at(c, i * kBlock + half * (kBlock / 2) + 16 * p) = put(i0 + i, p);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int* to_row = out_row[set] + 32 * (S::WM * wm + j);
        // 16 bytes a lane at any alignment: a row of results may begin anywhere
        const int valid = (a.n - col0) * (int)sizeof(E);    // bytes of a row
#pragma unroll
        for (int i = 0; i < 32 * kRow / 1024; ++i) {
            const int p = 16 * (64 * i + lane), row = p / kRow, byte = p % kRow, r = to_row[row];
            const u32x4 v = *(const u32x4*)at(row, byte);
            if (r < 0 || byte >= valid) continue;
            uint8_t* to = (uint8_t*)(out + r * stride + col0) + byte;
            if (byte + 16 <= valid) {
                *(Anywhere*)to = v;
            } else {                                        // the end of a row
                typedef __attribute__((ext_vector_type(16 / sizeof(E)))) E Many;
                const Many all = __builtin_bit_cast(Many, v);
#pragma unroll
                for (int e = 0; e < 16 / (int)sizeof(E); ++e)
                    if (byte + (e + 1) * (int)sizeof(E) <= valid) ((E*)to)[e] = all[e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    auto store = [&](const Where& t, int set) __attribute__((always_inline)) {
        lane_s = anew(threadIdx.x & 63);
        if (S::kLoop && t.slot >= 0) {                      // sums of a part of k, as the lanes have them
            int32_t* to = a.tail + (int64_t)t.slot * (S::kOuts * S::kRows) + (wave * (S::WN * S::WM * 4) * 64 + lane_s) * 4;
#pragma unroll
            for (int i = 0; i < S::WN; ++i)
#pragma unroll
                for (int j = 0; j < S::WM; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *(i32x4*)(to + ((j * S::WN + i) * 4 + e) * 256) = i32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
            return;
        }
#pragma unroll
        for (int j = 0; j < S::WM; ++j) {
            const int c = lane_s & 31, half = lane_s >> 5;
            const float xs = x_scale[set][32 * (S::WM * wm + j) + c];
            auto results = [&](int i, int e, float (&y)[4]) {       // four neighbouring ones of block i
                const int o = 32 * (S::WN * wn + i) + 16 * half + e;
                const f32x4 sc = *(const f32x4*)(w_scale[set] + o), bi = *(const f32x4*)(bias[set] + o);
#pragma unroll
                for (int f = 0; f < 4; ++f) y[f] = finish(acc[i][j][e + f], xs, sc[f], bi[f]);
            };
            auto wide = [&](auto* out, int64_t stride, auto put) __attribute__((always_inline)) {  // 4 bytes each, 256 of a row at a time
                constexpr int kBlocks = S::WN < 2 ? S::WN : 2;
#pragma unroll
                for (int i = 0; i < S::WN; i += kBlocks) turned(t, set, j, i, Int<kBlocks>(), out, stride, put);
            };
            if (!EXPERTS && a.part) {
                wide(a.part + (int64_t)blockIdx.y * a.m * a.n, (int64_t)a.n, [&](int i, int p) {
                    const i32x16& z = acc[i][j];
                    return u32x4{(uint32_t)z[4 * p], (uint32_t)z[4 * p + 1], (uint32_t)z[4 * p + 2], (uint32_t)z[4 * p + 3]};
                });
            } else if (EXPERTS && a.products) {
                wide(a.products, (int64_t)a.n, [&](int i, int p) {
                    float y[4];
                    results(i, 4 * p, y);
                    return __builtin_bit_cast(u32x4, f32x4{y[0], y[1], y[2], y[3]});
                });
            } else {
                turned(t, set, j, 0, Int<S::WN>(), (T*)a.y, a.y_stride, [&](int i, int p) {
                    float y[4], z[4];
                    results(i, 8 * p, y);
                    results(i, 8 * p + 4, z);
                    return __builtin_bit_cast(u32x4, T8{(T)y[0], (T)y[1], (T)y[2], (T)y[3], (T)z[0], (T)z[1], (T)z[2], (T)z[3]});
                });
            }
        }
    };

    prepare(t);
#pragma unroll
    for (int i = 0; i < S::STAGES; ++i)
        if (t.first + i < t.last) copy(t.first + i, i);
    load_scales(t, 0);
    for (int turn = 0, set = 0;; ++turn, set ^= 1) {
        run(t);
        meet();                                             // nobody reads a stage any more, and the scales are there
        if constexpr (S::GK > 1) {                              // the parts of k meet
            typedef __attribute__((ext_vector_type(4))) int Sum;
            constexpr int kSums = S::WN * S::WM * 4;            // pieces of 16 bytes a lane
            static_assert((S::GK - 1) * S::GN * S::GM * kSums * 1024 <= S::STAGES * S::kBytes, "room for the parts");
            uint8_t* parts = &lds[0][0] + 16 * lane;
            if (wk > 0) {
#pragma unroll
                for (int p = 0; p < kSums; ++p) {
                    const i32x16& z = acc[p / 4 / S::WM][p / 4 % S::WM];
                    *(Sum*)(parts + ((wave - S::GN * S::GM) * kSums + p) * 1024) = Sum{z[p % 4 * 4], z[p % 4 * 4 + 1], z[p % 4 * 4 + 2], z[p % 4 * 4 + 3]};
                }
            }
            __syncthreads();
            if (wk > 0) return;
#pragma unroll
            for (int k = 0; k < S::GK - 1; ++k)
#pragma unroll
                for (int p = 0; p < kSums; ++p) {
                    const Sum v = *(const Sum*)(parts + ((wave + k * S::GN * S::GM) * kSums + p) * 1024);
                    i32x16& z = acc[p / 4 / S::WM][p / 4 % S::WM];
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[p % 4 * 4 + e] += v[e];
                }
        }
        Where next;
        const bool more = S::kLoop && where(turn + 1, next);
        if (more) {
            prepare(next);
            if (next.first < next.last) copy(next.first, 0);
            load_scales(next, set ^ 1);
        }
        store(t, set);
        if (!more) return;
        meet();                                             // results are turned, the second stage is free
        t = next;
        if (t.first + 1 < t.last) copy(t.first + 1, 1);
    }
}

// The results of tiles that were cut in parts of k: a wave for each block of 32 x 32, of a workgroup of four.  Memory bounds it:
// 4 bytes of each part a result.
template <int TYPE, class S, bool EXPERTS> __global__ __launch_bounds__(256) void w8_tail_kernel(Args a, int n_tiles, int m_tiles) {
    typedef typename Half<TYPE>::type T;
    typedef __attribute__((ext_vector_type(8))) T T8;
    constexpr int kUnits = S::kWaves * S::WM * S::WN;
    const int xcd = blockIdx.x % 8, own = blockIdx.x / 8 * 4 + (threadIdx.x >> 6), unit = own % kUnits, tile = own / kUnits;
    const List list = list_of<S, EXPERTS>(a, xcd, n_tiles, m_tiles);
    const int cut = list.length - list.whole;
    if (tile >= cut) return;
    Where t;
    locate<S, EXPERTS>(a, list.begin + list.whole + tile, n_tiles, m_tiles, t);
    const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
    const int wave = unit / (S::WM * S::WN), j = unit / S::WN % S::WM, i = unit % S::WN;
    const int at = t.m0 + 32 * (S::WM * (wave / S::GN) + j) + c, col = t.n0 + 32 * (S::WN * (wave % S::GN) + i) + 16 * half;
    const int32_t* from = a.tail + (int64_t)(xcd * S::kSlots + tile) * (S::kOuts * S::kRows) + (unit * 4 * 64 + lane) * 4;
    const int row = at >= t.m1 ? -1 : (EXPERTS ? a.order[at] : at);
    i32x4 sum[4] = {};
    for (int p = 0; p < list.parts; ++p, from += (int64_t)cut * (S::kOuts * S::kRows))
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += *(const i32x4*)(from + e * 256);
    if (row < 0 || col >= a.n || (EXPERTS && row >= a.routes)) return;
    const float xs = a.x_scales[EXPERTS ? x_row(a, row) : row];
    const float* ws = a.w_scales + (int64_t)t.expert * a.n + col;
    const bool whole = col + 16 <= a.n;
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const bool there = whole || col + e < a.n;
        const float bias = !EXPERTS && a.bias && there ? (float)((const T*)a.bias)[col + e] : 0.f;
        y[e] = finish(sum[e / 4][e % 4], xs, there ? ws[e] : 0.f, bias);
    }
    if (EXPERTS && a.products) {
        float* to = a.products + (int64_t)row * a.n + col;
        if (whole) {
#pragma unroll
            for (int e = 0; e < 16; e += 4) *(Anywhere*)(to + e) = __builtin_bit_cast(u32x4, f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]});
        } else {
            for (int e = 0; e < 16; ++e)
                if (col + e < a.n) to[e] = y[e];
        }
        return;
    }
    T* to = (T*)a.y + row * a.y_stride + col;
    if (whole) {
#pragma unroll
        for (int e = 0; e < 16; e += 8)
            *(Anywhere*)(to + e) = __builtin_bit_cast(u32x4, T8{(T)y[e], (T)y[e + 1], (T)y[e + 2], (T)y[e + 3], (T)y[e + 4], (T)y[e + 5], (T)y[e + 6], (T)y[e + 7]});
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (col + e < a.n) to[e] = (T)y[e];
    }
}

// The tiles that calls are cut into (outputs x rows of a workgroup).  128 x 128 comes twice: with four stages and a compute
// unit for itself, and with two stages and two to a compute unit, which suits more tiles than compute units.
typedef Tile<4, 2, 2, 4, 1, 128, 2> Tile256x256;
typedef Tile<2, 2, 2, 4, 1, 64, 3> Tile128x256;
typedef Tile<2, 1, 2, 4, 1, 128, 4> Tile128x128;
typedef Tile<2, 1, 2, 4, 1, 128, 2> Pair128x128;
typedef Tile<1, 1, 2, 4, 1, 128, 3> Tile64x128;
typedef Tile<1, 1, 2, 2, 1, 128, 3> Tile64x64;
typedef Tile<1, 1, 1, 1, 8, 256, 4> Tile32x32;
// Sums shared out to two or four waves: a compute unit that has one tile needs more waves than its blocks of 32 x 32 give (200
// rows by 4096 x 4096: 64 x 64 11.1 us, by twice the waves 9.2; 128 by 4096 x 8192, 64 x 32 by four times 12.1; 64 by 1024 x
// 8192: 32 x 32 by four waves 8.1, by the eight that it has above 7.0).
typedef Tile<1, 1, 2, 4, 2, 256, 3> Shared64x128;
typedef Tile<1, 1, 2, 2, 2, 256, 3> Shared64x64;
typedef Tile<1, 1, 2, 1, 4, 256, 4> Shared64x32;
// They, and rows alone (w8_rows.h): 16 outputs by 16 or 8 waves, 32 outputs by 4.
enum Kernel { kTile256x256, kTile128x256, kTile128x128, kPair128x128, kTile64x128, kTile64x64, kTile32x32, kShared64x128, kShared64x64, kShared64x32, kRows16, kRows16Few, kRows32, kKernels };

// Workgroups for so many tiles: as many for each XCD, one for each of 256 compute units where they go on.
template <class S> inline unsigned workgroups(const Args& a, int64_t tiles) {
    int64_t each = (tiles + 7) / 8;
    if (S::kLoop && a.tail) each = (each + S::kSlots - 1) / S::kSlots * S::kSlots;      // parts fill the last round at most
    return (unsigned)(8 * (S::kLoop && each > 32 ? 32 : each));
}
// Sums of the tiles that are cut: a tile for each compute unit at most.
constexpr size_t kTailBytes = (size_t)256 * 256 * 256 * sizeof(int32_t);
template <int TYPE, class S, bool EXPERTS> void launch_tail(const Args& a, int n_tiles, int m_tiles, hipStream_t stream) {
    if constexpr (S::kLoop)
        if (a.tail)
            hipLaunchKernelGGL((w8_tail_kernel<TYPE, S, EXPERTS>), dim3(8u * (S::kSlots / 2) * S::kWaves * S::WM * S::WN / 4), dim3(256), 0,
                               stream, a, n_tiles, m_tiles);
}

// Whether rows that far apart need the kernel for that, Tile64x128 with FAR.
inline bool far(int64_t rows, int64_t stride, int64_t k) { return (rows - 1) * stride + k > (int64_t)0xffffffff; }

// What a kernel takes (us): `start` beside the loop, `step` for 1024 of k, `step` times 1 + `full` with a workgroup on each
// of the 256 compute units (rows: with 16 rows), and `pair` times that for two workgroups each (0: not for so many).  Chosen
// for 900 measured calls of 1 to 8192 rows, 64 to 32768 outputs and k of 128 to 16384 such that the kernel of the shortest
// estimate is as near to the shortest measured one as they go: 1.6% longer on average, 37% at most.  Those
// whose sums are shared out, for 330 more: of 400 others 122 take them then, in 0.94 of the time without them on average, 0.77 to
// 1.17.  Of 440 others of 1 to 256 rows the choice is 1.3% longer than the shortest on average, 28% at most.
struct Form {
    int outs, rows;
    double start, step, pair, full;
};
constexpr Form kForms[kKernels] = {
    {256, 256, 12.7, 5.6, 1.73, 0.69}, {128, 256, 4.2, 4.3, 1.58, 0.98},
    {128, 128, 3.91, 2.27, 2.17, 0.78}, {128, 128, 3.14, 2.42, 1.3, 1.01}, {64, 128, 2.26, 1.67, 1.56, 0.7},
    {64, 64, 2.26, 1.58, 1.3, 0.38},    {32, 32, 2.32, 0.48, 1.24, 0.71},  {64, 128, 3.7, 1.13, 0, 0.62},
    {64, 64, 2.8, 1.2, 0, 0.19},        {64, 32, 2.94, 0.716, 0, 0.2},     {16, 16, 1.1, 0.32, 1.84, 1.37},
    {16, 16, 0.26, 0.424, 1.76, 1.16},  {32, 16, 0.46, 0.98, 1.5, 1.24},
};
// The time of a kernel that has so many tiles, for k of a part and so many bytes of weights; m: rows, of an expert or of all.
inline double estimate(Kernel kernel, int64_t tiles, int64_t k, int64_t bytes, int64_t m) {
    const Form& f = kForms[kernel];
    const int64_t rest = tiles % 512;
    const double rounds = f.pair * (double)(tiles / 512) + (rest == 0 ? 0 : (rest <= 256 ? 1 : f.pair));
    const double fill = kernel >= kRows16 ? (m < 16 ? (double)m / 16 : 1) : (tiles < 256 ? (double)tiles / 256 : 1);
    // Sixteen rows of 4096 bytes or a multiple lie in the same memory channels, and eight waves ask for half of them at a
    // time: one row by 4096 x 4096 5.5 us, by 16 waves 5.2; by 4096 x 4112 4.8 and 4.9.
    const double same = kernel == kRows16Few && k % 4096 == 0 ? 1.4 : 1;
    const double t = (f.start + same * f.step * (1 + f.full * fill) * (double)k / 1024) * rounds, memory = (double)bytes / 5.2e6;
    return t > memory ? t + 0.05 * memory : memory + 0.05 * t;      // what is less decides between equal ones
}
// What it gains (us) to cut the last of so many tiles of 256 x 256 in parts of k: a part of a round instead of a whole one, for
// a launch that reads their sums, 256 KB a part.  Measured without and with it: 4096 rows by 4608 x 14336 308 and 240 us, 2048
// by 2048 x 16384 148 and 80, 6144 by 4096 x 8192 191 and 189, 4096 by 5120 x 4096 99 both.
inline double tail_gain(int64_t tiles, int64_t k) {
    const Form& f = kForms[kTile256x256];
    const int rest = (int)((tiles + 7) / 8 % 32), parts = tail_parts(rest, (int)((k + 127) / 128));
    if (parts <= 1) return 0;
    const double whole = 1 + f.full * rest / 32, part = 1 + f.full * rest * parts / 32;
    return f.step * (whole - part / parts) * (double)k / 1024 - (4 + 0.5 * rest * parts);
}

}  // namespace w8
