// Weight gradient of a linear layer, dw[i][j] (+)= sum_t dy[t][i] x[t][j] (zpp.h),
// on the matrix cores.
//
// Both operands lie along features while the sum runs over tokens, and an MFMA
// lane wants eight tokens of one feature.  So each lane fetches 4 tokens by 8
// features, turns them in registers (byte permutes pair the tokens; a
// checkpoint's codes are scaled on the way, exactly) and lays them into LDS
// feature by feature, from where a lane reads its 16 bytes at once.
//
// 4096x18176x4544 from a checkpoint 628-640 us, 1057-1077 TFLOP/s, from bf16 575, 1176
// (the library's product of that layout, its result in bf16: 632).  Long sums are bound
// by a turn's steps one after the other more than by any one of them: of a turn's 3230
// clocks from bf16 (3790 from codes) the matrix cores are busy for 2048 and the LDS for
// 1280, nearly the whole together, and the conversion of codes comes on top; the clock
// under that load is 1.5 to 1.8 GHz.  Short sums are bound by writing dw (one token
// into 8192x8192: 43 us, 6.3 TB/s).
#include <math.h>

#include <initializer_list>
#include <type_traits>

#include "zpp_act8.h"

namespace zpp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kStep = 64;  // tokens a turn
// Elements between tokens up to which a turn's offsets (64 tokens of 2 bytes an
// element) are 32 bits; tokens further apart are fetched one by one.
constexpr size_t kNear = (size_t)1 << 24;

struct WeightGradArgs {
    Mat dy, x;
    float *dw;
    size_t dw_stride;
    float *parts;  // the workspace: [splits][tail tiles][tile][tile]
    size_t rows, split_rows;
    uint32_t n, k, tiles_n, tiles_k;
    uint32_t whole;   // tiles whose tokens one workgroup takes all
    uint32_t splits;  // of the tokens of the tiles after those
    int accumulate;
    int near;  // a turn's tokens lie within 32-bit offsets of each other
};

// 4 tokens by 8 features as fetched.
template <int TYPE>
struct Piece {
    Chunk<TYPE> t[4];
};

// One operand as a lane sees it: where its pieces start.  A piece that starts
// past the last feature takes the last chunk instead, and a chunk's elements
// past the row's end whatever is there: both only reach results that are not
// stored.
template <int TYPE>
struct Operand {
    const uint8_t *data;  // of token 0
    const uint8_t *exps;
    size_t pitch;         // bytes between tokens
    size_t span;          // bytes from the first element to past the last
    uint32_t blocks;      // exponents between tokens
    uint32_t col;         // the lane's bytes into a token
    uint32_t at, exp_at;  // its bytes and exponents past a turn's first token
    uint32_t block;       // its exponent's place in a token
    uint32_t margin;      // tokens before the matrix's end whose chunks may pass it
};

template <int TYPE>
__device__ __forceinline__ Operand<TYPE> operand(const Mat &m, size_t rows, uint32_t cols,
                                                 uint32_t col, uint32_t token) {
    constexpr uint32_t kSize = TYPE == kBf16 ? 2 : 1;
    Operand<TYPE> o;
    const uint32_t last = (cols - 1) / 8 * 8;
    col = col < last ? col : last;
    o.data = reinterpret_cast<const uint8_t *>(m.data);
    o.exps = m.exps;
    o.pitch = m.stride * kSize;
    o.span = (rows - 1) * o.pitch + cols * kSize;
    o.blocks = (cols + kActBlock - 1) / kActBlock;
    o.col = col * kSize;
    o.block = col / kActBlock;
    o.at = token * (uint32_t)o.pitch + o.col;
    o.exp_at = token * o.blocks + o.block;
    // the last chunk ends last + 8 - cols elements past its row
    o.margin = cols % 8 ? (uint32_t)((last + 8 - cols + m.stride - 1) / m.stride) : 0;
    return o;
}

// Memory from an address that is the same in all lanes: the address and the
// distance between tokens stay in scalar registers, and a lane adds its 32 bits.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t memory_at(const uint8_t *p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, -1, 0x00027000);
}

// A turn whose tokens all lie `margin` and more before the matrix's end: whole
// chunks, which end inside the matrix.
__device__ __forceinline__ void fetch(Piece<kBf16> &p, const Operand<kBf16> &o, size_t token) {
    const __amdgpu_buffer_rsrc_t m = memory_at(o.data + token * o.pitch);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        p.t[i].w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                 m, o.at, i * (uint32_t)o.pitch, 0));
}
__device__ __forceinline__ void fetch(Piece<kI8> &p, const Operand<kI8> &o, size_t token) {
    const __amdgpu_buffer_rsrc_t m = memory_at(o.data + token * o.pitch);
    const __amdgpu_buffer_rsrc_t e = memory_at(o.exps + token * o.blocks);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        p.t[i].codes = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(
                                                     m, o.at, i * (uint32_t)o.pitch, 0));
        p.t[i].exp = __builtin_amdgcn_raw_buffer_load_b8(e, o.exp_at, i * o.blocks, 0);
    }
}

// Bytes off .. off + size(V) of an operand, which may pass its end by less than
// that: the last whole vector before the end is loaded then, and moved down to
// its place (what fills up reaches only results that are not stored).  An
// operand smaller than one vector is loaded byte by byte.
template <class V, int A>
__device__ __forceinline__ V load_inside(const uint8_t *p, size_t off, size_t span) {
    constexpr size_t kSize = sizeof(V);
    V v = {};
    if (__builtin_expect(span < kSize, 0)) {
        for (size_t b = off; b < span; ++b)
            v[(b - off) / 4] |= (uint32_t)p[b] << (8 * ((b - off) % 4));
        return v;
    }
    const uint32_t over = off + kSize > span ? (uint32_t)(off + kSize - span) : 0;
    v = ld_at<V, A>(p + (off - over));
    uint64_t w[kSize / 8 + 1] = {};
    __builtin_memcpy(w, &v, kSize);
    const uint32_t shift = 8 * (over % 8);
#pragma unroll
    for (uint32_t i = 0; i < kSize / 8; ++i) {
        if (kSize > 8 && over >= 8)
            w[i] = w[i + 1];
    }
#pragma unroll
    for (uint32_t i = 0; i < kSize / 8; ++i)
        w[i] = shift ? w[i] >> shift | w[i + 1] << (64 - shift) : w[i];
    __builtin_memcpy(&v, w, kSize);
    return v;
}
__device__ __forceinline__ void fetch_token(Chunk<kBf16> &c, const Operand<kBf16> &o, size_t token,
                                            bool inside) {
    const size_t off = token * o.pitch + o.col;
    c.w = inside ? ld_at<u32x4, 2>(o.data + off) : load_inside<u32x4, 2>(o.data, off, o.span);
}
__device__ __forceinline__ void fetch_token(Chunk<kI8> &c, const Operand<kI8> &o, size_t token,
                                            bool inside) {
    const size_t off = token * o.pitch + o.col;
    c.codes = inside ? ld_at<u32x2, 1>(o.data + off) : load_inside<u32x2, 1>(o.data, off, o.span);
    c.exp = o.exps[token * o.blocks + o.block];
}

// A turn at the end: tokens from `end` on are zeros.  `token`: the lane's first.
template <int TYPE>
__device__ __forceinline__ void fetch_end(Piece<TYPE> &p, const Operand<TYPE> &o, size_t token,
                                          size_t end, size_t rows) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        p.t[i] = Chunk<TYPE>{};
        if (token + i < end)
            fetch_token(p.t[i], o, token + i, token + i + o.margin < rows);
    }
}

// Codes are kept whole until they are laid into LDS: the compiler cut them apart
// at their load, and waited for it there (4096x18176x4544: 790 us, 661 so).
__device__ __forceinline__ void hold_piece(Piece<kBf16> &) {}
__device__ __forceinline__ void hold_piece(Piece<kI8> &p) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        hold(p.t[i]);
}

// Feature e of a piece with its four tokens side by side, as bf16.
__device__ __forceinline__ u32x2 turned(const Piece<kBf16> &p, int e, const float (&)[4]) {
    const uint32_t sel = e % 2 ? 0x07060302u : 0x05040100u;
    return u32x2{__builtin_amdgcn_perm(p.t[1].w[e / 2], p.t[0].w[e / 2], sel),
                 __builtin_amdgcn_perm(p.t[3].w[e / 2], p.t[2].w[e / 2], sel)};
}
// code * 2^e is a bf16 number: its high half is all of it.
__device__ __forceinline__ u32x2 turned(const Piece<kI8> &p, int e, const float (&scale)[4]) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] =
            __float_as_uint((float)(int8_t)(p.t[i].codes[e / 4] >> (8 * (e % 4))) * scale[i]);
    return u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u),
                 __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
}

// LDS holds a tile as [feature][64 tokens] bf16, 128 bytes a feature, in 16-byte
// units of 8 tokens.  Unit u of feature f lies at place u ^ key(f), the key made
// of f's low three bits, its bits 3 and 4 and the tile's highest: lanes that
// read one unit of 8 features in a row meet 8 different places, lanes that
// write one feature of 8 pieces as well (chunk_of), and the 32-feature steps
// of a wave's reads keep the key, so that they differ by a constant.
template <uint32_t TILE>
__device__ __forceinline__ uint32_t unit_at(uint32_t f, uint32_t u) {
    const uint32_t key = (f ^ (f >> 3 & 3) ^ (f / (TILE / 2) << 2)) & 7;
    return f * (kStep * 2) + (u ^ key) * 16;
}
// The chunk of the p-th pair of lanes: bit 2 and the highest exchanged.
template <uint32_t TILE>
__device__ __forceinline__ uint32_t chunk_of(uint32_t p) {
    constexpr uint32_t kHigh = TILE / 16;
    const uint32_t low = p >> 2 & 1, high = p / kHigh & 1;
    return (p & ~(kHigh | 4u)) | high << 2 | low * kHigh;
}

// Four of a piece's features laid into a tile.
template <uint32_t TILE, int HALF, int TYPE>
__device__ __forceinline__ void put_half(uint8_t *tile, const Piece<TYPE> &p, uint32_t chunk,
                                         uint32_t group) {
    float scale[4] = {};
    if constexpr (TYPE == kI8) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            scale[i] = act_scale(p.t[i].exp);
    }
#pragma unroll
    for (int e = HALF * 4; e < HALF * 4 + 4; ++e)
        *reinterpret_cast<u32x2 *>(tile + unit_at<TILE>(chunk * 8 + e, group / 2) + group % 2 * 8) =
            turned(p, e, scale);
}

// The dispatcher deals workgroups to the 8 XCDs in turn; each XCD takes a run of
// consecutive places of the `count` in a launch.
__device__ __forceinline__ uint32_t xcd_run(uint32_t w, uint32_t count) {
    const uint32_t xcd = w % 8, q = count / 8, r = count % 8;
    return xcd * q + (xcd < r ? xcd : r) + w / 8;
}

// Tile t.  Tiles are ordered in bands of kBand tile rows, so that the 32 that an
// XCD works on at a time share few rows and columns in its L2.
constexpr uint32_t kBand = 8;
__device__ __forceinline__ void tile_at(uint32_t t, uint32_t tiles_n, uint32_t tiles_k,
                                        uint32_t &tile_n, uint32_t &tile_k) {
    const uint32_t band = t / (kBand * tiles_k), first = band * kBand;
    const uint32_t high = tiles_n - first < kBand ? tiles_n - first : kBand;
    const uint32_t at = t - first * tiles_k;
    tile_n = first + at % high;
    tile_k = at / high;
}

template <int X, int TILE, int WAVES_N, int WAVES_K>
__global__ __launch_bounds__(WAVES_N *WAVES_K *kWave) void weight_grad_kernel(WeightGradArgs a) {
    constexpr int MN = TILE / WAVES_N / 32, MK = TILE / WAVES_K / 32;
    constexpr uint32_t kChunks = TILE / 8, kBytes = TILE * kStep * 2;
    // pieces a lane, kApart tokens from each other
    constexpr uint32_t kPieces = kChunks * kStep / 4 / (WAVES_N * WAVES_K * kWave);
    constexpr uint32_t kApart = kStep / kPieces;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];  // [2 turns][2 operands][kBytes]
    const uint32_t tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    // the whole tiles first, then the splits of the tail's, split by split
    const bool whole = blockIdx.x < a.whole;
    const uint32_t tail = a.tiles_n * a.tiles_k - a.whole;
    uint32_t tile, split = 0, tile_n, tile_k;
    if (whole) {
        tile = xcd_run(blockIdx.x, a.whole);
    } else {
        const uint32_t at = xcd_run(blockIdx.x - a.whole, tail * a.splits);
        split = at / tail;
        tile = a.whole + at % tail;
    }
    tile_at(tile, a.tiles_n, a.tiles_k, tile_n, tile_k);
    const uint32_t n0 = tile_n * TILE, k0 = tile_k * TILE;
    const size_t tokens = whole ? a.rows : a.split_rows;
    const size_t begin = split * tokens;
    const size_t end = begin + tokens < a.rows ? begin + tokens : a.rows;

    // the lane's piece: neighbouring lanes take the two halves of a unit
    const uint32_t chunk = chunk_of<TILE>(tid / 2 % kChunks), group = tid % 2 + 2 * (tid / (2 * kChunks));
    const uint32_t wn = (uint32_t)__builtin_amdgcn_readfirstlane((int)(wave / WAVES_K)) * (TILE / WAVES_N);
    const uint32_t wk = wave % WAVES_K * (TILE / WAVES_K);
    const Operand<kBf16> od = operand<kBf16>(a.dy, a.rows, a.n, n0 + chunk * 8, group * 4);
    const Operand<X> ox = operand<X>(a.x, a.rows, a.k, k0 + chunk * 8, group * 4);

    f32x16 acc[MN][MK];
#pragma unroll
    for (int i = 0; i < MN; ++i)
#pragma unroll
        for (int j = 0; j < MK; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[i][j][e] = 0.0f;

    Piece<kBf16> pd[kPieces];
    Piece<X> px[kPieces];
    auto get_dy = [&](size_t token) {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p)
            fetch(pd[p], od, token + p * kApart);
    };
    auto get_x = [&](size_t token) {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p)
            fetch(px[p], ox, token + p * kApart);
    };
    // half of a piece's features laid into LDS
    auto put_dy = [&](uint32_t buffer, auto half) {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p)
            put_half<TILE, decltype(half)::value>(lds + buffer * (2 * kBytes), pd[p], chunk,
                                                  group + p * kApart / 4);
    };
    auto put_x = [&](uint32_t buffer, auto half) {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p)
            hold_piece(px[p]);
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p)
            put_half<TILE, decltype(half)::value>(lds + buffer * (2 * kBytes) + kBytes, px[p],
                                                  chunk, group + p * kApart / 4);
    };
    constexpr std::integral_constant<int, 0> low;
    constexpr std::integral_constant<int, 1> high;
    auto put = [&](uint32_t buffer) {
        put_dy(buffer, low);
        put_dy(buffer, high);
        put_x(buffer, low);
        put_x(buffer, high);
    };
    bf16x8 fd[MN], fx[2][MK];
    auto read_x = [&](uint32_t buffer, uint32_t kk, auto set) {
        constexpr int S = decltype(set)::value;
        const uint8_t *from = lds + buffer * (2 * kBytes) + kBytes;
#pragma unroll
        for (int j = 0; j < MK; ++j)
            fx[S][j] = *reinterpret_cast<const bf16x8 *>(
                from + unit_at<TILE>(wk + j * 32 + lane % 32, kk * 2 + lane / 32));
    };
    auto read_dy = [&](uint32_t buffer, uint32_t kk, int i) {
        const uint8_t *from = lds + buffer * (2 * kBytes);
        fd[i] = *reinterpret_cast<const bf16x8 *>(
            from + unit_at<TILE>(wn + i * 32 + lane % 32, kk * 2 + lane / 32));
    };
    auto read = [&](uint32_t buffer, uint32_t kk, auto set) {
        read_x(buffer, kk, set);
#pragma unroll
        for (int i = 0; i < MN; ++i)
            read_dy(buffer, kk, i);
    };
    // The products of one step, and after the last one of each of dy's fragments
    // its read for step kk of `buffer` into the same registers (two sets of them
    // left no registers: 8192^3 947 us, 925 so).  A wave at its products goes before
    // one that lays tokens into LDS: 925 -> 906 us; with codes, whose conversion
    // then waits too long, 973 -> 1006, so not there.
    auto multiply = [&](auto set, uint32_t buffer, int kk) {
        constexpr int S = decltype(set)::value;
        if (kk >= 0) {
            if constexpr (S == 0)
                read_x(buffer, kk, high);
            else
                read_x(buffer, kk, low);
        }
        if constexpr (X == kBf16)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < MN; ++i) {
#pragma unroll
            for (int j = 0; j < MK; ++j)
                acc[i][j] =
                    __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[i], fx[S][j], acc[i][j], 0, 0, 0);
            if (kk >= 0)
                read_dy(buffer, kk, i);
        }
        if constexpr (X == kBf16)
            __builtin_amdgcn_s_setprio(0);
    };
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };

    // Turn s is multiplied from one buffer while turn s + 1, fetched a turn ago,
    // is laid into the other and turn s + 2 is on its way to registers.  A turn is
    // four steps of 16 tokens, each with the next step's LDS reads ahead of its
    // products; the barrier stands before the last step, whose products then cover
    // the other buffer's first reads.
    const uint32_t margin = od.margin > ox.margin ? od.margin : ox.margin;
    size_t turns = a.near ? (end - begin) / kStep : 0;
    if (turns && begin + turns * kStep + margin > a.rows)
        --turns;
    uint32_t buffer = 0;
    size_t token = begin + turns * kStep;  // of the turns at the end, fetched apart
    auto get_end = [&] {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) {
            fetch_end(pd[p], od, token + p * kApart + group * 4, end, a.rows);
            fetch_end(px[p], ox, token + p * kApart + group * 4, end, a.rows);
        }
    };
    if (turns) {
        const size_t last = begin + (turns - 1) * kStep;
        get_x(begin);
        get_dy(begin);
        put(0);
        if (turns > 1) {
            get_x(begin + kStep);
            get_dy(begin + kStep);
        }
        __syncthreads();
        read(0, 0, low);
        for (size_t at = begin; at < last; at += kStep) {
            const size_t next = at + 2 * kStep < last ? at + 2 * kStep : last;
            fence();
            put_x(buffer ^ 1, low);
            multiply(low, buffer, 1);
            fence();
            put_x(buffer ^ 1, high);
            get_x(next);
            multiply(high, buffer, 2);
            fence();
            put_dy(buffer ^ 1, low);
            put_dy(buffer ^ 1, high);
            get_dy(next);
            multiply(low, buffer, 3);
            fence();
            __syncthreads();
            buffer ^= 1;
            multiply(high, buffer, 0);
        }
        if (token < end)
            get_end();
        multiply(low, buffer, 1);
        multiply(high, buffer, 2);
        multiply(low, buffer, 3);
        multiply(high, buffer, -1);
        buffer ^= 1;
    } else if (token < end) {
        get_end();
    }
    while (token < end) {
        // the other buffer's readers are past the last barrier
        put(buffer);
        __syncthreads();
        token += kStep;
        if (token < end)
            get_end();
#pragma unroll 1
        for (uint32_t kk = 0; kk < kStep / 16; ++kk) {
            read(buffer, kk, low);
            multiply(low, buffer, -1);
        }
        buffer ^= 1;
    }

    // lane l holds column l % 32 and, in register r, row 8 (r / 4) + 4 (l / 32) + r % 4
    const bool direct = whole || a.splits == 1;
    float *out = a.dw + n0 * a.dw_stride + k0;
    size_t stride = a.dw_stride;
    if (!direct) {
        out = a.parts + ((size_t)split * tail + (tile - a.whole)) * (TILE * TILE);
        stride = TILE;
    }
    // A lane's rows are apart by multiples of the stride that are the same in all
    // lanes.  Sixteen of dw's elements are on their way at a time where dw is added
    // to, and rows are checked in the last row of tiles alone, by groups of eight
    // (each element checked and addressed by itself: 1x300x300 7.9 us, 5.2 so;
    // 128x4544x18176 added to dw 384, 144).
    auto store = [&](auto add, auto check) {
#pragma unroll
        for (int j = 0; j < MK; ++j) {
            const uint32_t col = wk + j * 32 + lane % 32;
            if (k0 + col >= a.k)
                continue;
            const uint32_t row = wn + 4 * (lane / 32);
            float *p = out + row * stride + col;
#pragma unroll
            for (int i = 0; i < MN; ++i) {
                // f(r, q) for the rows that there are
                auto rows = [&](auto &&f) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const uint32_t first = n0 + wn + i * 32 + 8 * g;
                        float *q = p + (i * 32 + 8 * g) * stride;
                        if (!decltype(check)::value || first + 8 <= a.n) {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                f(4 * g + r, q + r * stride);
                        } else if (first < a.n) {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (first + 4 * (lane / 32) + r < a.n)
                                    f(4 * g + r, q + r * stride);
                        }
                    }
                };
                if constexpr (decltype(add)::value) {
                    float was[16];
                    rows([&](int r, const float *q) { was[r] = *q; });
                    rows([&](int r, float *q) { *q = was[r] + acc[i][j][r]; });
                } else {
                    rows([&](int r, float *q) { *q = acc[i][j][r]; });
                }
            }
        }
    };
    constexpr std::true_type yes;
    constexpr std::false_type no;
    const bool check = direct && a.n - n0 < TILE;
    if (direct && a.accumulate) {
        if (check)
            store(yes, yes);
        else
            store(yes, no);
    } else if (check) {
        store(no, yes);
    } else {
        store(no, no);
    }
}

// dw (+)= the tail tiles' splits, in order: a workgroup takes 2 rows of a tile,
// lanes neighbouring columns.  Loads wait for each other's splits no more than they
// have to (one split at a time, 4 rows: 8192x128x128 25.2 us, 11.8 so).
constexpr uint32_t kJoinRows = 2;
template <int TILE>
__global__ __launch_bounds__(TILE) void weight_grad_join(WeightGradArgs a) {
    const uint32_t tail = a.tiles_n * a.tiles_k - a.whole;
    const uint32_t t = blockIdx.x / (TILE / kJoinRows), row = blockIdx.x % (TILE / kJoinRows) * kJoinRows;
    uint32_t tile_n, tile_k;
    tile_at(a.whole + t, a.tiles_n, a.tiles_k, tile_n, tile_k);
    const uint32_t n0 = tile_n * TILE + row, col = tile_k * TILE + threadIdx.x;
    if (n0 >= a.n || col >= a.k)
        return;
    const float *p = a.parts + (size_t)t * (TILE * TILE) + row * TILE + threadIdx.x;
    // rows past the last are the last again, and not stored
    const uint32_t rows = a.n - n0 < kJoinRows ? a.n - n0 : kJoinRows;
    float sum[kJoinRows] = {};
    // U splits' loads at a time; those past the last are not added
    auto add = [&](auto at_a_time) {
        constexpr uint32_t U = decltype(at_a_time)::value;
        for (uint32_t s = 0; s < a.splits; s += U) {
            float v[U][kJoinRows];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const size_t split = s + u < a.splits ? s + u : a.splits - 1;
#pragma unroll
                for (uint32_t r = 0; r < kJoinRows; ++r)
                    v[u][r] = p[split * tail * (TILE * TILE) + (r < rows ? r : rows - 1) * TILE];
            }
#pragma unroll
            for (uint32_t u = 0; u < U; ++u)
#pragma unroll
                for (uint32_t r = 0; r < kJoinRows; ++r)
                    sum[r] += s + u < a.splits ? v[u][r] : 0.0f;
        }
    };
    if (a.splits <= 3)
        add(std::integral_constant<uint32_t, 3>());
    else
        add(std::integral_constant<uint32_t, 8>());
#pragma unroll
    for (uint32_t r = 0; r < kJoinRows; ++r)
        if (r < rows) {
            float *out = a.dw + (size_t)(n0 + r) * a.dw_stride + col;
            *out = a.accumulate ? *out + sum[r] : sum[r];
        }
}

// The gradient of no tokens.
__global__ __launch_bounds__(256) void weight_grad_zero(float *dw, uint32_t n, uint32_t k,
                                                        size_t stride) {
    const size_t total = (size_t)n * k;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total;
         i += (size_t)gridDim.x * 256)
        dw[i / k * stride + i % k] = 0.0f;
}

constexpr size_t kMostSplits = 64;

struct GradShape {
    uint32_t tile, splits;
    size_t tiles, whole, split_rows;
    size_t parts() const { return splits > 1 ? splits * (tiles - whole) * tile * tile : 0; }
};

// Tile, and into how many splits of the tokens, with the smallest expected time.
// Workgroups run in rounds over the CUs (two of tile 128 fit a CU, one of tile
// 256): as many whole rounds of tiles as there are take their tokens undivided, or
// none does where the tiles are few; the rest are split, which shortens the last
// round and costs the traffic of the partial results.  A round is as long as its
// turns and a fixed part; the constants, in us, are fitted to 50 sizes measured with
// each tile and 1 to 64 splits, from bf16 and from checkpoints, of which the choice
// misses the fastest by 1% on average; of 32 other sizes by 2%, at worst by 22%
// (770x320x3648 from bf16: 16.7 us, 13.7 undivided).  Tile 128 against 256, nothing split:
// 4096x18176x4544 785 / 570, 2048x4096x4096 82 / 66, 4096x2048x2048 50 / 83,
// 300x2048x2048 11 / 16.  Splits of tile 128, 1 / 4 / 16: 8192x1024x1024 82 / 33 /
// 40, 8192x256x256 80 / 26 / 14, 1000x1000x1000 16 / 18 / 33.
GradShape grad_shape(size_t rows, size_t n, size_t k) {
    const size_t turns = (rows + kStep - 1) / kStep;
    GradShape best = {};
    double least = 1e30;
    for (const uint32_t tile : {128u, 256u}) {
        const size_t tiles = ((n + tile - 1) / tile) * ((k + tile - 1) / tile);
        const size_t slots = tile == 256 ? kCus : 2 * kCus;
        const auto round = [&](double per, double groups) {
            return tile == 256      ? 1.45 * per + 6.5
                   : groups <= kCus ? 0.75 * per + 3.0
                                    : 1.22 * per + 2.7;
        };
        for (size_t splits = 1; splits <= kMostSplits && splits <= turns; ++splits) {
            const size_t per = (turns + splits - 1) / splits;
            if ((turns + per - 1) / per != splits)
                continue;  // the same as a smaller number
            const size_t whole = splits == 1 ? tiles : tiles / slots * slots;
            const double rest = (double)(tiles - whole) * (double)splits;
            double time =
                ceil((double)whole / (double)slots) * round((double)turns, (double)whole);
            if (rest > 0)
                time += ceil(rest / (double)slots) * round((double)per, rest) + 1.5 +
                        0.1 * (double)splits + 2.0 * rest * tile * tile * 4.0 / 11e6;
            if (time < least) {
                least = time;
                best = {tile, (uint32_t)splits, tiles, whole, per * kStep};
            }
        }
    }
    return best;
}

template <int X, int TILE, int WAVES_N, int WAVES_K>
hipError_t start(const WeightGradArgs &a, const GradShape &s, hipStream_t stream) {
    constexpr size_t kLds = 2 * 2 * TILE * kStep * 2;
    const void *kernel =
        reinterpret_cast<const void *>(weight_grad_kernel<X, TILE, WAVES_N, WAVES_K>);
    static std::atomic<uint64_t> asked{0};
    const hipError_t e = allow_lds(kernel, kLds, asked);
    if (e != hipSuccess)
        return e;
    const size_t tail = s.tiles - s.whole, groups = s.whole + tail * s.splits;
    hipLaunchKernelGGL((weight_grad_kernel<X, TILE, WAVES_N, WAVES_K>), dim3((unsigned)groups),
                       dim3(WAVES_N * WAVES_K * kWave), kLds, stream, a);
    if (s.splits > 1 && tail)
        hipLaunchKernelGGL((weight_grad_join<TILE>), dim3((unsigned)(tail * (TILE / kJoinRows))),
                           dim3(TILE), 0, stream, a);
    return hipGetLastError();
}

template <int X>
hipError_t start(const WeightGradArgs &a, const GradShape &s, hipStream_t stream) {
    return s.tile == 256 ? start<X, 256, 2, 4>(a, s, stream) : start<X, 128, 2, 2>(a, s, stream);
}

}  // namespace

size_t weight_grad_workspace(size_t rows, size_t n, size_t k) {
    return grad_shape(rows, n, k).parts() * sizeof(float);
}

hipError_t launch_weight_grad(const Mat &dy, const Mat &x, int x_type, size_t rows, size_t n,
                              size_t k, const Mat &dw, int accumulate, void *workspace,
                              hipStream_t stream) {
    WeightGradArgs a = {};
    a.dy = dy;
    a.x = x;
    a.dw = reinterpret_cast<float *>(dw.data);
    a.dw_stride = dw.stride;
    a.n = (uint32_t)n;
    a.k = (uint32_t)k;
    if (rows == 0) {
        if (!accumulate) {
            const size_t groups = (n * k + 255) / 256;
            hipLaunchKernelGGL(weight_grad_zero, dim3((unsigned)(groups < 8 * kCus ? groups : 8 * kCus)),
                               dim3(256), 0, stream, a.dw, a.n, a.k, a.dw_stride);
        }
        return hipGetLastError();
    }
    const GradShape s = grad_shape(rows, n, k);
    // a grid has 2^32 - 1 work-items at most
    if (s.tiles > UINT32_MAX / 512 / s.splits)
        return hipErrorInvalidConfiguration;
    a.parts = reinterpret_cast<float *>(workspace);
    a.rows = rows;
    a.split_rows = s.split_rows;
    a.tiles_n = (uint32_t)((n + s.tile - 1) / s.tile);
    a.tiles_k = (uint32_t)((k + s.tile - 1) / s.tile);
    a.whole = (uint32_t)s.whole;
    a.splits = s.splits;
    a.accumulate = accumulate;
    a.near = dy.stride <= kNear && x.stride <= kNear && k <= kNear;
    return x_type == kI8 ? start<kI8>(a, s, stream) : start<kBf16>(a, s, stream);
}

}  // namespace zpp
