// Attention of new tokens over the paged cache: sequences with many rows
// (prompts and chunks of them).
//
// Rows of a sequence and a KV head are its new tokens times the query heads that
// share the head, token by token; so the heads of a group share every key and value
// that is read, and a tile of 256 rows (128 for heads of more than 128 elements) is
// few tokens wide.
#include <hip/hip_runtime.h>

#include <float.h>

#include <algorithm>

#include "attend_common.h"
#include "attend_few.h"
#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl_internal.h"

namespace tl {
namespace {

constexpr int kKeys = 64;               // cached tokens of a step

// Row tiles are numbered through the batch with gaps, which needs no sum over
// the batch: sequence b's begin at floor(rows before it / ROWS) + b, or, in a batch of
// mostly few rows, at floor(rows before it / (kFewRows + 1)); both leave room for
// all of them (number_tiles).
__device__ __forceinline__ int64_t first_tile(const AttendLaunch& F, int64_t b) {
    const AttendParams& P = F.a;
    return clamp_offset(P.c, P.c.q_offset[b]) * P.group / F.tile_per + (F.tile_each ? b : 0);
}

// The last sequence whose first tile is at most `tile`: 64 ways at a time.
__device__ __forceinline__ int64_t tile_seq(const AttendLaunch& F, int64_t tile) {
    int64_t lo = 0, hi = F.a.c.n_seqs;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane_id() * step;
        const bool below = at < hi && first_tile(F, at) <= tile;
        const int k = max((int)__popcll(__ballot(below)) - 1, 0);
        lo += k * step;
        hi = min(lo + step, hi);
    }
    return lo;
}

// One piece: lane l copies the 16 bytes at its `src` to LDS address lds + 16 l
// (lds the same in every lane), straight from memory.  An instruction that the
// compiler does not track, so that reads of the other buffer do not wait for
// it; `settle` waits for the copies (vmcnt) before a barrier hands them over.
__device__ __forceinline__ void copy_piece(const uint16_t* src, uint32_t lds) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\t" TL_M0_WAIT "\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src)
                 : "memory", "m0");
}

// The same for 4 bytes a lane.
__device__ __forceinline__ void copy_words(const int32_t* src, uint32_t lds) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\t" TL_M0_WAIT "\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(src)
                 : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// Four 16-bit words of a column: within 16 lanes, lane i gives the address of
// 4 words of row i / 4 (of 4 rows x 16 words) and takes column i.
__device__ __forceinline__ uint2 read_column4(const void* lds) {
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    return __builtin_bit_cast(uint2,
                              __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)lds));
}

// The value of the lane 32 away.
__device__ __forceinline__ float other_half(float x) {
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, lane_id() < 32 ? r[1] : r[0]);
}

// Bits 0 .. k of 64 (none for k < 0).
__device__ __forceinline__ uint64_t bits_to(int32_t k) { return k < 0 ? 0 : ~0ull >> (63 - min(k, 63)); }

// The tokens t0 .. t0 + 63 that a row at position p sees.
__device__ __forceinline__ uint64_t seen_bits(int32_t window, int32_t sinks, int32_t p, int32_t t0) {
    uint64_t r = bits_to(p - t0);
    if (window > 0) r &= ~bits_to(p - window - t0) | bits_to(sinks - 1 - t0);
    return r;
}

// What the piece numbers of a token's row are exchanged with: the same piece of
// 16 consecutive tokens lies in 16 places of the 256 bytes that the banks
// hold (keys), and so do 4 consecutive pieces of 4 (values).
template <int PIECES>
__device__ __forceinline__ int key_exchange(int token) {
    return PIECES > 8 ? token & 15 : token >> 1 & 7;
}
template <int PIECES>
__device__ __forceinline__ int value_exchange(int token) {
    return PIECES > 8 ? (token & 3) << 2 : (token >> 1 & 1) << 2;
}

// 256 rows (128 for head_dim > 128) of one sequence and KV head over one part
// of its tokens, 32 rows a wavefront.  The products run as K Q^T and V^T P^T
// (32 x 32 matrix instructions), so that a lane keeps one row (lane % 32)
// throughout: scores, weights, maximum and sums; the first product's result is
// the second's operand as it lies: in both, lane group g = lane / 32 has the
// tokens 4 g .. 4 g + 3 and 8 + 4 g .. of each 16.  Keys and values go from memory
// straight to LDS, token by token; the values are turned when they are read.
// 16-byte pieces of a token's row are exchanged (xor) so that the lanes that read
// together meet in no bank.
//
// A step (64 tokens) has a matrix phase, the last step's V^T P^T and this
// one's K Q^T, and a softmax phase, which take about as long.  The two wavefronts of
// a SIMD are a phase apart, a barrier after each phase keeps them so: one's matrix
// instructions run under the other's softmax.  (For head_dim > 128 a SIMD's
// registers hold one wavefront, which takes the phases in turn.)  Copies of later
// steps are issued between the matrix instructions, one at a time.
//
// 32768 tokens through a window of 4096, 8 heads on one KV head: 0.56 ms, 925
// TFLOP/s; 8 ragged prompts of up to 4096 tokens, 32 heads on 8: 0.54 ms, 813
// (a 16384^3 product of the library: 1363).  A step takes 4040 cycles, of which the
// matrix units are busy 2048; over the launch, its first and last steps included, they
// are busy 42% and 37% of the cycles, at 1.97 GHz (few_rows alone runs at 2.31).
// What holds a step up most is the operands' reads from LDS: without those of the
// keys it takes a fifth less, and without the exponentials, the copies or the values'
// reads 6 to 14%.  A wavefront gets 32 bytes a cycle from LDS, just what its matrix
// instructions use with 32 rows; 64 rows a wavefront would halve that, but the compiler
// does not keep their scores in registers.
template <int DP>
struct TileLds {
    // Steps in LDS: step v copies the keys of step v + kRing - 1 and the values
    // of step v + kRing - 2, and looks up step v + kRing + 1.
    static constexpr int kRing = DP > 128 ? 2 : 3;
    u32x4 keys[kRing][kKeys * (DP / 8)];        // of step v in v % kRing
    u32x4 values[kRing][kKeys * (DP / 8)];
    int64_t where[8][kKeys];                    // of step v in v % 8
    uint64_t present[8];
    int32_t pages[4][kKeys];                    // of the steps that are looked up, a wavefront's each
};

template <bool F16, int DP, bool EXACT>
__device__ __forceinline__ void tile_rows(const AttendLaunch& F, int64_t block, TileLds<DP>& lds) {
    constexpr int kTileWaves = tile_waves(DP), kTileThreads = kTileWaves * kWave, kTileRows = tile_rows_of(DP);
    constexpr int kSteps = DP / 16;                     // matrix instructions of a score
    constexpr int kBlocks = DP / 32;                    // of 32 elements of the output
    constexpr int kPieces = DP / 8;                     // 16-byte pieces of a row
    constexpr int kLoads = kKeys * kPieces / kTileThreads;          // pieces of keys, and of values, a thread stages
    constexpr int kTokenStep = kTileThreads / kPieces;              // from one to the next
    constexpr int kRing = TileLds<DP>::kRing;
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int D = EXACT ? DP : c.head_dim;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = lane_id(), n = lane & 31, g = lane >> 5;
    const bool second = wave >= 4;                      // the wavefronts that are a phase behind

    auto& key_lds = lds.keys;
    auto& value_lds = lds.values;
    auto& where = lds.where;
    auto& present = lds.present;
    auto& pages = lds.pages;

    // KV head fastest, then the part, then the row tile, the last (longest) first
    int64_t x = block;
    const int32_t kvh = (int32_t)(x % c.n_kv_heads);
    x /= c.n_kv_heads;
    const int32_t part = (int32_t)(x % F.tiles.count);
    x /= F.tiles.count;
    const int64_t tile = F.tile_count - 1 - x;
    const int64_t b = tile_seq(F, tile);
    const SeqRows s = seq_rows(c, b);
    const int64_t rows = (int64_t)s.n * P.group;
    const int64_t row0 = (tile - first_tile(F, b)) * kTileRows;
    if (rows <= kFewRows || row0 < 0 || row0 >= rows) return;

    const int32_t base = s.length - s.n;                // position of the first new token
    const int64_t row = row0 + wave * kWaveRows + n;
    const bool real = row < rows;
    const int32_t token = (int32_t)((real ? row : rows - 1) / P.group);
    const int32_t head = kvh * P.group + (int32_t)((real ? row : rows - 1) - (int64_t)token * P.group);
    const int32_t pos = base + token;
    // positions of the workgroup's rows, and of the wavefront's
    const int32_t first_pos = base + (int32_t)(row0 / P.group);
    const int32_t last_pos = base + (int32_t)((min(row0 + kTileRows, rows) - 1) / P.group);
    const int64_t wave_row = row0 + wave * kWaveRows;
    const bool idle = wave_row >= rows;
    const int32_t wave_first = base + (int32_t)(wave_row / P.group);
    const int32_t wave_last = base + (int32_t)((min(wave_row + kWaveRows, rows) - 1) / P.group);

    const TileList tiles = visible_tiles<kKeys>(c, P.window, P.sinks, first_pos, last_pos);
    const int32_t per = max(F.tiles.tokens / kKeys, (tiles.count + F.tiles.count - 1) / F.tiles.count);
    const int32_t v_first = (int32_t)min((int64_t)tiles.count, (int64_t)part * per);
    const int32_t v_end = (int32_t)min((int64_t)tiles.count, (int64_t)(part + 1) * per);
    const int32_t count = v_end - v_first;              // steps, numbered from 0 below

    f32x16 acc[kBlocks];
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] = 0.0f;
    float m = kNone, l = 0.0f;
    bool special = false;               // this thread's values need the rows one by one

    if (count > 0) {
        u32x4 q[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 16 * k + 8 * g;
            q[k] = u32x4{0, 0, 0, 0};
            if (real && (EXACT || d < D))
                q[k] = *(const u32x4*)(P.query + (s.first + token) * P.query_token_stride +
                                       (int64_t)head * P.query_head_stride + d);
        }
        const int32_t* const table_row = c.table + b * c.table_width;

        // What this thread stages: slot tid + i kTileThreads of the keys and
        // of the values, which hold piece (slot ^ exchange) of token slot / kPieces.
        const int my_token = tid / kPieces, slot = tid % kPieces;
        const int key_piece = slot ^ key_exchange<kPieces>(my_token);
        constexpr int kOdd = kTokenStep % 16;       // 8: every other token has another exchange
        const int value_piece = slot ^ value_exchange<kPieces>(my_token);
        const uint16_t* const keys = c.key + (int64_t)kvh * c.head_stride + key_piece * 8;
        const uint16_t* const values = c.value + (int64_t)kvh * c.head_stride + value_piece * 8;
        const int odd_step = (key_piece ^ kOdd) * 8 - key_piece * 8;
        const bool key_in[2] = {EXACT || key_piece * 8 < D, EXACT || (key_piece ^ kOdd) * 8 < D};
        const bool value_in = EXACT || value_piece * 8 < D;

        // The pages of step v's tokens, a token a lane; and, when they are here,
        // where the tokens lie.  (A token that no row sees, or without a page,
        // copies some page's, which is not used; steps from `count` on copy the
        // last one's again.)
        const uint32_t end = (uint32_t)tiles.end;
        auto lookup = [&](int32_t v) {
            const uint32_t t = min((uint32_t)(tiles.tile(v_first + v) * kKeys + lane), end - 1);
            copy_words(table_row + div_u32(t, c.div_page), lds_address(pages[wave & 3]));
        };
        auto keep_lookup = [&](int32_t v) {
            const uint32_t t = (uint32_t)(tiles.tile(v_first + v) * kKeys + lane), u = min(t, end - 1);
            const bool seen = t < end && sees(P.window, P.sinks, max(first_pos, (int32_t)u), (int32_t)u);
            const uint32_t in_page = u - div_u32(u, c.div_page) * (uint32_t)c.page_tokens;
            const int32_t page = pages[wave & 3][lane];
            const bool there = seen && page >= 0 && page < c.n_pages;
            const uint64_t mask = __ballot(there);
            where[v & 7][lane] = there ? page * c.page_stride + (int64_t)in_page * c.token_stride : 0;
            if (lane == 0) present[v & 7] = mask;
        };
        // What is copied in step v.  `find` reads where it lies, a phase before.
        int64_t key_from[kLoads], value_from[kLoads];
        const uint32_t key_to = lds_address(key_lds) + wave * (kWave * 16), value_to = lds_address(value_lds) + wave * (kWave * 16);
        constexpr uint32_t kBufferBytes = kKeys * kPieces * 16, kLoadBytes = kTileThreads * 16;
        uint64_t there = 0;             // the tokens of step v that are copied
        auto find = [&](int32_t v) {
            const int k = min(v + kRing - 1, count - 1) & 7, y = min(v + kRing - 2, count - 1) & 7;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                key_from[i] = where[k][my_token + i * kTokenStep];
                value_from[i] = where[y][my_token + i * kTokenStep];
            }
            there = present[min(v, count - 1) & 7];
        };
        auto copy_key = [&](int buffer, int i) {
            if (key_in[i & 1])
                copy_piece(keys + (key_from[i] + (i & 1 ? odd_step : 0)), key_to + buffer * kBufferBytes + i * kLoadBytes);
        };
        auto copy_value = [&](int buffer, int i) {
            if (value_in) copy_piece(values + value_from[i], value_to + buffer * kBufferBytes + i * kLoadBytes);
        };
        auto copy_all = [&](int key_buffer, int value_buffer) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                copy_key(key_buffer, i);
                copy_value(value_buffer, i);
            }
        };
        // After the copies of step v: values of tokens that nobody sees are 0;
        // and whether one that some rows see and others do not is not finite,
        // which would reach the others as 0 x value.
        auto settle = [&](int32_t v, uint64_t there, int value_buffer) {
            // (with three steps in LDS this step's own copies may still be under
            // way: each wavefront issues 2 kLoads)
            if constexpr (kRing == 3 && kLoads == 2) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
            else if constexpr (kRing == 3 && kLoads == 1) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const int32_t t0 = tiles.tile(v_first + v) * kKeys, t_last = t0 + kKeys - 1;
            const bool all = t_last <= first_pos && (P.window == 0 || t0 > last_pos - P.window || t_last < P.sinks);
            if (v >= count || (there == ~0ull && all)) return;
            for (int i = 0; i < kLoads; ++i) {
                u32x4* const at = &value_lds[value_buffer][tid + i * kTileThreads];
                if (!(there >> (my_token + i * kTokenStep) & 1)) {
                    *at = u32x4{0, 0, 0, 0};
                } else if (!all) {
                    const u32x4 y = *at;
                    special |= not_finite2<F16>(y[0]) || not_finite2<F16>(y[1]) || not_finite2<F16>(y[2]) ||
                               not_finite2<F16>(y[3]);
                }
            }
        };
        // A barrier after a phase: nothing moves across it.
        auto phase_end = [&] {
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };

        // pieces beyond head_dim stay 0; and the first step takes a product of
        // zeros
        for (int i = tid; i < kRing * kKeys * kPieces; i += kTileThreads) {
            if (!EXACT || i >= (kRing - 1) * kKeys * kPieces) value_lds[0][i] = u32x4{0, 0, 0, 0};
            if constexpr (!EXACT) key_lds[0][i] = u32x4{0, 0, 0, 0};
        }
        if (wave <= kRing && wave < count) lookup(wave);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (wave <= kRing && wave < count) keep_lookup(wave);
        __syncthreads();
        // what the steps before the first one copy: keys 0 .. kRing - 2, values
        // 0 .. kRing - 3
        if constexpr (kRing == 3) {
            find(-1);
            copy_all(1, 0);
        }
        find(1 - kRing);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) copy_key(0, i);
        // the queries are there before the first copies of the loop are under way
#pragma unroll
        for (int k = 0; k < kSteps; ++k) asm volatile("" : "+v"(q[k]));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();

        // where this lane reads: keys of token 32 h + n, and columns of the values
        const int key_at = n * kPieces, key_turn = key_exchange<kPieces>(n);
        const int value_token = 4 * g + (lane & 15) / 4;
        int value_at[kBlocks];          // bytes
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
            const int piece = (4 * j + 2 * (lane >> 4 & 1) + (lane & 3) / 2) ^ value_exchange<kPieces>(value_token);
            value_at[j] = (value_token * kPieces + piece) * 16 + (lane & 1) * 8;
        }
        // the two products of a step
        f32x16 sc[2];
        u32x4 w[2][2];
        // (the last step's first), operands read kAhead instructions ahead: left to
        // itself the compiler saves registers and waits for every read
        constexpr int kProducts = 4 * kBlocks;
        static_assert(kProducts == 2 * kSteps);
        constexpr int kAhead = 4;
        auto multiply = [&](int now, int before) {      // places of this step and the last one
            const unsigned char* const old_values = (const unsigned char*)value_lds[before];
            const u32x4* const new_keys = key_lds[now];
            // (the copies' places are the ones that were read last)
            const int key_buffer = before, value_buffer = kRing == 3 ? (now == 2 ? 0 : now + 1) : now;
            u32x4 a[kAhead];
            auto read = [&](int i) {
                if (i < kProducts) {
                    const unsigned char* const p = old_values + value_at[i % kBlocks] + 16 * (i / kBlocks) * kPieces * 16;
                    const uint2 lo = read_column4(p), hi = read_column4(p + 8 * kPieces * 16);
                    a[i % kAhead] = u32x4{lo.x, lo.y, hi.x, hi.y};
                } else if (i < 2 * kProducts) {
                    const int k = (i - kProducts) / 2, h = (i - kProducts) % 2;
                    a[i % kAhead] = new_keys[key_at + 32 * h * kPieces + ((2 * k + g) ^ key_turn)];
                }
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * kProducts; ++i) {
                if (i < kProducts) {
                    const int j = i % kBlocks, y = i / kBlocks;
                    acc[j] = mfma32<F16>(a[i % kAhead], w[y / 2][y % 2], acc[j]);
                } else {
                    const int k = (i - kProducts) / 2, h = (i - kProducts) % 2;
                    if (k == 0)
#pragma unroll
                        for (int e = 0; e < 16; ++e) sc[h][e] = 0.0f;
                    sc[h] = mfma32<F16>(a[i % kAhead], q[k], sc[h]);
                }
                read(i + kAhead);
                // the copies, one at a time
                constexpr int kEvery = 2 * kProducts / (2 * kLoads);
                if (i % kEvery == kEvery / 2) {
                    const int y = i / kEvery;
                    if (y < kLoads) copy_key(key_buffer, y);
                    else copy_value(value_buffer, y - kLoads);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int y = 0; y < 2; ++y) w[h][y] = u32x4{0, 0, 0, 0};
        find(0);
        if (second) phase_end();
        int now = 0;                    // v % kRing
        for (int32_t v = 0; v <= count; ++v) {
            // ---- matrix phase
            const int before = now == 0 ? kRing - 1 : now - 1, after = now == kRing - 1 ? 0 : now + 1;
            const bool looks = wave == (v & 3) && v + kRing + 1 < count;
            const uint64_t seen = there;
            if (looks) lookup(v + kRing + 1);
            const int32_t t0 = tiles.tile(v_first + v) * kKeys, t_last = t0 + kKeys - 1;
            // (once a step is past the wavefront's rows all later ones are)
            const bool was_on = v == 0 || tiles.tile(v_first + v - 1) * kKeys <= wave_last;
            const bool on = !idle && v < count && t0 <= wave_last;
            if (!idle && was_on) multiply(now, before);
            else copy_all(before, kRing == 3 ? after : now);
            if (second) settle(v, seen, now);
            phase_end();
            // ---- softmax phase
            find(v + 1);
            if (on) {
                const bool full = seen == ~0ull && t_last <= wave_first &&
                                  (P.window == 0 || t0 > wave_last - P.window || t_last < P.sinks);
                if (!full) {
                    const uint64_t bits = (seen & seen_bits(P.window, P.sinks, pos, t0)) >> (4 * g);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t half = (uint32_t)(bits >> (32 * h));
                            sc[h][i] = half & (1u << (8 * (i / 4) + i % 4)) ? sc[h][i] : -INFINITY;
                        }
                }
                float tops[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    tops[u] = fmaxf(sc[0][u], sc[1][u]);
#pragma unroll
                    for (int i = u + 4; i < 16; i += 4) tops[u] = fmaxf(fmaxf(tops[u], sc[0][i]), sc[1][i]);
                }
                float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                top = fmaxf(top, other_half(top));
                // The sums are only scaled down when the maximum has grown by
                // more than 2^kGrowTiles for some row: weights that much larger lose
                // nothing.
                if (__any((top - m) * F.score_scale > kGrowTiles<F16> || (m == kNone && top > kNone))) {
                    const float m2 = fmaxf(m, top), keep = weight(m, m2, F.score_scale);
                    l *= keep;
                    m = m2;
#pragma unroll
                    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[j][i] *= keep;
                }
                // (the difference of scores first only where they are so large
                // that it matters: 32 instructions)
                float back = m == kNone ? kLiftTiles<F16> : fmaf(-m, F.score_scale, kLiftTiles<F16>);
                if (__any(fabsf(back) > 65536.0f)) {
                    back = kLiftTiles<F16>;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 16; ++i) sc[h][i] -= m;
                }
                float sum[4] = {0, 0, 0, 0};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float a = exp2_fast(fmaf(sc[h][i], F.score_scale, back));
                        const float z = exp2_fast(fmaf(sc[h][i + 1], F.score_scale, back));
                        sum[i / 2 % 4] += a + z;
                        w[h][i / 8][i % 8 / 2] = pack2<F16>(a, z);
                    }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            }
            if (!second) settle(v, seen, now);
            if (looks) keep_lookup(v + kRing + 1);
            phase_end();
            now = after;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (!second) phase_end();
        l += __shfl_xor(l, 32);
    }

    const int64_t to = (s.first + token) * P.n_heads + head;
    const bool split = F.tiles.count > 1;
    if (__syncthreads_or(special)) {
        for (int r = 0; r < kWaveRows; ++r) {
            const int64_t rr = wave_row + r;
            if (rr >= rows) break;
            const int32_t tok = (int32_t)(rr / P.group), hd = kvh * P.group + (int32_t)(rr - (int64_t)tok * P.group);
            const RowSums y = row_alone<F16, kKeys>(P, b, s.first + tok, hd, base + tok, tiles, v_first, v_end, F.score_scale);
            const int64_t out = (s.first + tok) * P.n_heads + hd, part_slot = out * F.tiles.count + part;
            const int d = (lane & 31) * 8;
            if (lane < 32 && d < D) {
                const float f = y.l == 0.0f ? 0.0f : 1.0f / y.l;
                for (int e = 0; e < 8; ++e) {
                    if (split) F.tiles.sums[part_slot * D + d + e] = y.acc[e] * kLiftedTiles<F16>;
                    else P.out[out * D + d + e] = from_float<F16>(y.l == 0.0f ? 0.0f : y.acc[e] * f);
                }
            }
            if (lane == 0) {
                if (split) *(float2*)(F.tiles.stats + part_slot * 2) = make_float2(y.m, y.l * kLiftedTiles<F16>);
                else if (P.lse) P.lse[out] = log_sum(y.m, y.l, F.score_scale);
            }
        }
        return;
    }
    if (!real) return;
    const int64_t slot = to * F.tiles.count + part;
    const float f = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * j + 2 * i + 4 * g;
            if (!EXACT && d >= D) continue;
            f32x4 o = {acc[j][i], acc[j][i + 1], acc[j][i + 2], acc[j][i + 3]};
            if (split) {
                if (l != 0.0f) *(f32x4*)(F.tiles.sums + slot * D + d) = o;
            } else {
                if (l == 0.0f) o = f32x4{0, 0, 0, 0};
                *(uint2*)(P.out + to * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
            }
        }
    if (g == 0) {
        if (split) *(float2*)(F.tiles.stats + slot * 2) = make_float2(m, l);
        else if (P.lse) P.lse[to] = log_sum(m, l * kUnliftTiles<F16>, F.score_scale);
    }
}

// Workgroups of tile_rows first, then those of few_rows: compute on some CUs
// and reading on the others.  Two chunks of 512 tokens and 62 single tokens over
// 9001 to 16384 cached ones: 0.71 ms, 1.00 in two launches.
template <bool F16, int DP, bool EXACT>
__global__ __launch_bounds__(tile_waves(DP) * kWave, DP > 128 ? 1 : 2) void mixed_kernel(AttendLaunch F, int64_t first) {
    __shared__ union {
        TileLds<DP> tile;
        FewLds<tile_waves(DP), DP> few;
    } lds;
    const int64_t tiles = F.tile_count * F.a.c.n_kv_heads * F.tiles.count;
    const int64_t block = blockIdx.x + first;
    if (block < tiles) tile_rows<F16, DP, EXACT>(F, block, lds.tile);
    else few_rows<F16, DP, EXACT, tile_waves(DP), false>(F, block - tiles, lds.few);
}

template <bool F16, int DP>
hipError_t launch_dim(const AttendLaunch& f, int64_t few_blocks, hipStream_t stream) {
    const int64_t blocks = f.tile_count * f.a.c.n_kv_heads * f.tiles.count + few_blocks * f.few.count;
    return launch_all(blocks, tile_waves(DP) * kWave, [&](dim3 grid, int64_t first) {
        const dim3 block(tile_waves(DP) * kWave);
        if (f.a.c.head_dim == DP) hipLaunchKernelGGL((mixed_kernel<F16, DP, true>), grid, block, 0, stream, f, first);
        else hipLaunchKernelGGL((mixed_kernel<F16, DP, false>), grid, block, 0, stream, f, first);
    });
}

template <bool F16>
hipError_t launch_type(const AttendLaunch& f, int64_t few_blocks, hipStream_t stream) {
    if (f.a.c.head_dim <= 64) return launch_dim<F16, 64>(f, few_blocks, stream);
    if (f.a.c.head_dim <= 128) return launch_dim<F16, 128>(f, few_blocks, stream);
    return launch_dim<F16, 256>(f, few_blocks, stream);
}

}  // namespace

hipError_t launch_mixed(const AttendLaunch& f, int64_t few_blocks, hipStream_t stream) {
    return f.a.f16 ? launch_type<true>(f, few_blocks, stream) : launch_type<false>(f, few_blocks, stream);
}

}  // namespace tl
