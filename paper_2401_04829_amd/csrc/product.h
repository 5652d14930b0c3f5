// Tiles of a matrix product C = A B^T on matrix instructions, as the operators
// that do something with the product's elements use them.
//
// A has M rows and B has N of them, over K.  Either is given by rows of K
// elements on end (k contiguous) or turned over, K rows of its M (N) elements.
// A workgroup takes a tile of TM x TN, a wavefront MT x NT instructions of 16 x
// 16, whose results stay in registers; K is taken in chunks of KB bytes, which
// go through LDS in STAGES buffers: while one is multiplied the next ones are on
// their way, with one barrier per chunk.
//
// Which row of A an instruction's row is, is free to choose as long as the
// results are read that way: row p of tile (run j, place e) is
//     16 own j + own p + e,  own = 8, 4, 2 or 1 tiles side by side,
// so that a lane, which has rows 4 g .. 4 g + 3 of each tile, has 4 own of A's
// rows on end, and so that an operand that is turned over is read from LDS in
// packs of `own` elements: a lane reads 8 rows of K and swaps their 16-bit
// elements in pairs.  B's rows go by the same rule, a lane has `own` on end.
#pragma once

#include "tokens.h"

namespace gnnshap {

// How a product's operand lies in memory.
struct Operand {
  const void* p;
  int64_t stride;   // elements from row to row (of M or N; turned over: of K)
  int64_t rows;     // M or N
};

template <class T>
constexpr int own_tiles(int tiles) {
  return tiles % 8 == 0 && sizeof(T) == 2 ? 8 : tiles % 4 == 0 ? 4 : tiles % 2 == 0 ? 2 : 1;
}

// DIRECT: memory to LDS without registers between, for operands whose packs of
// 16 bytes are aligned and whole; else by way of registers, at any address.
template <class T_, int MT_, int NT_, int WAVES_M, int WAVES_N, int KB_, int STAGES_, bool A_TURNED, bool B_TURNED,
          bool DIRECT_>
struct Product {
  using T = T_;
  static constexpr int MT = MT_, NT = NT_, KB = KB_, STAGES = DIRECT_ ? STAGES_ : 2;
  static constexpr bool DIRECT = DIRECT_, kTurnedB = B_TURNED;
  static constexpr int TM = 16 * MT * WAVES_M, TN = 16 * NT * WAVES_N;
  static constexpr int kWaves = WAVES_M * WAVES_N, kThreads = 64 * kWaves;
  static constexpr int kOwnA = own_tiles<T>(MT), kOwnB = own_tiles<T>(NT);
  static constexpr int KE = KB / sizeof(T);        // of K, a chunk
  static constexpr int kVec = 16 / sizeof(T), kSteps = KB / 64;
  static constexpr int kBytesA = TM * KB, kBytesB = TN * KB, kStage = kBytesA + kBytesB;
  static constexpr int kLds = STAGES * kStage;
  // Bytes of LDS of a launch: short sums need few buffers, and more workgroups fit a compute unit.
  static int lds_for(int64_t K, int segments) {
    const int64_t chunks = (K + KE - 1) / KE * segments;
    return static_cast<int>(chunks < 1 ? 1 : chunks < STAGES ? chunks : STAGES) * kStage;
  }
  // Moves of 1,024 bytes: each wavefront takes the same number of them (some of the last are made twice).
  static constexpr int kMoves = kStage / 1024, kLoads = (kMoves + kWaves - 1) / kWaves;
  static_assert(kBytesA % 1024 == 0 && kBytesB % 1024 == 0, "an operand's chunk is whole moves");
  static constexpr unsigned kNowhere = 0x80000000u;   // an offset behind every buffer: reads 0

  f4_t acc[MT][NT];

  // Row of the operand behind place `at` of its tile in LDS (a wavefront's tiles one after the other).
  template <int TILES, int OWN>
  static __device__ __forceinline__ int row_of(int at) {
    const int in = at % (16 * TILES), tile = in / 16, p = in % 16;
    return at - in + 16 * OWN * (tile / OWN) + OWN * p + tile % OWN;
  }
  // Swaps an LDS row's packs so that 16 lanes of 16 rows meet 16 places.
  static __device__ __forceinline__ int swapped(int row) { return KB == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }

  // What a lane moves to byte `at` of a stage: the byte offset from the
  // operand's first element of this tile and chunk, the rows (of M, or of K if
  // turned over) and the k's in front of it.
  template <bool TURNED, int TILES, int OWN, int SIZE>
  static __device__ __forceinline__ void source(int at, int64_t stride, int64_t& offset, int& row, int& k) {
    if constexpr (TURNED) {
      k = at / (SIZE * static_cast<int>(sizeof(T)));
      row = at % (SIZE * static_cast<int>(sizeof(T))) / static_cast<int>(sizeof(T));
      offset = (k * stride + row) * static_cast<int64_t>(sizeof(T));
    } else {
      const int place = at / KB, pack = at % KB / 16 ^ swapped(place);
      row = row_of<TILES, OWN>(place);
      k = pack * kVec;
      offset = (row * stride + k) * static_cast<int64_t>(sizeof(T));
    }
  }
  // Whether the move is of A.
  static __device__ __forceinline__ bool of_a(int move) { return move * 1024 < kBytesA; }

  // acc = sum over K of A[m0 ..] B[n0 ..]; `segments` times K, for each of
  // which A and B start as many bytes further on.
  __device__ __forceinline__ void run(char* lds, const Operand& A, const Operand& B, int64_t m0, int64_t n0, int64_t K,
                                      int segments = 1, int64_t a_segment = 0, int64_t b_segment = 0) {
    clear_sums();
    const int per = static_cast<int>((K + KE - 1) / KE);
    int chunks = per * segments;
    if (chunks == 0) return;
    const char* const a0 =
        static_cast<const char*>(A.p) + (A_TURNED ? m0 : m0 * A.stride) * static_cast<int64_t>(sizeof(T));
    const char* const b0 =
        static_cast<const char*>(B.p) + (B_TURNED ? n0 : n0 * B.stride) * static_cast<int64_t>(sizeof(T));
    const int64_t a_step = (A_TURNED ? KE * A.stride : KE) * static_cast<int64_t>(sizeof(T));
    const int64_t b_step = (B_TURNED ? KE * B.stride : KE) * static_cast<int64_t>(sizeof(T));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t m_left = A.rows - m0, n_left = B.rows - n0;
    // the chunk that is asked for next
    const char *a = a0, *b = b0;
    int64_t k_left = K;
    int segment = 0;
    const auto advance = [&] {
      a += a_step;
      b += b_step;
      k_left -= KE;
      if (k_left <= 0) {
        ++segment;
        a = a0 + segment * a_segment;
        b = b0 + segment * b_segment;
        k_left = K;
      }
    };

    if constexpr (DIRECT) {
      unsigned offset[kLoads];
      int ks[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int move = (wave + j * kWaves) % kMoves;
        int64_t off;
        int row;
        if (of_a(move)) {
          source<A_TURNED, MT, kOwnA, TM>(move * 1024 + lane * 16, A.stride, off, row, ks[j]);
          offset[j] = row < m_left ? static_cast<unsigned>(off) : kNowhere;
        } else {
          source<B_TURNED, NT, kOwnB, TN>(move * 1024 - kBytesA + lane * 16, B.stride, off, row, ks[j]);
          offset[j] = row < n_left ? static_cast<unsigned>(off) : kNowhere;
        }
      }
      const unsigned room = static_cast<unsigned>(
          reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds));
      // the `step`-th share of a chunk's moves; the last one goes on to the next chunk
      const auto issue = [&](int c, int step) {
        const int left = k_left < KE ? static_cast<int>(k_left) : KE;
        const unsigned to = room + (c % STAGES) * kStage;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          if (j < step * kLoads / kSteps || j >= (step + 1) * kLoads / kSteps) continue;
          const int move = (wave + j * kWaves) % kMoves;
          const uintptr_t base = reinterpret_cast<uintptr_t>(of_a(move) ? a : b);
          const u4_t buffer = {static_cast<unsigned>(base), static_cast<unsigned>(base >> 32) & 0xFFFFu, kNowhere - 1u,
                               0x00020000u};
          unsigned off = offset[j];
          if (left < KE && ks[j] >= left) off = kNowhere;
          to_lds(buffer, off, to + move * 1024);
        }
        if (step == kSteps - 1) advance();
      };
#pragma unroll
      for (int c = 0; c < STAGES - 1; ++c)
        if (c < chunks)
#pragma unroll
          for (int step = 0; step < kSteps; ++step) issue(c, step);
      if (chunks == 1 && K <= KE / kSteps) {  // a step is all there is
        wait<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        multiply<1>(lds, [](int) {});
        chunks = 0;
      }
#pragma unroll 1
      for (int c = 0; c < chunks; ++c) {
        // this chunk is there, and nobody reads the one before it any more
        if (c + STAGES - 2 < chunks)
          wait<(STAGES - 2) * kLoads>();
        else
          wait<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        multiply(lds + (c % STAGES) * kStage, [&](int step) {
          if (c + STAGES - 1 < chunks) issue(c + STAGES - 1, step);
        });
      }
      wait<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      join_sums();
    } else {
      u4_t held[kLoads];
      const auto fetch = [&] {
        const int left = k_left < KE ? static_cast<int>(k_left) : KE;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int move = (wave + j * kWaves) % kMoves;
          int64_t off;
          int row, k;
          bool in;
          int whole;   // elements of the pack that are there
          if (of_a(move)) {
            source<A_TURNED, MT, kOwnA, TM>(move * 1024 + lane * 16, A.stride, off, row, k);
            in = row < m_left && k < left;
            whole = A_TURNED ? static_cast<int>(m_left - row < kVec ? m_left - row : kVec) : left - k;
          } else {
            source<B_TURNED, NT, kOwnB, TN>(move * 1024 - kBytesA + lane * 16, B.stride, off, row, k);
            in = row < n_left && k < left;
            whole = B_TURNED ? static_cast<int>(n_left - row < kVec ? n_left - row : kVec) : left - k;
          }
          const char* const from = (of_a(move) ? a : b) + off;
          u4_t x = {0u, 0u, 0u, 0u};
          if (in) {
            if (whole >= kVec) {
              __builtin_memcpy(&x, from, 16);
            } else {
              Pack<T, kVec> y{};
#pragma unroll
              for (int e = 0; e < kVec; ++e)
                if (e < whole) y.v[e] = reinterpret_cast<const T*>(from)[e];
              x = __builtin_bit_cast(u4_t, y);
            }
          }
          held[j] = x;
        }
        advance();
      };
      const auto put = [&](int c) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int move = (wave + j * kWaves) % kMoves;
          *reinterpret_cast<u4_t*>(lds + (c & 1) * kStage + move * 1024 + lane * 16) = held[j];
        }
      };
      fetch();
      put(0);
#pragma unroll 1
      for (int c = 0; c < chunks; ++c) {
        if (c + 1 < chunks) fetch();
        __syncthreads();
        multiply(lds + (c & 1) * kStage, [](int) {});
        if (c + 1 < chunks) put(c + 1);
      }
      __syncthreads();
      join_sums();
    }
  }

  // 16 bytes a lane from `off` on (0 behind the buffer's end) to LDS at `to` + 16 lane.
  static __device__ __forceinline__ void to_lds(u4_t buffer, unsigned off, unsigned to) {
    u4_t b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __builtin_amdgcn_readfirstlane(buffer[i]);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(b)
                 : "memory", "m0");
  }
  // At most LEFT loads of this wavefront are on their way, and its reads of LDS are done.
  template <int LEFT>
  static __device__ __forceinline__ void wait() {
    static_assert(LEFT < 64, "the counter ends at 63");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
  }

  typedef T vec8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f4_t mfma(u4_t a, u4_t b, f4_t c) {
    if constexpr (std::is_same_v<T, bf16_t>)
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
  }
  // fp32, small tiles: a sum is kept in kParts parts, which take the fours of K in
  // turn and are added at the end, so that fewer roundings meet a large sum: dw
  // of 6,151 rows 5.0e-7 off instead of 1.4e-6, dh of 712 tokens 1.3e-7 instead of
  // 3.4e-7, for 2 to 9 % of the time.  (Of large tiles two parts cost 5 to 8 %.)
  static constexpr int kParts = sizeof(T) == 2 || MT * NT > 4 ? 1 : 8;
  f4_t more[kParts > 1 ? kParts - 1 : 1][MT][NT];
  __device__ __forceinline__ void add_product(int step, int i, int j, u4_t a, u4_t b) {
    if constexpr (sizeof(T) == 2) {
      acc[i][j] = mfma(a, b, acc[i][j]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int part = (4 * step + e) % kParts;
        f4_t& c = part == 0 ? acc[i][j] : more[part > 0 ? part - 1 : 0][i][j];
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void clear_sums() {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        acc[i][j] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 1; p < kParts; ++p) more[p - 1][i][j] = f4_t{0.f, 0.f, 0.f, 0.f};
      }
  }
  __device__ __forceinline__ void join_sums() {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int p = 1; p < kParts; ++p) acc[i][j] += more[p - 1][i][j];
  }

  // A wavefront's operands of one step: 64 bytes of K, of which the lane's
  // quarter g has 16 (8 or 4 elements).
  template <bool TURNED, int TILES, int OWN, int SIZE>
  static __device__ __forceinline__ void operands(u4_t (&x)[TILES], const char* part, int first, int step) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    if constexpr (!TURNED) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int row = first + 16 * i + r;
        x[i] = *reinterpret_cast<const u4_t*>(part + row * KB + (((4 * step + g) ^ swapped(row)) << 4));
      }
    } else if constexpr (sizeof(T) == 2) {
      static_assert(OWN % 2 == 0, "elements are swapped in pairs");
#pragma unroll
      for (int j = 0; j < TILES / OWN; ++j) {
        unsigned v[8][OWN / 2];
        const char* const p = part + (32 * step + 8 * g) * SIZE * 2 + (first + 16 * OWN * j + OWN * r) * 2;
#pragma unroll
        for (int k = 0; k < 8; ++k) __builtin_memcpy(&v[k][0], __builtin_assume_aligned(p + k * SIZE * 2, 2 * OWN), 2 * OWN);
#pragma unroll
        for (int e = 0; e < OWN; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[j * OWN + e][k] =
                __builtin_amdgcn_perm(v[2 * k + 1][e / 2], v[2 * k][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < TILES / OWN; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          unsigned v[OWN];
          const char* const p = part + (16 * step + 4 * g + k) * SIZE * 4 + (first + 16 * OWN * j + OWN * r) * 4;
          __builtin_memcpy(&v[0], __builtin_assume_aligned(p, 4 * OWN), 4 * OWN);
#pragma unroll
          for (int e = 0; e < OWN; ++e) x[j * OWN + e][k] = v[e];
        }
    }
  }

  static __device__ __forceinline__ int wave_m() { return (threadIdx.x >> 6) % WAVES_M * 16 * MT; }
  static __device__ __forceinline__ int wave_n() { return (threadIdx.x >> 6) / WAVES_M * 16 * NT; }

  // A chunk's products; f(step) is called once a step's operands are asked of LDS.
  // Moves of the next chunk go there, so that they do not delay these, in equal
  // shares, and a wavefront that multiplies goes before one that reads (bf16,
  // 2,048 x 49,152 x 4,096 at 256 x 256: 725 us with all moves in front, 678 in
  // shares, 637 in shares and by priority; 10,000 x 32,768 x 2,048: 1,189, 1,129, 1,093).
  template <int STEPS = kSteps, class F>
  __device__ __forceinline__ void multiply(const char* stage, F f) {
#pragma unroll
    for (int step = 0; step < STEPS; ++step) {
      u4_t a[MT], b[NT];
      operands<B_TURNED, NT, kOwnB, TN>(b, stage + kBytesA, wave_n(), step);
      operands<A_TURNED, MT, kOwnA, TM>(a, stage, wave_m(), step);
      f(step);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) add_product(step, i, j, a[i], b[j]);
      __builtin_amdgcn_s_setprio(0);
    }
  }

  // What a lane has of the tile: for each n = col(t) the rows run(j) .. run(j) + 4 kOwnA - 1 of A,
  // of which the i-th is at(j, i, t).
  static constexpr int kRuns = MT / kOwnA, kRun = 4 * kOwnA;
  static __device__ __forceinline__ int run_of(int j) {
    return wave_m() + 16 * kOwnA * j + 4 * kOwnA * ((threadIdx.x & 63) >> 4);
  }
  static __device__ __forceinline__ int col_of(int t) {
    return wave_n() + 16 * kOwnB * (t / kOwnB) + kOwnB * (threadIdx.x & 15) + t % kOwnB;
  }
  __device__ __forceinline__ float at(int j, int i, int t) const { return acc[j * kOwnA + i % kOwnA][t][i / kOwnA]; }

  // The tile's columns t of the wavefront, 16 rows of C^T of 16 MT elements of
  // type O each, by way of LDS so that 16 bytes a lane lie on end in memory
  // (straight from the registers they would be 64 or more apart): value(j, i)
  // gives the element, store(n, m, pack) takes 16 / sizeof(O) of them from row m
  // of A on for row n of B.  Call it behind run(); lds as there.
  template <class O, class V, class F>
  __device__ __forceinline__ void rows_out(char* lds, int t, V value, F store) const {
    constexpr int kPack = kRun * static_cast<int>(sizeof(O)) < 16 ? kRun : 16 / static_cast<int>(sizeof(O));
    constexpr int kPieces = 16 * MT / kPack, kBytes = kPack * static_cast<int>(sizeof(O));
    static_assert(kWaves * 16 * 16 * MT * static_cast<int>(sizeof(O)) <= kStage, "a wavefront's rows fit");
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    char* const room = lds + wave * (16 * kPieces * kBytes);
    const auto at_piece = [&](int row, int piece) {
      return room + (row * kPieces + (piece ^ (kPieces >= 16 ? row & 15 : row & (kPieces - 1)))) * kBytes;
    };
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < kRuns; ++j)
#pragma unroll
      for (int i = 0; i < kRun; i += kPack) {
        Pack<O, kPack> x;
#pragma unroll
        for (int e = 0; e < kPack; ++e) x.v[e] = value(j, i + e);
        __builtin_memcpy(__builtin_assume_aligned(at_piece(r, (16 * kOwnA * j + 4 * kOwnA * g + i) / kPack), kBytes), &x,
                         kBytes);
      }
    __builtin_amdgcn_wave_barrier();
    const int first = wave_n() + 16 * kOwnB * (t / kOwnB) + t % kOwnB;
#pragma unroll
    for (int at = 0; at < 16 * kPieces; at += 64) {
      const int row = (at + lane) / kPieces, piece = (at + lane) % kPieces;
      Pack<O, kPack> x;
      __builtin_memcpy(&x, __builtin_assume_aligned(at_piece(row, piece), kBytes), kBytes);
      store(first + kOwnB * row, wave_m() + piece * kPack, x);
    }
  }
};

// Whether a product's direct loads can take an operand: whole aligned packs, offsets within 2^31 bytes.
template <class T>
inline bool direct_operand(const void* p, int64_t stride, int64_t inner, int64_t tile_rows) {
  constexpr int kVec = 16 / sizeof(T);
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % kVec == 0 && inner % kVec == 0 &&
         stride <= (int64_t(1) << 30) / static_cast<int64_t>(sizeof(T)) / tile_rows;
}

// The tile of workgroup `number` of tiles_m x tiles_n: the workgroups of an XCD (every eighth)
// take tiles on end, eight rows of tiles by all columns at a time, so that those that run
// together share operands in its cache.
struct TileAt {
  int m, n;
};
__device__ __forceinline__ TileAt tile_at(unsigned number, unsigned tiles_m, unsigned tiles_n) {
  const unsigned all = tiles_m * tiles_n, xcd = number % 8, each = all / 8, more = all % 8;
  const unsigned p = xcd * each + (xcd < more ? xcd : more) + number / 8;
  constexpr unsigned kRows = 8;
  const unsigned band = p / (kRows * tiles_n), in = p - band * kRows * tiles_n;
  const unsigned rows = tiles_m - band * kRows < kRows ? tiles_m - band * kRows : kRows;
  return TileAt{static_cast<int>(band * kRows + in % rows), static_cast<int>(in / rows)};
}

}  // namespace gnnshap
