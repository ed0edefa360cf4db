// Tiles of rows over the blocks of a dispatch, loads straight into LDS, and SwiGLU's
// activation: what the experts' products share.  Internal header.
#pragma once

#include "operators.hpp"

namespace uep {

// v, with what follows from it computed where it is used: a persistent loop would
// otherwise hold every lane's address of its rare parts in registers throughout
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

__device__ __forceinline__ int64_t readlane64(int64_t v, int l) {
  const uint32_t lo = readlane(static_cast<int>(v), l), hi = readlane(static_cast<int>(v >> 32), l);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// an address that is the same in all lanes, in scalar registers
template <class T>
__device__ __forceinline__ T *uniform(T *p) {
  const uintptr_t v = reinterpret_cast<uintptr_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<T *>(static_cast<uintptr_t>(hi) << 32 | lo);
}

// A tile of rows of one block: its first row, rows and weight.
struct RowTile {
  int64_t row;
  int32_t rows, w;
};

// Row tiles are numbered block by block.  Blocks are looked at in runs of 64, one a
// lane; a wave holds one run's blocks, and the runs' tile counts, in registers.  Where a
// block is out of order or out of [0, M], or has rows and no weight, that is reported and
// there are no tiles at all, so that what is numbered lies within M rows.  Every lane
// must be active in each call.  Args: block_off, block_w (or null), n_block, n_w, M, status.
template <int kTileRows>
struct RowTiles {
  int64_t lo;               // this lane's block of run `run`:
  int rows, w;              //   its first row, rows, weight
  int before, tiles;        //   its tiles, and the run's before it
  int run, n_run;
  int run_before, run_tiles;  // of run `lane`
  int total;                // tiles in all

  // false (in the whole wave) if a block of run r is not sound
  template <class Args>
  __device__ bool load(const Args &a, int r) {
    run = r;
    bool sound = true;
    const int g = r * kWave + lane_id();
    lo = 0;
    rows = w = 0;
    if (g < a.n_block) {
      lo = a.block_off[g];
      const int64_t hi = a.block_off[g + 1];
      w = a.block_w ? a.block_w[g] : g;
      sound = lo >= 0 && hi >= lo && hi <= a.M && (hi == lo || (w >= 0 && w < a.n_w));
      if (sound)
        rows = static_cast<int>(hi - lo);
      else
        report(a.status, ULTRAEP_EDATA);
    }
    tiles = rows > 0 ? (rows - 1) / kTileRows + 1 : 0;
    before = wave_scan_incl(tiles) - tiles;
    return !ballot(!sound);
  }
  // s_run: 32 words of LDS, free again after the call's last barrier
  template <class Args>
  __device__ void count(const Args &a, int *s_run, int wave, int n_waves) {
    n_run = (a.n_block + kWave - 1) / kWave;
    if (n_run == 1) {
      const bool sound = load(a, 0);
      run_before = 0;
      total = sound ? readlane(before + tiles, kWave - 1) : 0;
      run_tiles = lane_id() == 0 ? total : 0;
      return;
    }
    for (int r = wave; r < n_run; r += n_waves) {
      const bool sound = load(a, r);
      if (lane_id() == kWave - 1) s_run[r] = sound ? before + tiles : -1;
    }
    __syncthreads();
    run_tiles = lane_id() < n_run ? s_run[lane_id()] : 0;
    __syncthreads();
    run_before = wave_scan_incl(run_tiles) - run_tiles;
    total = readlane(run_before, kWave - 1);  // (fewer than 64 runs)
    if (ballot(run_tiles < 0)) total = 0;
    run = -1;
  }
  // tile < total
  template <class Args>
  __device__ RowTile find(const Args &a, int tile) {
    int t = tile;
    if (n_run > 1) {
      const int r = __builtin_ctzll(ballot(tile >= run_before && tile < run_before + run_tiles));
      t -= readlane(run_before, r);
      if (r != run) load(a, r);
    }
    const int l = __builtin_ctzll(ballot(t >= before && t < before + tiles));
    const int first = (t - readlane(before, l)) * kTileRows;
    return {readlane64(lo, l) + first, min(readlane(rows, l) - first, kTileRows), readlane(w, l)};
  }
};

// 16 bytes a lane from base + off straight into LDS, lane l's at lds + 16 l.
// The wait for it is the caller's (vmcnt).  A scalar register that the vector ALU wrote may be an
// address 5 instructions later, which the compiler does not see to here; in the built code
// they lie further apart (tests/test_written_out.py).
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

// The same from a buffer of `range` bytes at `base`, to lds + at; where the offset is out of
// range, as kBufferBytes always is, zeros are written.  `past` is added to an offset bit by
// bit.
constexpr uint32_t kBufferBytes = 1u << 31;
__device__ __forceinline__ v4i buffer_of(const void *base, uint32_t range) {
  const uint64_t at = reinterpret_cast<uintptr_t>(base);
  // (address, no stride; bytes; raw 32-bit data)
  return v4i{static_cast<int>(at), static_cast<int>(at >> 32 & 0xFFFF), static_cast<int>(range), 0x00020000};
}
__device__ __forceinline__ void buffer_to_lds(const void *base, uint32_t range, uint32_t off, uint32_t lds, int at) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(buffer_of(base, range)), "n"(at)
               : "memory", "m0", "scc");
}
__device__ __forceinline__ void buffer_to_lds(const void *base, uint32_t range, uint32_t off, uint32_t past,
                                              uint32_t lds, int at) {
  uint32_t from;
  asm volatile("s_add_u32 m0, %1, %5\n\tv_or_b32 %0, %2, %3\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds"
               : "=&v"(from)
               : "s"(lds), "v"(off), "v"(past), "s"(buffer_of(base, range)), "n"(at)
               : "memory", "m0", "scc");
}

// 4 bytes a lane, as the first
__device__ __forceinline__ void load_word_to_lds(const void *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
template <class T>
__device__ __forceinline__ uint32_t lds_address(T *p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) T *)p));
}

// v / (1 + exp(-v)) by the hardware's exp2 and reciprocal: a relative error of
// (1.23 |v| + 6) 2^-24 at most (exp's, 1 of the sum, 2 of the reciprocal, 1 of the product) for
// v >= -87.3; below, where it is under 2e-36 in magnitude, it becomes 0.  |v| 2^-24 is far below the
// rounding of 8-bit operands or of a bf16 result, and fp32 results are held to it; with expf and
// a division the epilogue's arithmetic costs 65 us of 3350 at 131072 x 4096 x 7168 in 8-bit integers.
__device__ __forceinline__ float silu(float v) { return v * fast_rcp(1.f + fast_exp(-v)); }

}  // namespace uep
