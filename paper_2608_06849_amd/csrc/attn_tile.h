// Tiles of 64 keys in LDS, shared by the attention kernels that stage K/V there: direct
// loads, waits and the swizzle of token-major rows.
#pragma once
#include "aoh_device.h"

namespace aoh {

constexpr int kBN = 64;          // keys per tile

// Swizzle of a tile's rows: chunk c of row r is stored at c ^ kx(r) in a K
// tile and c ^ vx(r) in a V tile.  K operands are read 16 bytes a lane down 32
// rows: 16 consecutive rows take 16 different 16-byte columns of the 64 banks
// (a row of d_head 64 spans half of them, so two rows share a pattern).  V
// operands are read as 4 rows x 64 bytes a half wave: the four land in
// different quarters.
template <int D>
struct PPTile {
  static constexpr int kChunks = D / 8;                     // 16-byte chunks of a row
  static constexpr uint32_t kBytes = kBN * D * 2;           // one K or V tile
  static __device__ __forceinline__ int kx(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int vx(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }
  static __device__ __forceinline__ int koff(int r, int c) { return r * D + 8 * (c ^ kx(r)); }
  static __device__ __forceinline__ int voff(int r, int c) { return r * D + 8 * (c ^ vx(r)); }
};

// Direct global -> LDS load of 16 bytes per lane: lane L's bytes land at
// lds_row + 16 L (one contiguous 1 KB block per wave).  Issued as inline
// assembly so that the compiler does not treat every later LDS read as
// possibly depending on it (it would wait for all outstanding loads before
// each one); the kernel orders these loads itself with s_waitcnt and barriers.
// Nor does it count hazards in there: a write of M0 needs one wait state before the
// load, and the write comes right before it.
__device__ __forceinline__ void lds_dma16(const void* gptr, const void* lds_row) {
  const uint32_t m0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds_row));
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(gptr), "{m0}"(m0) : "memory");
}

// s_waitcnt immediates (gfx9 encoding: vmcnt [3:0] and [15:14], expcnt [6:4],
// lgkmcnt [11:8]); a field at its maximum does not wait.
constexpr int kWaitVm0 = 0x0 | (0x7 << 4) | (0xF << 8);
constexpr int wait_vm(int n) { return n | (0x7 << 4) | (0xF << 8); }  // n < 16
constexpr int kWaitLgkm0 = 0xF | (0x7 << 4) | (0x0 << 8) | (0x3 << 14);

}  // namespace aoh
