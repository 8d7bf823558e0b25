// Grouped products whose sizes, strides and bases are multiples of 16 bytes, for
// groups of many rows (grouped.h states the products; grouped.hip has the kernels
// for everything else).
//
// A workgroup of eight waves computes 256 x 256 results; the sum advances by
// tiles of 128 bytes (64 bf16 or 128 8-bit values) of both operands, 32 KiB each,
// which go from memory to LDS without passing through registers.  The waves form
// two groups of four, one wave of each to a SIMD.  Group 0 holds result rows 0-127
// and loads operand A, group 1 rows 128-255 and operand B; a wave has 128 x 64
// results.  The groups walk the same tiles one phase apart: in an M phase a wave
// issues its share of the loads and reads the fragments of one tile into
// registers, in a C phase it issues their 32 MFMAs, so that each SIMD's matrix
// pipe is fed by one wave while the other reads:
//   group 0, phase 2t:   M(t): load A tile t+1 (t >= 1), fragments of tile t
//   group 0, phase 2t+1: C(t), then wait until A tile t+1 has landed
//   group 1, phase 2t+1: M(t): load B tile t+2, fragments of tile t, wait until B
//                        tile t+1 has landed
//   group 1, phase 2t+2: C(t)
// A has two LDS stages, B three; a stage is filled again only after both groups
// have read it.
//
// An operand that lies along the sum is kept as 256 rows of 128 bytes; one that
// lies across it as 64 rows of 512 bytes, read with the transposing LDS load.  The
// loads are bounds-checked buffer loads: whatever lies past the sum's end or past
// the last row arrives as zeros.
#include "grouped_fast.h"

namespace eaas {
namespace {

constexpr int kB = 256;               // result rows and columns of a tile
constexpr int kThreads = 512;
constexpr int kStage = 32768;         // bytes of one operand's tile
constexpr int kSA = 2, kSB = 3;       // stages of A and B
constexpr int kLds = (kSA + kSB) * kStage;
constexpr int kInst = 8;              // loads of one wave per tile of its operand

template <int DIR, bool I8>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void grouped_pp_kernel(GroupedParams p) {
  constexpr bool A_ACROSS = DIR == kGradWeights, B_ACROSS = DIR != kForward;
  constexpr int ESZ = I8 ? 1 : 2;
  constexpr int SUM = 128 / ESZ;
  constexpr int MBW = 4, NBW = 2, KK = 4;
  __shared__ __attribute__((aligned(1024))) char smem_raw[kLds];
  GroupedTile t;
  if (!find_tile<DIR, kB, kB, kThreads>(p, reinterpret_cast<int*>(smem_raw), t)) return;

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int grp = wave >> 2, w4 = wave & 3;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)smem_raw);

  const int cols = columns<DIR>(p);
  const int sum_end = DIR == kForward ? p.K : DIR == kGradRows ? p.N : t.end - t.beg;
  const int tiles = ceil_div(sum_end, SUM);
  const int split = blockIdx.y;
  const int first = (int)((long long)tiles * split / p.splits);
  const int nk = (int)((long long)tiles * (split + 1) / p.splits) - first;
  const char* w = p.b + (DIR == kGradWeights ? 0 : (size_t)t.e * p.N * p.K * ESZ);
  const long long a_row = p.lda * ESZ, b_row = p.ldb * ESZ;  // bytes of a row

  // Loads of an operand by the four waves of its group, chunks of 16 bytes swapped
  // within the row as the fragment reads expect them:
  //   along:  instruction q of wave w moves rows (w + 4q)*8 .. +8 (lane l: row l/8,
  //           chunk l%8)
  //   across: instruction q of wave w moves sum rows w*16 + 2q .. +2 (lane l: row
  //           l/32, chunk l%32)
  // along the sum: rows i (gathered, for the forward product's tokens) or j
  const char* along_base = nullptr;
  uint32_t along_off[kInst], along_bytes = 0;
  // across it: columns from i0 or j0
  const char* across_base = nullptr;
  uint32_t across_off[2];
  if (grp == 0 ? !A_ACROSS : !B_ACROSS) {
    const int row0 = lane >> 3;
    const int chunk = (lane & 7) ^ swz_along(w4 * 8 + row0);  // (the same for every q)
    if (grp == 0) {
      const bool gather = DIR == kForward && p.perm;
      along_base = gather ? p.a : p.a + t.i0 * a_row;
      along_bytes = (uint32_t)(((gather ? p.R / p.k : t.i_valid) - 1) * a_row +
                               (long long)sum_end * ESZ);
#pragma unroll
      for (int q = 0; q < kInst; ++q) {
        const int row = min((w4 + 4 * q) * 8 + row0, t.i_valid - 1);
        const int src = gather ? source_row(p, t.i0 + row) : row;
        along_off[q] = (uint32_t)(src * a_row) + chunk * 16;
      }
    } else {
      along_base = w + t.j0 * b_row;
      along_bytes = (uint32_t)(min(kB, cols - t.j0) * b_row);
#pragma unroll
      for (int q = 0; q < kInst; ++q)
        along_off[q] = (uint32_t)(((w4 + 4 * q) * 8 + row0) * b_row) + chunk * 16;
    }
  } else {
    const int h = lane >> 5;
    const long long row = grp == 0 ? a_row : b_row;
    // rows w4*16 + 2q + h; q even and odd differ in the chunks' order
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
      const int r = 2 * odd + h;
      const int chunk = (lane & 31) ^ swz_across(r);
      across_off[odd] = (uint32_t)((grp == 0 ? t.i0 : t.j0) * ESZ + chunk * 16);
      if (!(DIR == kGradWeights && grp == 1 && p.perm))
        across_off[odd] += (uint32_t)((w4 * 16 + r) * row);
    }
    if (grp == 0) across_base = p.a + t.beg * row;
    else if (DIR == kGradRows) across_base = w;
    else across_base = p.perm ? p.b : p.b + t.beg * row;
  }
  // the chunk of the sum that this lane loads, and how many exist in the last tile
  const int my_chunk = (lane & 7) ^ swz_along(w4 * 8 + (lane >> 3));

  auto issue_along = [&](int kt, uint32_t lds) {
    const int at = first + kt;  // tile of the whole sum
    const i32x4 d = descriptor(along_base + (size_t)at * 128, along_bytes - (uint32_t)at * 128);
    const bool in = at * 8 + my_chunk < ceil_div(sum_end * ESZ, 16);
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      load_lds16(d, in ? along_off[q] : kNowhere, lds + (w4 + 4 * q) * 1024);
  };
  auto issue_across = [&](int kt, uint32_t lds, long long row, int width) {
    const int s0 = (first + kt) * 64;
    const int left = min(64, sum_end - s0);
    const i32x4 d = descriptor(across_base + s0 * row,
                               (uint32_t)((left - 1) * row + (long long)width * ESZ));
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      load_lds16(d, across_off[q & 1] + (uint32_t)((q & ~1) * 2 * row), lds + (w4 * 16 + 2 * q) * 512);
  };
  // Gathered rows of x: their slots come through the scalar cache (a vector load
  // here would make the compiler wait for the loads it does not know about), one
  // tile before they are used.
  int slots[2 * kInst];
  auto fetch_slots = [&](int kt) {
    const CONST_AS int32_t* perm = (const CONST_AS int32_t*)p.perm;
    const int s0 = t.beg + (first + kt) * 64 + w4 * 16;
    if (s0 + 2 * kInst <= p.R) {
#pragma unroll
      for (int i = 0; i < 2 * kInst; ++i) slots[i] = perm[s0 + i];
    } else {
#pragma unroll
      for (int i = 0; i < 2 * kInst; ++i) slots[i] = perm[min(s0 + i, p.R - 1)];
    }
  };
  auto issue_gathered = [&](int kt, uint32_t lds) {
    const int left = sum_end - (first + kt) * 64 - w4 * 16;
    const i32x4 d = descriptor(
        across_base, (uint32_t)((p.R / p.k - 1) * b_row + (long long)cols * ESZ));
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      uint32_t at[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t src = token_of(p, slots[2 * q + h]);
        at[h] = 2 * q + h < left ? src * (uint32_t)b_row : kNowhere;
      }
      const uint32_t base = lane < 32 ? at[0] : at[1];
      load_lds16(d, base == kNowhere ? kNowhere : base + across_off[q & 1],
                 lds + (w4 * 16 + 2 * q) * 512);
    }
    if (kt + 1 < nk) fetch_slots(kt + 1);
  };
  auto issue = [&](int kt) {
    if (grp == 0) {
      const uint32_t dst = lds0 + (kt % kSA) * kStage;
      if constexpr (A_ACROSS) issue_across(kt, dst, a_row, p.N);
      else issue_along(kt, dst);
    } else {
      const uint32_t dst = lds0 + (kSA + kt % kSB) * kStage;
      if constexpr (!B_ACROSS) issue_along(kt, dst);
      else if (DIR == kGradWeights && p.perm) issue_gathered(kt, dst);
      else issue_across(kt, dst, b_row, cols);
    }
  };

  // fragment addresses: lane l holds row or column l % 32 of a block and 16 bytes
  // of the sum, half l / 32 of the k-step
  const int lrow = lane & 31, khalf = lane >> 5;
  const int s_l = swz_along(lrow);
  const int tg = lane >> 4, ti = lane & 15;  // transposing load: group of 16, lane in it
  const int t_row = (tg >> 1) * 8 + (ti >> 2);
  const int t_low = (tg & 1) * 2 + ((ti & 3) >> 1);
  const int t_swz = swz_across(ti >> 2);
  int a_at[MBW], b_at[NBW];
#pragma unroll
  for (int i = 0; i < MBW; ++i) {
    const int c0 = grp * 128 + i * 32;
    a_at[i] = A_ACROSS ? t_row * 512 + ((((c0 >> 3) + t_low) ^ t_swz) << 4) + (ti & 1) * 8
                       : (c0 + lrow) * 128;
  }
#pragma unroll
  for (int j = 0; j < NBW; ++j) {
    const int c0 = w4 * 64 + j * 32;
    b_at[j] = B_ACROSS ? t_row * 512 + ((((c0 >> 3) + t_low) ^ t_swz) << 4) + (ti & 1) * 8
                       : (c0 + lrow) * 128;
  }
  typedef typename std::conditional<I8, i32x16, f32x16>::type Acc;
  Acc acc[MBW][NBW];
#pragma unroll
  for (int i = 0; i < MBW; ++i)
#pragma unroll
    for (int j = 0; j < NBW; ++j) acc[i][j] = Acc{};
  const LDS_AS char* smem = (const LDS_AS char*)smem_raw;

  u32x4 fa[KK][MBW], fb[KK][NBW];
  auto fragment = [&](auto across, const LDS_AS char* stage, int at, int kk) {
    if constexpr (decltype(across)::value) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      const LDS_AS char* src = stage + at + kk * 8192;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                     (LDS_AS s16x4*)(src)));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                     (LDS_AS s16x4*)(src + 2048)));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      return *reinterpret_cast<const LDS_AS u32x4*>(stage + at + (((2 * kk + khalf) ^ s_l) << 4));
    }
  };
  auto load_frags = [&](int kt) {
    const LDS_AS char* sa = smem + (kt % kSA) * kStage;
    const LDS_AS char* sb = smem + (kSA + kt % kSB) * kStage;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
      for (int j = 0; j < NBW; ++j)
        fb[kk][j] = fragment(std::integral_constant<bool, B_ACROSS>{}, sb, b_at[j], kk);
#pragma unroll
      for (int i = 0; i < MBW; ++i)
        fa[kk][i] = fragment(std::integral_constant<bool, A_ACROSS>{}, sa, a_at[i], kk);
    }
    // the stage may be filled again right after the next barrier
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  auto mfmas = [&]() {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int i = 0; i < MBW; ++i)
#pragma unroll
        for (int j = 0; j < NBW; ++j) {
          if constexpr (I8)
            acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(
                __builtin_bit_cast(i32x4, fb[kk][j]), __builtin_bit_cast(i32x4, fa[kk][i]),
                acc[i][j], 0, 0, 0);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8, fb[kk][j]), __builtin_bit_cast(bf16x8, fa[kk][i]),
                acc[i][j], 0, 0, 0);
        }
    __builtin_amdgcn_s_setprio(0);
  };
  auto phase_end = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };

  if (nk > 0) {
    if (DIR == kGradWeights && grp == 1 && p.perm) fetch_slots(0);
    // the first two tiles of each operand; tile 0 must have landed before the first
    // barrier
    issue(0);
    if (nk > 1) {
      issue(1);
      wait_vmcnt<kInst>();
    } else {
      wait_vmcnt<0>();
    }
    phase_end();
    // both groups pass 2*nk + 1 barriers: group 1 idles in the first phase, group
    // 0 in the last
    if (grp == 0) {
      for (int kt = 0; kt < nk; ++kt) {
        if (kt >= 1 && kt + 1 < nk) issue(kt + 1);
        load_frags(kt);
        phase_end();
        mfmas();
        wait_vmcnt<0>();
        phase_end();
      }
      phase_end();
    } else {
      phase_end();
      for (int kt = 0; kt < nk; ++kt) {
        if (kt + 2 < nk) issue(kt + 2);
        load_frags(kt);
        if (kt + 2 < nk) wait_vmcnt<kInst>();
        else wait_vmcnt<0>();
        phase_end();
        mfmas();
        phase_end();
      }
    }
  }

  // (the last barrier is behind every wave's fragment reads)
  way_out<DIR, I8, 2>(p, t, split, grp * 128, t.j0 + w4 * 64, acc,
                   (LDS_AS float*)(smem_raw + wave * kWayOutBytes));
}

}  // namespace

template <int DIR, bool I8>
hipError_t launch_grouped_pp(const GroupedParams& p, long long tiles, hipStream_t stream) {
  if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((grouped_pp_kernel<DIR, I8>), dim3((unsigned)tiles, (unsigned)p.splits),
                     dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template hipError_t launch_grouped_pp<kForward, false>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kForward, true>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kGradRows, false>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kGradWeights, false>(const GroupedParams&, long long, hipStream_t);

}  // namespace eaas
