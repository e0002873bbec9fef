// Which slices of a tensor group norm keeps in the registers of a workgroup (host arithmetic; gn.hip has the kernels).
#pragma once

namespace acc {

constexpr int kMaxSliceGroups = 256;                   // groups of a slice

struct Slice {
  int hw, c, groups, per;
  int k, s, slices;                                    // groups and channels of a slice, slices of an image
  int tpr, rpi, trips, rest;                           // hw = trips * rpi + rest
  int all;                                             // slices of all images
};

// The slices of a tensor, if they fit: 64 bytes of channels (a line of memory is then read by two workgroups at most) or as many groups as it takes for
// whole threads; 32 bytes where 64 do not fit.  Threads and rows of a workgroup: the fewest threads whose registers hold a slice.  Not where a few workgroups would have long
// slices to work on and the rest of the chip nothing: there the two launches, which cut an image's rows, are faster (forward, us, slices / two launches: 51200 values in a slice, bf16,
// 1 image 40x40 of 512 channels, 16 workgroups 10.0 / 16.2; 100352, bf16 56x56 of 256, 2 images, 16 workgroups 13.6 / 11.8, 8 images, 64 15.4 / 18.0).
// Slices of 32 bytes have 1024 threads, and a compute unit (of 256) holds one such workgroup: their time goes by whole rounds of 256, and a line of memory is read by twice as many
// workgroups, so they pay where they are most of one round and no more.  us, slices / two launches, operands that are in no cache, 128, 176, 192, 256, 304, 512, 1024 workgroups:
//   backward, fp32, 55x55, 128 channels in 16 groups       29 / 22   31 / 29   31 / 30   33 / 40   55 / 45   60 / 60   115 / 90
//   backward, fp32, 56x56, 64 channels in 32               27 / 27   29 / 35   30 / 36   31 / 40   52 / 44   55 / 61   101 / 90
//   backward, bf16, 56x56, 256 in 32                       30 / 27   32 / 33   32 / 35   34 / 48   57 / 53   61 / 62   116 / 104
//   forward, fp32, 80x80, 128 in 16                        28 / 24   30 / 31   31 / 32   34 / 39   55 / 46   63 / 60   123 / 116
//   forward, bf16, 80x80, 256 in 32                        30 / 30   32 / 33   33 / 34   36 / 40   59 / 44   69 / 62   129 / 123
// Of 884 sizes timed both ways (40 to 2048 workgroups, maps of 48x48 to 96x96, both types) the way taken is more than 5 % behind the other in 88 (35 % at
// most, bf16, 48x48 and 50x50 of 512 channels at 448 to 512 workgroups), 1.3 % on average.
constexpr int kSliceGroups = 64, kSliceValues = 60000, kNarrowLeast = 176, kNarrowMost = 256;
struct SliceCfg {
  Slice sl;
  int nt, r;                                           // 0: does not fit
};
// rows of a thread of 1024 that fit 128 registers beside what else it needs
constexpr int slice_rows(int v, bool perch, bool backward) { return !backward ? 20 : v == 4 ? (perch ? 8 : 10) : (perch ? 6 : 8); }
inline SliceCfg slice_cfg(int n, int hw, int c, int groups, int v, int es, bool backward) {
  SliceCfg f{};
  const int per = c / groups;
  if ((long)hw * c * es >= 1L << 32) return f;
  auto fits = [&](int k) {
    const int tpr = k * per / v;
    if (tpr > 256) return false;
    auto rows = [&](int nt) { return (int)(((long)hw + nt / tpr - 1) / (nt / tpr)); };
    const int nt = rows(256) <= (backward ? 4 : 8) ? 256 : rows(512) <= (backward ? 8 : 16) ? 512 : rows(1024) <= slice_rows(v, per % v != 0, backward) ? 1024 : 0;
    if (!nt || (long)n * (groups / k) * nt >= (1L << 32) - 8192) return false;         // (a launch has fewer than 2^32 threads)
    f.nt = nt;
    f.r = rows(nt);
    f.sl = Slice{hw, c, groups, per, k, k * per, groups / k, tpr, nt / tpr, hw / (nt / tpr), hw % (nt / tpr), n * (groups / k)};
    return true;
  };
  int narrow = 0;                                      // the widest slice of 32 bytes or more that is narrower than 64
  for (int k = 1; k <= groups && k <= kMaxSliceGroups; ++k) {
    if (groups % k != 0 || (long)k * per % v != 0) continue;
    const long bytes = (long)k * per * es;
    if (bytes < 64 && k < groups) {
      if (bytes >= 32) narrow = k;
      continue;
    }
    if (fits(k)) {
      if (f.sl.all < kSliceGroups && (long)hw * k * per > kSliceValues) f.nt = 0;
    } else if (narrow && fits(narrow) && (f.sl.all < kNarrowLeast || f.sl.all > kNarrowMost)) {
      f.nt = 0;
    }
    return f;
  }
  return f;
}

}  // namespace acc
