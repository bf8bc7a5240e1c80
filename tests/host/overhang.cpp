// The launches of rows and weights put into 8 bits have more blocks than work where there are
// more than one dimension of a grid holds.  The blocks behind the last row, or the last
// 128 x 128 elements, must touch nothing; the last ones before them do.
#include <stdio.h>

#include "cpu_device.hpp"

#include "quantise.hip"

namespace gg {
void set_error(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vprintf(fmt, ap);
  va_end(ap);
}
int pack_rows(const gg_rows_t* r, const char*, int64_t, int64_t, uint32_t, bool, KRows* out) {
  *out = {(char*)r->data, r->stride, (char*)r->scales, r->scales_stride, r->group};
  return GG_OK;
}
}  // namespace gg
extern "C" hipError_t hipGetLastError() { return hipSuccess; }
extern "C" const char* hipGetErrorString(hipError_t) { return ""; }

static int64_t launched;
static int bad;

// The launches that follow are of `items`, `per_block` to a block.
static void look(const char* what, int64_t items, int64_t per_block) {
  on_launch = [=](dim3 grid, dim3 block, const std::function<void()>& lane) {
    const int64_t blocks = (int64_t)grid.x * grid.y, used = (items + per_block - 1) / per_block;
    ++launched;
    if (blocks < used) {
      printf("%s of %lld: %lld blocks for %lld\n", what, (long long)items, (long long)blocks, (long long)used);
      ++bad;
    }
    const auto touches = [&](int64_t b) {
      for (unsigned t : {0u, 1u, (unsigned)block.x / 2, (unsigned)block.x - 1})
        if (faults(grid, block, b, t, lane)) return true;
      return false;
    };
    for (int64_t b : {(int64_t)0, used / 2, used - 1})
      if (!touches(b)) {
        printf("%s of %lld: block %lld does nothing\n", what, (long long)items, (long long)b);
        ++bad;
      }
    for (int64_t i = 0, over = blocks - used; i < 1000 && over > 0; ++i) {
      const int64_t b = used + (over - 1) * i / 999;
      if (!touches(b)) continue;
      printf("%s of %lld: block %lld of %lld touches memory\n", what, (long long)items, (long long)b,
             (long long)blocks);
      ++bad;
      break;
    }
  };
}

int main(int argc, char** argv) {
  const bool rows = argc > 1 && !strcmp(argv[1], "rows");
  char* p = no_memory(1ull << 40);
  if (!p) return 2;
  const int64_t full = 1 << 21;
  for (const int32_t t : {GG_F32, GG_F16, GG_BF16}) {
    const gg_rows_t x = {p, 0, t, 0, nullptr, 0};
    if (rows) {
      // one scale to a wide row, to a narrow one, and by groups
      for (const int64_t n : {(int64_t)5, full - 1, full, full + 1, full + 3, (int64_t)2'450'000, (int64_t)1 << 27}) {
        const gg_rows_t one = {p, 1024, GG_E4M3, 0, p, 4}, by = {p, 1024, GG_E4M3, 128, p, 64};
        look("wide rows", n, 1);
        if (gg_quantise_rows(&x, n, 1000, &one, nullptr)) ++bad;
        look("narrow rows", n * 16, 1024);       // 16 lanes a row
        if (gg_quantise_rows(&x, n, t == GG_F32 ? 64 : 128, &one, nullptr)) ++bad;
        look("groups of rows", n * (t == GG_F32 ? 256 : 128), 1024);
        if (gg_quantise_rows(&x, n, 1000, &by, nullptr)) ++bad;
      }
    } else {
      for (const int64_t across : {1, 3, 16, 17, 40, 131'072}) {
        const gg_blocks_t q = {p, 1 << 25, p, 1 << 20};
        look("weights", across << 17, 1);
        if (gg_quantise_blocks(&x, 1 << 24, across * 128 - (across % 3), &q, nullptr, nullptr)) ++bad;
        if (gg_quantise_blocks(&x, 1 << 24, across * 128 - (across % 3), nullptr, &q, nullptr)) ++bad;
      }
    }
  }
  printf("%lld launches\n", (long long)launched);
  return bad ? 1 : 0;
}
