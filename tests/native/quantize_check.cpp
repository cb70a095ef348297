// Which sources of dr_quantize are streamed, and where the loads of their rows begin, on the CPU.
// Exit status 0 when every streamed load begins at whole 16 bytes.
#include <cstdio>
#include <initializer_list>

#include "quant_kernels.h"

using namespace dr;

int main() {
  int errors = 0, streamed = 0, cases = 0;
  for (int64_t size : {2, 4})
    for (uint32_t cols = 8; cols < 3000; cols += cols < 600 ? 1 : 37)
      for (int64_t stride : {(int64_t)cols, (int64_t)cols + 1, ceil_div(cols, 8) * 8, ceil_div(cols, 4) * 4, ceil_div(cols, 8) * 8 + 8})
        for (uintptr_t base : {1u << 20, (1u << 20) + (unsigned)size, (1u << 20) + 8u}) {
          if (stride < cols) continue;
          ++cases;
          if (!whole_pieces(reinterpret_cast<const void*>(base), stride, cols, size)) continue;
          ++streamed;
          for (int64_t row : {0, 1, 2, 7})
            for (uint32_t col = 0; col < ceil_div(cols, 512) * 512; col += 8)  // the first column of load_row8
              errors += (base + (row * stride + (col < cols - 8 ? col : cols - 8)) * size) % 16 != 0;
        }
  std::printf("%d of %d sources streamed, %d errors\n", streamed, cases, errors);
  return errors || !streamed;
}
