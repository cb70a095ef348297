// What the products of pairs copy to LDS of the fused weights (product_index.h), on the CPU, as the kernel addresses it.
//   gated_check F COLS SH TILE
// Every tile of TILE rows of b (TILE / 2 pairs), tiles behind the last pair among them (the parts of a cut tile may lie there).
// Exit status 0 when everything holds.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "product_index.h"

static int errors = 0;
#define CHECK(c, ...)                                   \
  do {                                                  \
    if (!(c)) {                                         \
      if (errors < 20) {                                \
        std::fprintf(stderr, "FAIL %s: ", #c);          \
        std::fprintf(stderr, __VA_ARGS__);              \
        std::fprintf(stderr, "\n");                     \
      }                                                 \
      ++errors;                                         \
    }                                                   \
  } while (0)

using namespace dr;

int main(int argc, char** argv) {
  if (argc != 5) return 2;
  auto arg = [&](int i) { return (uint32_t)std::strtoul(argv[i], nullptr, 0); };
  const uint32_t f = arg(1), cols = arg(2), sh = arg(3), tile = arg(4), kb = (cols + 127) / 128;
  const int64_t stride = (int64_t)kb * 128 + 16;
  std::vector<uint8_t> data(2 * f * stride), adata(kb * 128);
  const QView a{adata.data(), nullptr, (int64_t)kb * 128, 1, cols, 1, 0};
  const QView b{data.data(), nullptr, stride, f, cols, (2 * f + (1u << sh) - 1) >> sh, (int32_t)sh};  // gate's rows
  const int64_t half_bytes = f * stride;
  const uint32_t scale_bytes = (kb + 3) / 4 * b.srows * 4;
  uint64_t copies = 0;
  for (uint32_t n0 = 0; n0 < f + tile; n0 += tile / 2) {
    ProductSource s = product_source(a, b, 128, tile / 2, 0, n0, 0, kb), none = s;
    no_product_source(none);
    for (uint32_t block = 0; block <= kb; ++block, next_block(s, none)) {
      const bool behind = block == kb;  // copies of nothing
      CHECK(s.block == (behind ? 0 : block), "block %u, copied %u", block, s.block);
      for (uint32_t at = 0; at < tile; ++at) {
        const uint32_t pair = pair_of(at), second = second_of(at);
        CHECK(pair < tile / 2, "pair %u of row %u", pair, at);
        const uint8_t* base = s.b + (second ? half_bytes : 0);
        for (uint32_t piece = 0; piece < 8; ++piece) {
          const uint32_t lane = pair * (uint32_t)stride + piece * 16;
          CHECK(s.block * 128 <= s.bbytes, "a scalar offset of %u in a buffer of %u bytes", s.block * 128, s.bbytes);
          const bool in = lane < s.bbytes - s.block * 128;
          if (behind) {
            CHECK(!in, "copies behind the last item");
            continue;
          }
          if (n0 < f) CHECK(in == (n0 + pair < f), "pair %u of the tile at %u", pair, n0);
          if (!in) continue;
          ++copies;
          const int64_t byte = base - data.data() + lane + (int64_t)s.block * 128;
          CHECK(byte >= 0 && byte + 16 <= (int64_t)data.size() && byte % stride + 16 <= (int64_t)kb * 128, "byte %lld of the data", (long long)byte);
          CHECK(byte / stride / f == second, "row %lld is not of half %u", (long long)(byte / stride), second);
          if (n0 < f) CHECK(byte == ((int64_t)second * f + n0 + pair) * stride + (int64_t)block * 128 + piece * 16, "byte %lld", (long long)byte);
        }
        const uint32_t code = pair_code_at(s.bfirst, pair + second * f, (int32_t)sh), plane = s.block / 4 * b.srows * 4;
        CHECK(plane <= scale_bytes, "a scalar offset of %u in a buffer of %u bytes", plane, scale_bytes);
        if (code < scale_bytes - plane) CHECK(code + plane + 4 <= scale_bytes, "codes at %u", code + plane);
        if (!behind && n0 + pair < f)
          CHECK(code < scale_bytes - plane && code / 4 == (second * f + n0 + pair) >> sh, "code %u of pair %u in half %u", code, n0 + pair, second);
      }
    }
  }
  std::printf("%llu copies, %d errors\n", (unsigned long long)copies, errors);
  return errors != 0;
}
