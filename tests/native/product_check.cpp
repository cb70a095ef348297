// What the tiled products copy to LDS (product_index.h), on the CPU, as the kernel goes through it.
//   product_check ROWS_A ROWS_B COLS SH_A SH_B TILE QUARTERS AHEAD
// Items: every tile of c (every quarter of tiles of twice the size with QUARTERS, so that some lie outside of c), the column
// blocks in one part or in two, one item after another, copies AHEAD blocks ahead of the products.
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

struct Item {
  uint32_t m0, n0, j0, j1;
};

// Copies of `size` bytes at a lane's offset and a scalar one, from a buffer of `length` bytes that begins at `begin` of the
// operand: nothing where the lane's offset is not below length - scalar in 32 bits, which must not wrap.
static bool inside(uint32_t lane, uint32_t scalar, uint32_t length) {
  CHECK(scalar <= length, "a scalar offset of %u in a buffer of %u bytes", scalar, length);
  return lane < length - scalar;
}

static void check_operand(const QView& q, const uint8_t* base, uint32_t bytes, uint32_t codes, uint32_t block, uint32_t tile, uint32_t kb,
                          int64_t first, bool wanted) {
  const int64_t padded = (int64_t)kb * 128;
  const uint32_t scale_bytes = (kb + 3) / 4 * q.srows * 4, scale_at = codes + block / 4 * q.srows * 4;
  for (uint32_t row = 0; row < tile; ++row) {
    for (uint32_t piece = 0; piece < 8; ++piece) {
      const uint32_t lane = row * (uint32_t)q.stride + piece * 16;
      const bool in = inside(lane, block * 128, bytes);
      if (wanted) CHECK(in == (first + row < q.rows), "row %u of the tile at %lld", row, (long long)first);
      if (!in) continue;
      const int64_t at = base - q.data + lane + (int64_t)block * 128;
      CHECK(at / q.stride < q.rows && at % q.stride + 16 <= padded, "byte %lld of the data", (long long)at);
      if (wanted) CHECK(at == (first + row) * q.stride + (int64_t)block * 128 + piece * 16, "byte %lld of the data", (long long)at);
    }
    const uint32_t lane = 4 * (row >> q.sh);
    if (inside(lane, scale_at, scale_bytes)) CHECK(lane + scale_at + 4 <= scale_bytes, "codes at %u", lane + scale_at);
    if (wanted && first + row < q.rows)
      CHECK(lane + scale_at == 4 * ((uint64_t)(block / 4) * q.srows + ((first + row) >> q.sh)), "codes of row %lld", (long long)first + row);
  }
}

int main(int argc, char** argv) {
  if (argc != 9) return 2;
  auto arg = [&](int i) { return (uint32_t)std::strtoul(argv[i], nullptr, 0); };
  const uint32_t rows[2] = {arg(1), arg(2)}, cols = arg(3), sh[2] = {arg(4), arg(5)}, tile = arg(6), quarters = arg(7), ahead = arg(8);
  const uint32_t kb = (cols + 127) / 128;
  std::vector<uint8_t> data[2];
  QView q[2];
  for (int i = 0; i < 2; ++i) {
    const int64_t stride = (int64_t)kb * 128 + 16 * i;
    data[i].resize(rows[i] * stride);
    q[i] = QView{data[i].data(), nullptr, stride, rows[i], cols, (rows[i] + (1u << sh[i]) - 1) >> sh[i], (int32_t)sh[i]};
  }
  std::vector<Item> items;
  const uint32_t big = tile << quarters;
  for (uint32_t parts = 1; parts <= 2 && kb >= parts * ahead; ++parts)
    for (uint32_t part = 0; part < parts; ++part)
      for (uint32_t m = 0; m < (rows[0] + big - 1) / big * big; m += tile)
        for (uint32_t n = 0; n < (rows[1] + big - 1) / big * big; n += tile)
          items.push_back({m, n, kb * part / parts, kb * (part + 1) / parts});

  auto source_of = [&](const Item& t) { return product_source(q[0], q[1], tile, tile, t.m0, t.n0, t.j0, t.j1); };
  // what is copied, in order, must be every item's blocks, and nothing behind them
  size_t copying = 0;
  uint32_t block = items[0].j0;
  ProductSource source = source_of(items[0]), upcoming = source;
  auto copy = [&] {
    const bool any = copying < items.size();
    const Item t = any ? items[copying] : items.back();
    CHECK(source.block == (any ? block : 0), "block %u, copied %u", block, source.block);
    check_operand(q[0], source.a, source.abytes, source.acodes, source.block, tile, kb, t.m0, any && t.m0 < rows[0]);
    check_operand(q[1], source.b, source.bbytes, source.bcodes, source.block, tile, kb, t.n0, any && t.n0 < rows[1]);
    if (!any) CHECK(!source.abytes && !source.bbytes, "copies behind the last item");
    if (any && ++block == t.j1 && ++copying < items.size()) block = items[copying].j0;
  };
  for (uint32_t i = 0; i < ahead; ++i) {
    if (i) next_block(source, upcoming);
    copy();
  }
  for (size_t i = 0; i < items.size(); ++i) {
    const bool more = i + 1 < items.size();
    upcoming = source_of(items[more ? i + 1 : i]);
    if (!more) no_product_source(upcoming);
    for (uint32_t j = items[i].j0; j < items[i].j1; ++j) {
      next_block(source, upcoming);
      copy();
    }
  }
  CHECK(copying == items.size(), "copied %zu of %zu items", copying, items.size());
  std::printf("%zu items, %d errors\n", items.size(), errors);
  return errors != 0;
}
