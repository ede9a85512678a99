// agcn_row_tiles.hpp on the host: for offsets that keep the rules the tiles cover every
// row once, with its group, and for any others each tile lies inside the matrix.
#include "wave_on_host.hpp"

#include "../paper_2308_11825_amd/csrc/agcn_row_tiles.hpp"

#include <cstdio>
#include <cstdlib>
#include <limits>
#include <random>

namespace {

struct Args {
  int64_t n;
  const int32_t* offsets;
  int32_t groups;
};

void require(bool ok, const char* what, const Args& p, int64_t a, int64_t b) {
  if (ok) return;
  std::printf("%s: n %lld groups %d: %lld %lld\n", what, (long long)p.n, p.groups, (long long)a, (long long)b);
  std::fflush(stdout);
  std::_Exit(1);
}

struct Found {
  agcn::Rows rows;
  uint32_t tn;
};

void inside(const Args& p, const agcn::Rows& r, int bm) {
  if (r.count <= 0) return;
  require(r.row >= 0 && r.row + r.count <= p.n, "rows outside the matrix", p, r.row, r.count);
  require(r.count <= bm, "more rows than a tile has", p, r.row, r.count);
  require(r.group >= -1 && r.group < p.groups, "no such group", p, r.group, 0);
}

// The tiles of the workgroups `blocks` of a launch (all of them: blocks < 0).
template <int BM>
std::vector<Found> tiles(const Args& p, int64_t tiles_n, int64_t blocks, uint32_t first = 0) {
  const int64_t slots = agcn::most_slots(p.n, p.groups, BM);
  gridDim.x = (uint32_t)(slots * tiles_n);
  std::vector<Found> out;
  if (blocks < 0) blocks = gridDim.x;
  out.resize((size_t)blocks);
  run_wave([&] {
    for (int64_t i = 0; i < blocks; ++i) {
      blockIdx.x = first + (uint32_t)i;
      uint32_t tn = 0;
      const agcn::Rows r = agcn::tile_rows<BM, true>(p, (uint32_t)tiles_n, (uint32_t)min<int64_t>(slots, 8), &tn);
      if (threadIdx.x == 0) out[(size_t)i] = {r, tn};
    }
  });
  for (const Found& f : out) {
    inside(p, f.rows, BM);
    require(f.rows.count <= 0 || (int64_t)f.tn < tiles_n, "column tile outside", p, f.tn, tiles_n);
  }
  return out;
}

template <int BM>
std::vector<Found> few(const Args& p, int64_t blocks, uint32_t first = 0) {
  gridDim.y = (uint32_t)agcn::few_rows_grid(p.n, p.groups, BM, true);
  std::vector<Found> out;
  if (blocks < 0) blocks = gridDim.y;
  out.resize((size_t)blocks);
  run_wave([&] {
    for (int64_t i = 0; i < blocks; ++i) {
      blockIdx.y = first + (uint32_t)i;
      const agcn::Rows r = agcn::few_rows<BM, true>(p);
      if (threadIdx.x == 0) out[(size_t)i] = {r, 0};
    }
  });
  for (const Found& f : out) inside(p, f.rows, BM);
  return out;
}

// Every row of each column tile once, with its group.
void covers(const Args& p, const std::vector<Found>& found, int64_t tiles_n) {
  std::vector<int> want((size_t)p.n, -1), seen((size_t)(p.n * tiles_n), 0);
  for (int e = 0; e < p.groups; ++e)
    for (int64_t r = p.offsets[e]; r < p.offsets[e + 1]; ++r) want[(size_t)r] = e;
  for (const Found& f : found)
    for (int64_t r = f.rows.row; r < f.rows.row + f.rows.count; ++r) {
      require(want[(size_t)r] == f.rows.group, "another group's rows", p, r, f.rows.group);
      ++seen[(size_t)(f.tn * p.n + r)];
    }
  for (size_t i = 0; i < seen.size(); ++i) require(seen[i] == 1, "a row not once", p, (int64_t)i, seen[i]);
}

template <int BM>
void valid(const Args& p) {
  for (int64_t tiles_n : {1, 3}) covers(p, tiles<BM>(p, tiles_n, -1), tiles_n);
  covers(p, few<BM>(p, -1), 1);
}

// A workgroup's rows among very many groups take few steps: not one per 64 groups.
void many_groups() {
  constexpr int kGroups = 1'000'000;
  std::vector<int32_t> off(kGroups + 1);
  for (int rows : {1, 70}) {
    for (int i = 0; i <= kGroups; ++i) off[(size_t)i] = i * rows;
    const Args p{(int64_t)kGroups * rows, off.data(), kGroups};
    const int64_t slots = agcn::most_slots(p.n, kGroups, 64);
    for (int64_t first : {int64_t{0}, slots / 2, slots - 4}) {
      const int64_t before = wave::exchanges;
      const std::vector<Found> found = tiles<64>(p, 1, 4, (uint32_t)first);
      require(wave::exchanges - before <= 4 * 64 * 40, "steps for four tiles", p, first, wave::exchanges - before);
      for (const Found& f : found)
        if (f.rows.count > 0)
          require(off[(size_t)f.rows.group] <= f.rows.row && f.rows.row + f.rows.count <= off[(size_t)f.rows.group + 1],
                  "another group's rows", p, f.rows.row, f.rows.group);
    }
    const int64_t before = wave::exchanges;
    few<64>(p, 4, (uint32_t)kGroups + 2);
    require(wave::exchanges - before <= 4 * 64 * 40, "steps past the first tiles", p, 0, wave::exchanges - before);
  }
}

// Launches of the quantiser: fewer than 2^32 threads, and at least a row.
void quantizer_launches() {
  for (int64_t blocks : {1, 2, 3, 1000, 131071, 131072}) {
    const int64_t rows = agcn::most_quantized_rows(blocks);
    const int64_t threads = (rows * blocks + 15) / 16 * 256;
    require(rows >= 1 && threads < (int64_t{1} << 32), "a launch too large", Args{rows, nullptr, 0}, blocks, threads);
  }
}

}  // namespace

int main() {
  quantizer_launches();
  many_groups();
  std::mt19937 rng(1);
  for (int groups : {0, 1, 5, 62, 63, 130, 254, 255, 1000, 4000}) {
    for (int n : {1, 64, 500, 1500}) {
      if (groups > 200 ? n != (groups == 255 ? 1500 : 64) : n > 500) continue;
      std::vector<int32_t> off((size_t)groups + 1);
      for (int kind = 0; kind < 3; ++kind) {  // spread, most of them empty, all rows in one group
        for (int32_t& o : off)
          o = kind == 0 ? (int32_t)(rng() % (unsigned)(n + 1)) : kind == 1 ? (int32_t)(rng() % 3 * (unsigned)n / 2) : 0;
        std::sort(off.begin(), off.end());
        if (kind == 2) std::fill(off.begin() + (groups + 1) / 2, off.end(), n);
        const Args p{n, off.data(), groups};
        valid<16>(p);
        valid<64>(p);
      }
    }
  }
  // Parts that overlap, so that their tiles are far more than any rows can have.
  constexpr int32_t kMost = std::numeric_limits<int32_t>::max(), kLeast = std::numeric_limits<int32_t>::min();
  for (int64_t n : {int64_t{1000}, int64_t{900'000}, int64_t{500'000'000}, int64_t{kMost}}) {
    for (int groups : {3, 150, 700}) {
      std::vector<int32_t> off((size_t)groups + 1);
      for (int kind = 0; kind < 4; ++kind) {
        for (size_t i = 0; i < off.size(); ++i)
          off[i] = kind == 0 ? (i % 2 ? (int32_t)n : 0) : kind == 1 ? (i % 2 ? 0 : (int32_t)n)
                 : kind == 2 ? (i % 2 ? kMost : kLeast) : (int32_t)rng();
        const Args p{n, off.data(), groups};
        const int64_t slots = agcn::most_slots(n, groups, 64);
        for (int64_t first : {int64_t{0}, slots / 2, slots - 8})
          if (first >= 0 && slots <= agcn::kMostTiles)  // (others are not launched)
            tiles<64>(p, 1, min<int64_t>(8, slots - first), (uint32_t)first);
        const int64_t y = agcn::few_rows_grid(n, groups, 16, true);
        for (int64_t first : {int64_t{0}, (int64_t)groups, y - 8})
          if (first >= 0 && y <= 65535)
            few<16>(p, min<int64_t>(8, y - first), (uint32_t)first);
      }
    }
  }
  std::printf("row tiles check ok\n");
  return 0;
}
