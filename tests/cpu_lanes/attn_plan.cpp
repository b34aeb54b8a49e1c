// attn_plan.cpp -- what cross attention launches, over the sizes that its
// entry points take: the launches are recorded, not run.  Each keeps to what a
// launch may have (below 2^32 threads along x, below 2^16 blocks along y), has
// a block for every unit of its work, and every block its own; the workspace
// holds the sums of its parts.  Prints a line per check; exits 1 if one fails.
#include "lanes.h"

#include <stdio.h>

#include <random>

#define __ballot(v) ((uint64_t)(v))
#define __popcll(v) __builtin_popcountll(v)
#define __builtin_amdgcn_logf log2f

#include "../../paper_2512_00385_amd/csrc/ezsp_attn.h"

namespace ezsp {

struct Launch {
  const char *kernel;
  dim3 grid, block;
  Attn a;
};
std::vector<Launch> launches;
void record(const char *kernel, dim3 grid, dim3 block, const Attn &a) {
  launches.push_back({kernel, grid, block, a});
}
void prof_begin(const char *, hipStream_t) {}
void prof_end(hipStream_t) {}
void prof_bytes(const char *, double) {}
int check_hip(hipError_t, const char *) { return 0; }

}  // namespace ezsp

#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, st, a) \
  record(#kernel, grid, block, a)
#define hipGetLastError() hipSuccess

#define dispatch dispatch_forward
#include "../../paper_2512_00385_amd/csrc/ezsp_attn_fwd.hip"
#undef dispatch
#define dispatch dispatch_backward
#include "../../paper_2512_00385_amd/csrc/ezsp_attn_bwd.hip"
#undef dispatch

using namespace ezsp;

namespace {

bool ok = true;
void check(bool good, const char *what, const Launch &l) {
  if (good) return;
  ok = false;
  printf("%s: %s, %u x %u blocks, %d x %d, heads %d / %d of %d, %d clouds, "
         "%d parts\n", what, l.kernel, l.grid.x, l.grid.y, l.a.nq, l.a.nk,
         l.a.heads, l.a.kv_heads, l.a.dh, l.a.clouds, l.a.splits);
}
bool is(const Launch &l, const char *name) {
  return strstr(l.kernel, name) != nullptr;
}

struct Call {
  int64_t nq, nk;
  int heads, kv_heads, dh, type;
  int64_t clouds;  // 0: no offsets
};
AttnArgs args_of(const Call &c) {
  static int32_t offsets;  // (not read)
  static float word;
  AttnArgs a = {};
  a.nq = (int32_t)c.nq, a.nk = (int32_t)c.nk;
  a.heads = c.heads, a.kv_heads = c.kv_heads, a.dh = c.dh, a.type = c.type;
  a.n_clouds = (int32_t)c.clouds;
  if (c.clouds) a.q_off = a.k_off = &offsets;
  a.scale = 1.0f;
  a.dk = a.dv = &word;
  return a;
}
// the launches of a call's forward and backward passes, these without dq too
void call(const Call &c) {
  launches.clear();
  AttnArgs a = args_of(c);
  attn_fwd_run(a, nullptr);
  attn_bwd_run(a, nullptr);
  a.dq = a.dk;
  attn_bwd_run(a, nullptr);
}

void check_launches(const Call &c) {
  call(c);
  for (const Launch &l : launches) {
    check((uint64_t)l.grid.x * l.block.x < (uint64_t)1 << 32 &&
              l.grid.y < 1u << 16 && l.grid.z == 1 && l.grid.x > 0 &&
              l.grid.y > 0,
          "past what a launch may have", l);
    const uint64_t blocks = (uint64_t)l.grid.x * l.grid.y;
    check(l.grid.y == 1 || l.grid.x % kXcd == 0, "rows of uneven rounds", l);
    check(blocks <= (uint64_t)1 << 31, "numbers past 32 bits", l);
    if (is(l, "join") || is(l, "delta")) continue;
    check(blocks >= (uint64_t)l.a.tiles * l.a.kv_heads * l.a.splits,
          "fewer blocks than work", l);
  }
}

size_t reserved(const Call &c, bool backward) {
  Arena ar;
  AttnArgs a = {};
  attn_reserve(ar, c.nq, c.nk, c.heads, c.kv_heads, c.dh, backward, &a);
  return ar.off;
}
// what a call's parts and D take is there; and a call with too few keys and
// rows for parts asks for D alone (a piece's alignment apart)
void check_workspace(const Call &c) {
  const size_t forward = reserved(c, false), backward = reserved(c, true);
  const size_t delta = (size_t)c.nq * c.heads * sizeof(float);
  call(c);
  for (const Launch &l : launches) {
    if (l.a.splits == 1) continue;
    const size_t d = width_of((c.dh + 15) / 16), splits = l.a.splits;
    if (is(l, "k_attn_fwd"))
      check(splits * c.nq * c.heads * (d + 2) * sizeof(float) <= forward,
            "forward workspace too small", l);
    if (is(l, "k_attn_dq"))
      check(delta + splits * c.nq * c.heads * d * sizeof(float) <= backward,
            "dq workspace too small", l);
    if (is(l, "k_attn_dkv"))
      check(delta + splits * c.nk * c.kv_heads * 2 * d * sizeof(float) <=
                backward,
            "dk, dv workspace too small", l);
  }
  if (c.nk < 32)
    check(forward == 0, "workspace without parts", launches[0]);
  if (c.nk < 32 && c.nq * c.heads < 16)
    check(backward <= delta + 256, "workspace without parts", launches[0]);
}

// Every tile, head and part has one block, in rows of `row` blocks.
bool each_once(int32_t tiles, int32_t kv_heads, int32_t splits, bool batch,
               unsigned row) {
  const int32_t offsets = 0;
  AttnArgs args = {};
  args.heads = args.kv_heads = kv_heads, args.scale = 1.0f;
  if (batch) args.q_off = args.k_off = &offsets;
  Attn a = attn_of(args);
  a.tiles = tiles, a.splits = splits;
  const unsigned blocks = attn_grid(a);
  lanes::grid.x = std::min(row, blocks);
  lanes::grid.y = (blocks + lanes::grid.x - 1) / lanes::grid.x;
  std::vector<int> seen((size_t)tiles * kv_heads * splits);
  bool in_range = true;
  for (unsigned y = 0; y < lanes::grid.y; ++y)
    for (unsigned x = 0; x < lanes::grid.x; ++x) {
      lanes::block.x = x, lanes::block.y = y;
      int32_t t, h, s;
      if (!unit_of(a, t, h, s)) continue;
      if (t < 0 || t >= tiles || h < 0 || h >= kv_heads || s < 0 ||
          s >= splits)
        in_range = false;
      else
        ++seen[((size_t)t * kv_heads + h) * splits + s];
    }
  return in_range &&
         std::all_of(seen.begin(), seen.end(), [](int n) { return n == 1; });
}

}  // namespace

int main() {
  const int64_t far = ((int64_t)1 << 31) - 256, most = (int64_t)1 << 24;
  std::vector<Call> calls = {
      // the most clouds, the most rows and heads that the entry points take
      {1000, 50, 1, 1, 32, 0, most},       {1000, 50, 1, 1, 32, 1, most},
      {50, 1000, 1, 1, 64, 0, most},       {1000, far, 1, 1, 1, 0, most},
      {far, 1000, 1, 1, 1, 0, most},       {far, far, 1, 1, 1, 0, most / 2},
      {1000, 50, 2, 2, 32, 0, most / 2},   {far, 1, 1, 1, 8, 0, 0},
      {1, far, 1, 1, 8, 0, 0},             {far, far, 1, 1, 8, 0, 0},
      {far, far, 1, 1, 128, 1, 0},         {far / 1024, 7, 1024, 1024, 1, 0, 0},
      {far / 32, 1, 32, 32, 1, 0, 0},      {far / 32, 1, 32, 1, 1, 1, 0},
      {far / 2, 1 << 20, 2, 1, 64, 1, 5000}};
  std::mt19937 gen(1);
  for (int i = 0; i < 20000; ++i) {
    Call c;
    auto up_to = [&](double top) {  // evenly over the logarithm
      return (int64_t)exp(std::uniform_real_distribution<>(0.0, log(top))(gen));
    };
    c.kv_heads = (int)up_to(64.0);
    c.heads = c.kv_heads * (int)up_to(16.0);
    c.dh = 1 + (int)(gen() % 128);
    c.type = (int)(gen() % 2);
    c.nq = std::min(far, up_to(2147480000.0 / c.heads));
    c.nk = std::min(far, up_to(2147480000.0 / c.kv_heads));
    c.clouds = gen() % 2 ? up_to((double)most) : 0;
    const int64_t limit = (int64_t)1 << 25;  // as the entry points check
    if (c.clouds && ((c.nq * (c.heads / c.kv_heads) / 64 + c.clouds + 2) *
                             c.kv_heads >= limit ||
                     (c.nk / 64 + c.clouds + 2) * c.kv_heads >= limit))
      continue;
    calls.push_back(c);
  }
  for (const Call &c : calls) check_launches(c);
  printf("launches of %zu calls: %s\n", calls.size(), ok ? "fit" : "do not fit");
  const bool fit = ok;
  ok = true;
  calls.push_back({70001, 3, 2, 2, 16, 0, 0});
  calls.push_back({7, 31, 2, 1, 128, 1, 0});
  for (const Call &c : calls) check_workspace(c);
  const bool held = ok;
  printf("workspaces: %s\n", held ? "fit" : "do not fit");

  bool once = true;
  for (bool batch : {false, true})
    for (int32_t tiles : {1, 7, 31, 40, 129, 1000})
      for (int32_t heads : {1, 2, 3, 8, 12})
        for (int32_t splits : {1, 2, 5, 64})
          for (unsigned row : {64u, 1024u, kGridRow})
            once &= each_once(tiles, heads, splits, batch, row);
  printf("units: %s\n", once ? "one block each" : "wrong");
  return fit && held && once ? 0 : 1;
}
