// Host-side checks of csrc/pages_api.cpp (caches in pages) over the stand-in for the HIP runtime; argv[1] names the check.
#include "hip_host_stub.h"

#include "../../paper_2504_09261_amd/csrc/hack_api.cpp"
#include "../../paper_2504_09261_amd/csrc/pages_api.cpp"

#include <random>

namespace stub {
int device = 0;
std::vector<AppendArgs> appends;
struct Attention { AttnPagesArgs a; bool merge; };
std::vector<Attention> attentions;
size_t calls() { return appends.size() + attentions.size(); }
}  // namespace stub

extern "C" hipError_t hipGetDevice(int* d) { *d = stub::device; return hipSuccess; }

namespace hack {
void launch_append(hipStream_t, int, int, bool, int, AppendArgs a) { stub::appends.push_back(a); }
void launch_attn_pages(hipStream_t, int, int, bool merge, AttnPagesArgs a) { stub::attentions.push_back({a, merge}); }
}  // namespace hack

#define CHECK(c)                                    \
  do {                                              \
    if (!(c)) {                                     \
      printf("FAILED line %d: %s\n", __LINE__, #c); \
      return 1;                                     \
    }                                               \
  } while (0)
#define REFUSED(status, call)                       \
  do {                                              \
    const size_t before_ = stub::calls();           \
    CHECK((call) == (status));                      \
    CHECK(stub::calls() == before_);                \
  } while (0)

namespace {

constexpr int kH = 4, kD = 128;
void* const kStream = reinterpret_cast<void*>(0x10);

struct Context {
  hack_ctx* ctx = nullptr;
  explicit Context(int dtype = HACK_BF16, int heads = kH, int max_units = 2 * kH, int max_queries = 512) {
    hack_config cfg{0, heads, kD, dtype, max_units, 256, max_queries, 32};
    if (hack_create(&ctx, &cfg) != HACK_OK) abort();
  }
  ~Context() { hack_destroy(ctx); }
};

template <typename T = uint8_t>
T* at(uintptr_t a) { return reinterpret_cast<T*>(a); }   // device addresses that nothing follows
constexpr uintptr_t kA = 0x100000000, kB = 0x200000000, kC = 0x300000000, kE = 0x400000000, kF = 0x500000000;

// 100 pages of 64 rows of four heads, token by token; tables of 20 entries
hack_pages pages() { return hack_pages{at(kA), at(kB), 100, 64, 64 * kH * kD, kH * kD, kD, at<int32_t>(kC), 20, 20, at<int32_t>(kC + 0x1000), 0, 0}; }

int append_refusals() {
  Context c;
  double freq[64];
  for (int i = 0; i < 64; ++i) freq[i] = std::pow(10000.0, -i / 64.0);
  const hack_rope rope{HACK_ROPE_HALF, 128, 1, 1.f, freq};
  const hack_rows q{at(kE), at(kE + 0x1000000), 8, 8 * 10 * kD, 10 * kD, kD, nullptr, 0};
  const hack_rows k{at(kF), nullptr, kH, kH * 10 * kD, 10 * kD, kD, nullptr, 0}, v{at(kF + 0x1000000), nullptr, kH, kH * 10 * kD, 10 * kD, kD, nullptr, 0};
  const auto run = [&](const hack_rows* q, hack_rows k, hack_rows v, hack_pages p, int norm = HACK_NORM_NONE, float eps = 1e-6f, const hack_rope* r = nullptr,
                       const int32_t* pos = nullptr, const int32_t* fresh = nullptr, int B = 2, int N = 10) {
    return hack_append_pages(c.ctx, B, N, q, &k, &v, norm, eps, r, pos, 0, fresh, &p, kStream);
  };
  CHECK(run(&q, k, v, pages(), HACK_NORM_RMS, 1e-6f, &rope) == HACK_OK && stub::appends.size() == 1);
  {
    const AppendArgs& a = stub::appends.back();
    CHECK(a.own_rows == 1 && a.c.max_len == 20 * 64 && a.c.log2_rows == 6 && a.c.n == 10 && a.c.fault == c.ctx->fault + 2);
    CHECK(a.groups[0] > 0 && a.groups[1] > a.groups[0] && a.all_groups == a.groups[1] + (a.groups[1] - a.groups[0]));
    CHECK(a.v.tiles == a.t[1].tiles && a.v.tokens_log2 == a.t[1].tokens_log2);
  }
  CHECK(run(nullptr, k, v, pages()) == HACK_OK && stub::appends.back().groups[0] == 0 && stub::appends.back().all_groups == 2 * stub::appends.back().groups[1]);
  REFUSED(HACK_EINVAL, hack_append_pages(nullptr, 2, 10, &q, &k, &v, -1, 0.f, nullptr, nullptr, 0, nullptr, nullptr, kStream));
  REFUSED(HACK_EINVAL, hack_append_pages(c.ctx, 2, 10, &q, &k, &v, -1, 0.f, nullptr, nullptr, 0, nullptr, nullptr, kStream));
  hack_pages ok = pages();
  REFUSED(HACK_EINVAL, hack_append_pages(c.ctx, 2, 10, &q, nullptr, &v, -1, 0.f, nullptr, nullptr, 0, nullptr, &ok, kStream));
  REFUSED(HACK_EINVAL, hack_append_pages(c.ctx, 2, 10, &q, &k, nullptr, -1, 0.f, nullptr, nullptr, 0, nullptr, &ok, kStream));
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), 2));
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), HACK_NORM_RMS, 0.f));
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), HACK_NORM_UNIT, NAN));
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, nullptr, nullptr, at<int32_t>(kC + 2)));
  REFUSED(HACK_ECAPACITY, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, nullptr, nullptr, nullptr, 3));
  REFUSED(HACK_ECAPACITY, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, nullptr, nullptr, nullptr, 2, 513));
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, nullptr, nullptr, nullptr, 0));
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, nullptr, nullptr, nullptr, 2, 0));
  for (int i = 0; i < 9; ++i) {
    hack_rows x = k, y = v, z = q;
    if (i == 0) x.out = at(kE + 0x2000000);
    if (i == 1) y.out = at(kE + 0x2000000);
    if (i == 2) x.heads = 8;
    if (i == 3) y.heads = 1;
    if (i == 4) y.weight = at<float>(kE + 0x3000000);
    if (i == 5) x.weight = at<float>(kE + 0x3000000);   // without a norm
    if (i == 6) x.x = nullptr;
    if (i == 7) y.stride_n = 4;
    if (i == 8) z.out = nullptr;
    REFUSED(HACK_EINVAL, run(&z, x, y, pages()));
  }
  // memory that is read and written
  const uintptr_t cache_end = kA + 100ull * 64 * kH * kD * 2;
  for (int i = 0; i < 8; ++i) {
    hack_rows x = k, y = v, z = q;
    hack_pages p = pages();
    const int32_t *pos = nullptr, *fresh = nullptr;
    if (i == 0) x.x = at(cache_end - 16);
    if (i == 1) y.x = at(kB + 4096);
    if (i == 2) z.out = at(kB);
    if (i == 3) z.out = at(kE + 16);
    if (i == 4) z.out = at(kF + 4096);
    if (i == 5) p.table = at<int32_t>(kA + 4096);
    if (i == 6) p.len = at<int32_t>(kE + 0x1000000 + 64);   // under the queries' output
    if (i == 7) fresh = at<int32_t>(kB + 64);
    REFUSED(HACK_EINVAL, run(&z, x, y, p, HACK_NORM_NONE, 0.f, &rope, pos, fresh));
  }
  REFUSED(HACK_EINVAL, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, &rope, at<int32_t>(kA)));
  hack_rows in_place = q;
  in_place.out = at(kE);
  CHECK(run(&in_place, k, v, pages()) == HACK_OK);
  hack_rows behind = k;
  behind.x = at(cache_end);
  CHECK(run(&q, behind, v, pages()) == HACK_OK);
  // by head: positions are needed where rows turn
  hack_pages p = pages();
  p.by_head = 1;
  REFUSED(HACK_EINVAL, run(&q, k, v, p, HACK_NORM_NONE, 0.f, &rope));
  CHECK(run(&q, k, v, p) == HACK_OK);
  CHECK(run(&q, k, v, p, HACK_NORM_NONE, 0.f, &rope, at<int32_t>(kE + 0x4000000)) == HACK_OK && stub::appends.back().own_rows == 0);
  p.stride_head = 0;
  p.stride_row = kD;
  p.stride_page = 64 * kD;
  CHECK(run(&q, k, v, p) == HACK_OK);
  stub::device = 1;
  REFUSED(HACK_EINVAL, run(&q, k, v, pages()));
  stub::device = 0;
  hack_rope bad = rope;
  bad.rot_dim = 24;
  REFUSED(HACK_EUNSUPPORTED, run(&q, k, v, pages(), HACK_NORM_NONE, 0.f, &bad));
  return 0;
}

int cache_refusals() {
  Context c;
  const auto run = [&](hack_pages p, int B = 2) {
    return hack_attn_pages(c.ctx, B, 1, 8, at(kE), &p, nullptr, 0, nullptr, 0, 0.1f, at(kF), kStream);
  };
  CHECK(run(pages()) == HACK_OK);
  for (int i = 0; i < 26; ++i) {
    hack_pages p = pages();
    switch (i) {
      case 0: p.k = nullptr; break;
      case 1: p.v = nullptr; break;
      case 2: p.table = nullptr; break;
      case 3: p.len = nullptr; break;
      case 4: p.k = at(kA + 8); break;
      case 5: p.table = at<int32_t>(kC + 2); break;
      case 6: p.len = at<int32_t>(kC + 1); break;
      case 7: p.pages = 0; break;
      case 8: p.pages = 1ll << 31; break;
      case 9: p.page_rows = 8; break;
      case 10: p.page_rows = 48; break;
      case 11: p.page_rows = 1 << 17; break;
      case 12: p.table_pages = 0; break;
      case 13: p.table_stride = 19; break;
      case 14: p.stride_page = -64 * kH * kD; break;
      case 15: p.stride_row = kH * kD + 4; break;
      case 16: p.stride_page = 64 * kH * kD - 8; break;      // overlap
      case 17: p.stride_row = kH * kD - 8; break;
      case 18: p.stride_head = kD - 8; break;
      case 19: p.stride_head = 0; break;                     // not by head
      case 20: p.stride_page = INT64_MAX / 16 / 8 * 8; break;
      case 21: p.stride_row = 1 << 26; p.stride_page = 1ll << 40; break;
      case 22: p.max_len = -1; break;
      case 23: p.max_len = 20 * 64 + 1; break;
      case 24: p.v = at(kA + 4096); break;                   // K and V share rows
      case 25: p.table_stride = INT64_MAX / 2; break;
    }
    REFUSED(HACK_EINVAL, run(p));
  }
  // K and V in turn: whole pages, rows, heads
  hack_pages p = pages();
  p.stride_page *= 2;
  p.v = at(kA + 64 * kH * kD * 2);
  CHECK(run(p) == HACK_OK);
  p.v = at(kA + 64 * kH * kD * 2 - 16);
  REFUSED(HACK_EINVAL, run(p));
  p.v = at(kA + 64 * kH * kD * 2 + 16);
  REFUSED(HACK_EINVAL, run(p));
  p = pages();
  p.stride_row *= 2;
  p.stride_page *= 2;
  p.v = at(kA + kH * kD * 2);
  CHECK(run(p) == HACK_OK);
  p = pages();
  p.stride_head *= 2;
  p.stride_row *= 2;
  p.stride_page *= 2;
  p.v = at(kA + kD * 2);
  CHECK(run(p) == HACK_OK);
  p.v = at(kA + kD * 2 - 16);
  REFUSED(HACK_EINVAL, run(p));
  // heads first, a single page, rows of the table apart, a bound of its own, table longer than lengths can be
  p = pages();
  p.stride_head = 64 * kD;
  p.stride_row = kD;
  CHECK(run(p) == HACK_OK);
  p.pages = 1;
  p.stride_page = 0;
  CHECK(run(p) == HACK_OK);
  p = pages();
  p.table_stride = 33;
  p.max_len = 77;
  CHECK(run(p) == HACK_OK && stub::attentions.back().a.c.max_len == 77);
  p.table_pages = p.table_stride = INT32_MAX;
  p.max_len = 0;
  p.table = at<int32_t>(0x80000000000);
  p.len = at<int32_t>(0xF00000000000);
  CHECK(run(p) == HACK_OK && stub::attentions.back().a.c.max_len == INT32_MAX - 2 * kKeys);
  return 0;
}

int attn_refusals() {
  Context c;
  hack_pages p = pages();
  p.table_pages = p.table_stride = 2000;
  p.len = at<int32_t>(kC + 0x10000);
  const auto run = [&](const hack_shared* s, int n, int B = 2, int N = 1, int heads = 8, void* out = at(kF), float scale = 0.1f) {
    return hack_attn_pages(c.ctx, B, N, heads, at(kE), &p, nullptr, 0, s, n, scale, out, kStream);
  };
  const hack_shared both[] = {{0, 2, 100000}}, each[] = {{0, 1, 100000}, {1, 1, 100000}}, little[] = {{0, 2, 640}};
  CHECK(run(both, 1) == HACK_OK && stub::attentions.back().a.n_shared == 1 && stub::attentions.back().merge);
  CHECK(run(each, 2) == HACK_OK && stub::attentions.back().a.n_shared == 0);   // nothing is shared
  CHECK(run(little, 1) == HACK_OK && stub::attentions.back().a.n_shared == 0); // not worth a launch that joins
  CHECK(run(both, 0) == HACK_OK && stub::attentions.back().a.n_shared == 0);
  REFUSED(HACK_EINVAL, hack_attn_pages(nullptr, 2, 1, 8, at(kE), &p, nullptr, 0, nullptr, 0, 0.1f, at(kF), kStream));
  REFUSED(HACK_EINVAL, hack_attn_pages(c.ctx, 2, 1, 8, nullptr, &p, nullptr, 0, nullptr, 0, 0.1f, at(kF), kStream));
  REFUSED(HACK_EINVAL, hack_attn_pages(c.ctx, 2, 1, 8, at(kE), nullptr, nullptr, 0, nullptr, 0, 0.1f, at(kF), kStream));
  REFUSED(HACK_EINVAL, hack_attn_pages(c.ctx, 2, 1, 8, at(kE + 8), &p, nullptr, 0, nullptr, 0, 0.1f, at(kF), kStream));
  REFUSED(HACK_EINVAL, hack_attn_pages(c.ctx, 2, 1, 8, at(kE), &p, at<int32_t>(kC + 1), 0, nullptr, 0, 0.1f, at(kF), kStream));
  REFUSED(HACK_EINVAL, run(nullptr, 1));
  REFUSED(HACK_EINVAL, run(both, -1));
  REFUSED(HACK_ECAPACITY, run(both, 257));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 6));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 0));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 8, nullptr));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 8, at(kE)));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 8, at(kA + 4096)));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 8, at(kC)));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 8, at(kF), 0.f));
  REFUSED(HACK_EINVAL, run(both, 1, 2, 1, 8, at(kF), NAN));
  REFUSED(HACK_ECAPACITY, run(both, 1, 3));
  REFUSED(HACK_ECAPACITY, run(both, 1, 2, 513));
  REFUSED(HACK_EINVAL, run(both, 1, 1));   // a group beyond the batch
  const hack_shared wrong[][2] = {{{1, 1, 5}, {0, 1, 5}}, {{0, 2, 5}, {1, 1, 5}}, {{-1, 1, 5}, {1, 1, 5}}, {{0, 0, 5}, {1, 1, 5}},
                                  {{0, 1, -1}, {1, 1, 5}}, {{0, 1, 2000 * 64 + 1}, {1, 1, 5}}, {{0, INT32_MAX, 5}, {1, 1, 5}}};
  for (const auto& w : wrong) REFUSED(HACK_EINVAL, run(w, 2));
  // more queries than a launch takes: 2^31 - 64 rows
  REFUSED(HACK_ECAPACITY, run(nullptr, 0, 2, 512, 4 << 19));
  // heads of another context: a bad page or length that a kernel reported is the next call's error, once
  c.ctx->fault[2] = 1;
  REFUSED(HACK_EINVAL, run(both, 1));
  CHECK(std::string(hack_last_error(c.ctx)).find("page number") != std::string::npos);
  CHECK(run(both, 1) == HACK_OK && hack_check(c.ctx) == HACK_OK);
  c.ctx->fault[2] = 1;
  CHECK(hack_check(c.ctx) == HACK_EINVAL && hack_check(c.ctx) == HACK_OK);
  return 0;
}

// What the kernels make of a launch, for lengths that they find: the pairs and slots of all entries are inside what the host has laid out.
int plans() {
  std::mt19937 rng(7);
  const auto upto = [&](double most) { return (int)std::exp(std::uniform_real_distribution<double>(0.0, std::log(most + 1.0))(rng)); };
  for (int round = 0; round < 400; ++round) {
    const int H = upto(16) + 0, B = upto(64), G = upto(16), N = rng() % 2 ? 1 : upto(600), heads = std::max(H, 1);
    Context c(rng() % 3 ? HACK_BF16 : HACK_F32, heads, std::max(B, 1) * heads, 600);
    c.ctx->cus = 256;
    if (c.ctx->cfg.dtype == HACK_BF16) c.ctx->part_rows = 512 * 2 * 128;
    hack_pages p = pages();
    p.by_head = rng() % 4 == 0;
    p.stride_head = kD;
    p.stride_row = heads * kD;
    p.stride_page = 64ll * heads * kD;
    p.table_pages = std::max(1, upto(rng() % 4 ? 2000 : 3e7));
    p.table_stride = p.table_pages;
    p.table = at<int32_t>(0x80000000000);
    p.len = at<int32_t>(0xF00000000000);
    const int batch = std::max(B, 1), rows = std::max(N, 1), most = (int)std::min<int64_t>(64ll * p.table_pages, INT32_MAX - 64);
    std::vector<hack_shared> groups;
    for (int b = 0; b < batch && rng() % 4; ) {
      const int count = std::min(batch - b, std::max(1, upto(32)));
      groups.push_back({b, count, (int)(rng() % ((unsigned)most + 1u))});
      b += count + rng() % 2;
    }
    if (groups.size() > 256) groups.resize(256);
    CHECK(hack_attn_pages(c.ctx, batch, rows, heads * std::max(G, 1), at(kE << 8), &p, nullptr, 0, groups.data(), (int)groups.size(), 0.1f, at(kF << 8), kStream) == HACK_OK);
    const AttnPagesArgs& a = stub::attentions.back().a;
    const int64_t GN = (int64_t)a.G * rows;
    for (int tries = 0; tries < 4; ++tries) {
      std::vector<int> len(p.by_head ? batch * heads : batch);
      for (int& l : len) l = tries == 0 ? most : tries == 1 ? 0 : rng() % ((unsigned)most + 1u);
      if (tries == 3) std::fill(len.begin() + 1, len.end(), 1);
      std::vector<int> blocks[2], mult = {heads, p.by_head ? 1 : heads};
      for (int g = 0; g < a.n_shared; ++g) blocks[0].push_back(blocks_between(0, std::min(a.shared[g].rows, a.c.max_len)));
      for (size_t e = 0; e < len.size(); ++e) {
        int lo = 0;
        const int b = p.by_head ? (int)e / heads : (int)e;
        for (int g = 0; g < a.n_shared; ++g)
          if (b >= a.shared[g].first && b < a.shared[g].first + a.shared[g].count) lo = a.shared[g].rows;
        blocks[1].push_back(blocks_between(lo, len[e]));
      }
      const bool together = a.n_shared > 0;   // both parts are one launch
      float total[2] = {};
      for (int part = 0; part < 2; ++part)
        for (int n : blocks[part]) total[part] += (float)mult[part] * a.part[part].tiles * n;
      if (together) total[0] = total[1] = total[0] + total[1];
      int64_t pairs[2] = {}, rows = 0;
      bool joined = a.n_shared > 0;
      for (int part = 0; part < 2; ++part) {
        const int longest = blocks[part].empty() ? 0 : *std::max_element(blocks[part].begin(), blocks[part].end());
        const int chunk = chunk_blocks(total[part], longest, a.part[part]);
        for (int n : blocks[part]) {
          pairs[part] += (int64_t)mult[part] * entry_chunks(n, chunk);
          joined |= entry_chunks(n, chunk) > 1;
        }
        CHECK(pairs[part] <= a.part[part].pairs);
        CHECK(rows <= a.part[part].row0);
        rows = a.part[part].row0 + pairs[part] * a.part[part].tiles * a.part[part].queries;
      }
      CHECK(!joined || stub::attentions.back().merge);
      CHECK(!joined || rows <= c.ctx->part_rows);
    }
    CHECK((int64_t)a.part[1].tiles * a.part[1].queries >= GN);
    for (int g = 0; g < a.n_shared; ++g) CHECK((int64_t)a.part[0].tiles * a.part[0].queries >= a.shared[g].count * GN);
    CHECK(pairs_grid(a.part[0].pairs, a.part[0].tiles) + pairs_grid(a.part[1].pairs, a.part[1].tiles) <= kMostGroups);
    stub::attentions.clear();
  }
  return 0;
}

// Groups whose partial results find no room: every element reads its rows by itself, in the tiles that it has without groups.
int dropped_groups() {
  const auto call = [](int dtype, int heads, int batch, int group, int queries, int rows, int own, bool shared, int32_t (&form)[3]) {
    Context c(dtype, heads, batch * heads, 600);
    c.ctx->cus = 256;
    if (dtype == HACK_BF16) c.ctx->part_rows = 512 * 2 * 128;
    hack_pages p = pages();
    p.stride_head = kD;
    p.stride_row = heads * kD;
    p.stride_page = 64ll * heads * kD;
    p.table_pages = p.table_stride = (rows + own + 63) / 64;
    p.table = at<int32_t>(0x80000000000);
    p.len = at<int32_t>(0xF00000000000);
    const hack_shared s{0, batch, rows};
    stub::attentions.clear();
    if (hack_attn_pages(c.ctx, batch, queries, heads * group, at(kE << 8), &p, nullptr, 0, &s, shared, 0.1f, at(kF << 8), kStream) != HACK_OK) return false;
    const AttnPagesArgs& a = stub::attentions.back().a;
    form[0] = a.n_shared;
    form[1] = a.part[1].queries;
    form[2] = a.part[1].pairs;
    return true;
  };
  int32_t with[3], without[3];
  CHECK(call(HACK_BF16, 30, 8, 1, 64, 4096, 155, true, with) && with[0] == 1 && with[1] == kPageTileQueries);   // room: tiles as large as those of the shared rows
  const struct { int dtype, heads, batch, group, queries, rows; } none[] = {{HACK_BF16, 30, 32, 1, 64, 4096}, {HACK_BF16, 8, 1024, 1, 1, 8192}, {HACK_BF16, 8, 64, 4, 33, 4096},
                                                                            {HACK_F32, 32, 64, 1, 1, 4096}, {HACK_F32, 8, 256, 4, 1, 4096}};
  for (const auto& x : none) {
    CHECK(call(x.dtype, x.heads, x.batch, x.group, x.queries, x.rows, 155, true, with) && call(x.dtype, x.heads, x.batch, x.group, x.queries, x.rows, 155, false, without));
    printf("%d queries of %d x %d: tiles of %d, without groups %d\n", x.queries, x.heads, x.batch, with[1], without[1]);
    CHECK(with[0] == 0 && with[1] == without[1] && with[2] == without[2]);
  }
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  const std::string name = argc > 1 ? argv[1] : "";
  int r = 2;
  if (name == "append_refusals") r = append_refusals();
  if (name == "cache_refusals") r = cache_refusals();
  if (name == "attn_refusals") r = attn_refusals();
  if (name == "plans") r = plans();
  if (name == "dropped_groups") r = dropped_groups();
  if (r == 0) printf("ok\n");
  return r;
}
