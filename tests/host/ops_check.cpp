// Host-side checks of csrc/ops_api.cpp (rotary positions, norms, packed caches) over the stand-in for the HIP runtime; argv[1] names the check.
#include "hip_host_stub.h"

#include "../../paper_2504_09261_amd/csrc/hack_api.cpp"
#include "../../paper_2504_09261_amd/csrc/ops_api.cpp"

#include <cfloat>

namespace stub {
int device = 0;
std::vector<RotateArgs> rotations;
struct Pack : PackHead { std::vector<PackUnit> unit; };
struct Attention : AttnPackedHead { std::vector<AttnPackedUnit> unit; };
std::vector<Pack> packs, unpacks;
std::vector<Attention> attentions;
std::vector<int> queries;
size_t calls() { return rotations.size() + packs.size() + unpacks.size() + attentions.size(); }
}  // namespace stub

extern "C" hipError_t hipGetDevice(int* d) { *d = stub::device; return hipSuccess; }

namespace hack {
void launch_rotate(hipStream_t, int, int, bool, int, int, RotateArgs a) { stub::Quiet q; stub::rotations.push_back(a); }
void launch_pack(hipStream_t, int, int, PackHead h, const PackUnit* u, int n) { stub::Quiet q; stub::packs.push_back({h, {u, u + n}}); }
void launch_unpack(hipStream_t, int, int, PackHead h, const PackUnit* u, int n) { stub::Quiet q; stub::unpacks.push_back({h, {u, u + n}}); }
void launch_attn_packed(hipStream_t, int, int, int n, const AttnPackedHead& h, const AttnPackedUnit* u) {
  stub::Quiet q;
  stub::attentions.push_back({h, {u, u + h.n_units}});
  stub::queries.push_back(n);
}
}  // namespace hack

#define CHECK(c)                                    \
  do {                                              \
    if (!(c)) {                                     \
      printf("FAILED line %d: %s\n", __LINE__, #c); \
      return 1;                                     \
    }                                               \
  } while (0)
// The call fails that way and launches nothing.
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
  explicit Context(int dtype = HACK_BF16, int heads = kH, int max_units = 2 * kH) {
    hack_config cfg{0, heads, kD, dtype, max_units, 256, 512, 32};
    if (hack_create(&ctx, &cfg) != HACK_OK) abort();
  }
  ~Context() { hack_destroy(ctx); }
};

template <typename T = uint8_t>
T* at(uintptr_t a) { return reinterpret_cast<T*>(a); }   // device addresses that nothing follows
constexpr uintptr_t kA = 0x10000000, kB = 0x20000000, kC = 0x30000000, kE = 0x40000000;

int rotate_refusals() {
  Context c;
  double freq[64];
  float gain = 0.f;
  CHECK(hack_rope_freqs(128, 1, HACK_ROPE_PLAIN, 10000.0, 1.0, 0.0, freq, &gain) == HACK_OK && gain == 1.f);
  const hack_rope ok{HACK_ROPE_HALF, 128, 1, 1.f, freq};
  const hack_rows x{at(kA), at(kB), 4, 4 * 10 * kD, 10 * kD, kD, nullptr, 0};
  auto rot = [&](hack_rows r, hack_rope p, const int32_t* pos = nullptr, int64_t sb = 0, int32_t pos0 = 0, int B = 2, int N = 10) {
    return hack_rotate(c.ctx, B, N, &r, &p, pos, sb, pos0, kStream);
  };
  CHECK(rot(x, ok) == HACK_OK && stub::rotations.size() == 1);
  REFUSED(HACK_EINVAL, hack_rotate(nullptr, 2, 10, &x, &ok, nullptr, 0, 0, kStream));
  REFUSED(HACK_EINVAL, hack_rotate(c.ctx, 2, 10, nullptr, &ok, nullptr, 0, 0, kStream));
  REFUSED(HACK_EINVAL, hack_rotate(c.ctx, 2, 10, &x, nullptr, nullptr, 0, 0, kStream));
  REFUSED(HACK_EINVAL, rot(x, ok, nullptr, 0, 0, 0));
  REFUSED(HACK_EINVAL, rot(x, ok, nullptr, 0, 0, 2, 0));
  REFUSED(HACK_ECAPACITY, rot(x, ok, nullptr, 0, 0, 3));
  REFUSED(HACK_ECAPACITY, rot(x, ok, nullptr, 0, 0, 1, 513));
  for (int i = 0; i < 12; ++i) {
    hack_rows r = x;
    if (i == 0) r.x = nullptr;
    if (i == 1) r.out = nullptr;
    if (i == 2) r.x = at(kA + 8);
    if (i == 3) r.out = at(kB + 8);
    if (i == 4) r.heads = 0;
    if (i == 5) r.stride_b = -kD;
    if (i == 6) r.stride_h = kD + 4;
    if (i == 7) r.stride_n = INT64_MAX / 2;
    if (i == 8) r.weight = at<float>(kC);
    if (i == 9) r.out = at(kA + 16);            // overlap
    if (i == 10) r.out = at(kA + 2 * 4 * 10 * kD * 2 - 16);
    if (i == 11) { r.out = at(kA); r.stride_n = 2 * kD; }   // in place, but not in the layout of out
    REFUSED(HACK_EINVAL, rot(r, ok));
  }
  hack_rows r = x;
  r.out = at(kA);
  CHECK(rot(r, ok) == HACK_OK);                 // in place
  r.out = at(kA + 2 * 4 * 10 * kD * 2);
  CHECK(rot(r, ok) == HACK_OK);                 // right behind
  for (int i = 0; i < 8; ++i) {
    hack_rope p = ok;
    if (i == 0) p.layout = 2;
    if (i == 1) p.axes = 0;
    if (i == 2) p.axes = 3;
    if (i == 3) p.rot_dim = 0;
    if (i == 4) p.rot_dim = 144;
    if (i == 5) p.freq = nullptr;
    if (i == 6) p.gain = INFINITY;
    if (i == 7) p.axes = 2;                     // without positions
    REFUSED(HACK_EINVAL, rot(x, p));
  }
  hack_rope p = ok;
  p.rot_dim = 24;
  REFUSED(HACK_EUNSUPPORTED, rot(x, p));
  p.rot_dim = 16; p.axes = 2;
  REFUSED(HACK_EUNSUPPORTED, rot(x, p, at<int32_t>(kC)));
  freq[5] = NAN;
  REFUSED(HACK_EINVAL, rot(x, ok));
  freq[5] = 1.5e6;
  REFUSED(HACK_EINVAL, rot(x, ok));
  freq[5] = -INFINITY;
  REFUSED(HACK_EINVAL, rot(x, ok));
  freq[5] = -1e-30;
  CHECK(rot(x, ok) == HACK_OK && (stub::rotations.back().turns[5] == 0 || stub::rotations.back().turns[5] + 2 < 4));
  freq[5] = 0.1;
  REFUSED(HACK_EINVAL, rot(x, ok, at<int32_t>(kC + 2)));
  REFUSED(HACK_EINVAL, rot(x, ok, at<int32_t>(kC), 9));
  CHECK(rot(x, ok, at<int32_t>(kC), 10) == HACK_OK);
  REFUSED(HACK_EINVAL, rot(x, ok, nullptr, 0, INT32_MAX - 8));
  CHECK(rot(x, ok, nullptr, 0, INT32_MAX - 9) == HACK_OK);
  stub::device = 1;
  REFUSED(HACK_EINVAL, rot(x, ok));
  stub::device = 0;

  auto norm = [&](hack_rows q, const hack_rows* k, int kind = HACK_NORM_RMS, float eps = 1e-6f) {
    return hack_norm_rotate(c.ctx, 2, 10, &q, k, kind, eps, &ok, nullptr, 0, 0, kStream);
  };
  hack_rows k = x;
  k.x = at(kC); k.out = at(kE); k.heads = 2;
  CHECK(norm(x, &k) == HACK_OK && norm(x, nullptr) == HACK_OK);
  CHECK(hack_norm_rotate(c.ctx, 2, 10, &x, &k, HACK_NORM_UNIT, 1e-6f, nullptr, nullptr, 0, 0, kStream) == HACK_OK);
  REFUSED(HACK_EINVAL, hack_norm_rotate(nullptr, 2, 10, &x, &k, HACK_NORM_RMS, 1e-6f, &ok, nullptr, 0, 0, kStream));
  REFUSED(HACK_EINVAL, norm(x, &k, 2));
  REFUSED(HACK_EINVAL, norm(x, &k, -1));
  REFUSED(HACK_EINVAL, norm(x, &k, HACK_NORM_RMS, 0.f));
  REFUSED(HACK_EINVAL, norm(x, &k, HACK_NORM_RMS, NAN));
  for (int i = 0; i < 6; ++i) {
    hack_rows w = k;
    if (i == 0) w.out = x.out;                  // both outputs in one place
    if (i == 1) w.out = at(kA);                 // over the queries that are read
    if (i == 2) w.weight = at<float>(0x50000004);
    if (i == 3) { w.weight = at<float>(0x50000000); w.weight_stride_h = kD - 4; }
    if (i == 4) { w.weight = at<float>(0x50000000); w.weight_stride_h = kD + 2; }
    if (i == 5) { w.weight = at<float>(0x50000000); w.weight_stride_h = (int64_t)1 << 32; }
    REFUSED(HACK_EINVAL, norm(x, &w));
  }
  return 0;
}

int rope_freqs() {
  double f[64];
  float g;
  for (int i = 0; i < 9; ++i)
    CHECK(hack_rope_freqs(i == 0 ? 0 : i == 1 ? 130 : i == 2 ? 6 : 128, i == 2 ? 2 : i == 3 ? 3 : 1, i == 4 ? 4 : HACK_ROPE_PARTS, i == 5 ? 1.0 : 10000.0, i == 6 ? 0.5 : 2.0,
                          i == 7 ? 0.0 : 4096.0, i == 8 ? nullptr : f, &g) == HACK_EINVAL);
  CHECK(hack_rope_freqs(128, 1, HACK_ROPE_PLAIN, 10000.0, 1.0, 0.0, f, nullptr) == HACK_OK);
  for (int i = 0; i < 64; ++i) CHECK(std::fabs(f[i] / std::pow(10000.0, -i / 64.0) - 1) < 1e-14);
  CHECK(hack_rope_freqs(64, 2, HACK_ROPE_LINEAR, 10000.0, 4.0, 0.0, f, &g) == HACK_OK && g == 1.f);
  for (int i = 0; i < 32; ++i) CHECK(std::fabs(4 * f[i] / std::pow(10000.0, -(i % 16) / 16.0) - 1) < 1e-14);
  CHECK(hack_rope_freqs(64, 1, HACK_ROPE_BASE, 10000.0, 8.0, 0.0, f, &g) == HACK_OK);
  CHECK(f[0] == 1.0 && std::fabs(8 * f[31] / std::pow(10000.0, -31.0 / 32) - 1) < 1e-14);   // fastest stays, slowest by the factor
  CHECK(hack_rope_freqs(128, 1, HACK_ROPE_PARTS, 10000.0, 8.0, 4096.0, f, &g) == HACK_OK && std::fabs(g - (0.1 * std::log(8.0) + 1)) < 1e-6);
  double last = 0.0;
  for (int i = 0; i < 64; ++i) {
    const double plain = std::pow(10000.0, -i / 64.0), turns = 4096 * plain / 6.283185307179586, ratio = plain / f[i];
    CHECK(ratio >= last - 1e-12 && ratio > 1 - 1e-12 && ratio < 8 + 1e-9);
    last = ratio;
    if (turns > 33) CHECK(std::fabs(ratio - 1) < 0.35);      // the ramp begins and ends at whole pairs
    if (turns > 40) CHECK(std::fabs(ratio - 1) < 1e-12);
    if (turns < 0.8) CHECK(std::fabs(ratio - 8) < 1e-9);
  }
  // what the kernel gets: fractions of a turn, whole turns dropped, negative frequencies turned round
  Context c;
  double w[64] = {0};
  w[0] = 6.283185307179586 * 0.25;
  w[1] = 6.283185307179586 * 3.75;
  w[2] = -6.283185307179586 * 0.125;
  const hack_rope p{HACK_ROPE_HALF, 128, 1, 1.f, w};
  const hack_rows x{at(kA), at(kB), 1, 0, 0, kD, nullptr, 0};
  CHECK(hack_rotate(c.ctx, 1, 1, &x, &p, nullptr, 0, 0, kStream) == HACK_OK);
  const RotateArgs& a = stub::rotations.back();
  const double want[4] = {0.25, 0.75, 0.875, 0.0};   // w itself is rounded twice, the constant and the product: 3.75 turns 2 2^-53 = 8.4e-16
  for (int i = 0; i < 4; ++i) CHECK(std::fabs(std::ldexp((double)a.turns[i], -64) - want[i]) < 8.5e-16);
  return 0;
}

// Frequencies below zero turn exactly the other way.
int backward_frequencies() {
  Context c;
  double w[64], back[64];
  for (int i = 0; i < 64; ++i) {
    w[i] = i == 0 ? 1e6 : i == 1 ? 1e-30 : std::pow(10000.0, -i / 64.0);
    back[i] = -w[i];
  }
  const hack_rope forth{HACK_ROPE_HALF, 128, 1, 1.f, w}, p{HACK_ROPE_HALF, 128, 1, 1.f, back};
  const hack_rows x{at(kA), at(kB), 1, 0, 0, kD, nullptr, 0};
  CHECK(hack_rotate(c.ctx, 1, 1, &x, &forth, nullptr, 0, 0, kStream) == HACK_OK && hack_rotate(c.ctx, 1, 1, &x, &p, nullptr, 0, 0, kStream) == HACK_OK);
  const RotateArgs &a = stub::rotations[0], &b = stub::rotations[1];
  for (int i = 0; i < 64; ++i) CHECK(a.turns[i] + b.turns[i] == 0);
  return 0;
}

// The chunks of a unit cover its rows once, whatever its length.
int chunk_rows() {
  for (int64_t len : {1LL, 63LL, 64LL, 65LL, 1000LL, 131071LL, 2147483520LL, 2147483583LL, 2147483584LL, 2147483585LL, 2147483646LL, 2147483647LL}) {
    const int n = packed_blocks((int)len);
    CHECK(n == (len + 63) / 64);
    for (int64_t most : {1LL << 30, (long long)n, n / 2 + 1LL, n / 7 + 1LL, n / 1023 + 1LL}) {
      const int chunks = chunks_of(n, (int)std::min<int64_t>(most, n));
      int64_t end = 0;
      for (int c = 0; c < chunks; ++c) {
        const int lo = chunk_at(n, chunks, c), hi = chunk_at(n, chunks, c + 1);
        CHECK(lo < hi && hi - lo <= most && (int64_t)lo * 64 == end);
        const int64_t rows = rows_in((int)len, lo, hi);
        CHECK(rows >= 1 && rows <= (int64_t)(hi - lo) * 64);
        for (int each : {32, 64}) CHECK(stages_of((int)rows, each) == (rows + each - 1) / each);
        end += rows;
      }
      CHECK(end == len);
    }
  }
  return 0;
}

// Launches stay below 2^32 threads, 256 a work-group: units of many queries in several ones, and one unit of too many queries refused.
int large_launches() {
  constexpr int n = 1024;
  hack_ctx* ctx = nullptr;
  hack_config cfg{0, 1, kD, HACK_F32, n, 64, INT32_MAX, 32};
  CHECK(hack_create(&ctx, &cfg) == HACK_OK);
  std::vector<int64_t> off(n, 0);
  std::vector<int32_t> len(n, 64);
  const hack_packed_cache kv{at(kA), at(kA + 0x100000), nullptr, 64, off.data(), len.data()};
  for (int N : {1, 1 << 17, (1 << 18) - 15, (1 << 18) + 1, 3000001, 1 << 24, (1 << 25) - 16}) {
    stub::attentions.clear();
    CHECK(hack_attn_packed(ctx, n, N, at(0x100000000000), &kv, 0.1f, at(0x600000000000), kStream) == HACK_OK);
    std::vector<int> seen(n, 0);
    for (const auto& a : stub::attentions) {
      CHECK(((int64_t)a.n_units * a.n_chunks + 7) / 8 * 8 * a.q_tiles < (1 << 24) && a.n_units >= 1);
      for (const auto& u : a.unit) ++seen[u.unit];
    }
    for (int u = 0; u < n; ++u) CHECK(seen[u] == 1);
    if (N <= (1 << 18) - 16) CHECK(stub::attentions.size() == 1);
  }
  for (int N : {(1 << 25) - 15, INT32_MAX}) REFUSED(HACK_ECAPACITY, hack_attn_packed(ctx, 1, N, at(0x100000000000), &kv, 0.1f, at(0x600000000000), kStream));
  hack_destroy(ctx);
  return 0;
}

// Outputs of rotations over weights or positions, which other work-groups still read.
int rotation_shared_memory() {
  Context c;
  double freq[64];
  CHECK(hack_rope_freqs(128, 2, HACK_ROPE_PLAIN, 10000.0, 1.0, 0.0, freq, nullptr) == HACK_OK);
  const hack_rope rope{HACK_ROPE_HALF, 128, 2, 1.f, freq};
  constexpr int N = 10, B = 2;
  constexpr int64_t kBytes = (int64_t)B * 4 * N * kD * 2;
  const hack_rows x{at(kA), at(kB), 4, 4 * N * kD, N * kD, kD, nullptr, 0};
  const auto pos = [&](uintptr_t p, int64_t sb) { return hack_rotate(c.ctx, B, N, &x, &rope, at<int32_t>(p), sb, 0, kStream); };
  CHECK(pos(kB - 2 * N * 4, 0) == HACK_OK && pos(kB + kBytes, 0) == HACK_OK);
  REFUSED(HACK_EINVAL, pos(kB, 0));
  REFUSED(HACK_EINVAL, pos(kB + kBytes - 4, 0));
  REFUSED(HACK_EINVAL, pos(kB - 2 * N * 4 + 4, 0));
  CHECK(pos(kB - (50 + 2 * N) * 4, 50) == HACK_OK);
  REFUSED(HACK_EINVAL, pos(kB - (50 + 2 * N) * 4 + 4, 50));
  CHECK(pos(kB + kBytes, INT64_MAX) == HACK_OK);
  hack_rows k = x;
  k.x = at(kC); k.out = at(kE);
  const auto norm = [&](uintptr_t qw, int64_t qs, uintptr_t kw, int64_t ks, const hack_rope* r, uintptr_t p) {
    hack_rows a = x, b = k;
    a.weight = at<float>(qw);
    a.weight_stride_h = qs;
    b.weight = at<float>(kw);
    b.weight_stride_h = ks;
    return hack_norm_rotate(c.ctx, B, N, &a, &b, HACK_NORM_RMS, 1e-6f, r, at<int32_t>(p), 0, 0, kStream);
  };
  CHECK(norm(kB - kD * 4, 0, kE - (3 * 256 + kD) * 4, 256, &rope, kE + kBytes) == HACK_OK);
  REFUSED(HACK_EINVAL, norm(kB, 0, 0, 0, &rope, 0x50000000));
  REFUSED(HACK_EINVAL, norm(kE + kBytes - 16, 0, 0, 0, &rope, 0x50000000));   // the other tensor's output
  REFUSED(HACK_EINVAL, norm(0, 0, kB - (3 * 256 + kD) * 4 + 16, 256, &rope, 0x50000000));
  REFUSED(HACK_EINVAL, norm(0, 0, 0, 0, &rope, kE + 64));
  CHECK(norm(0, 0, 0, 0, nullptr, kE + 64) == HACK_OK);                       // positions are not read without a rotation
  return 0;
}

// Lists with strides whose product with the units passes 64 bits (one unit: nothing lies a stride away).
int far_lists() {
  for (int heads : {1, kH}) {
    Context c(HACK_BF16, heads);
    const int64_t off[kH] = {0, 64, 128, 192};
    const int32_t len[kH] = {40, 40, 40, 40};
    const hack_cache in{at(kA), at(kB), nullptr, 256, off, len};
    const hack_packed_cache out{at(0x7f0000000000), at(0x7f1000000000), nullptr, 256, off, len};
    for (int64_t stride : {(int64_t)40, (int64_t)1 << 33, INT64_MAX / 2, INT64_MAX}) {
      const int32_t* const kept = at<int32_t>(0x70000000);
      CHECK(hack_pack(c.ctx, 1, 0, &in, nullptr, nullptr, 0, kept, stride, nullptr, &out, kStream) == HACK_OK);
    }
  }
  return 0;
}

// Frequencies by parts at the ends of what is accepted: pairs that turn less than once over the trained length are divided, even the fastest.
int rope_parts_ends() {
  double f[64];
  for (double length : {1.0, 3.0, 6.28, 6.29, 30.0, 1e3, 1e9, 1e300})
    for (double base : {1.0001, 10.0, 1e4, 1e30}) {
      CHECK(hack_rope_freqs(64, 1, HACK_ROPE_PARTS, base, 8.0, length, f, nullptr) == HACK_OK);
      double last = 0.0;
      for (int i = 0; i < 32; ++i) {
        const double plain = std::pow(base, -i / 32.0), ratio = plain / f[i], turns = length * plain / 6.283185307179586;
        CHECK(ratio > 1 - 1e-12 && ratio < 8 + 1e-9 && ratio >= last - 1e-9);
        last = ratio;
        const double one_pair = std::pow(base, 1 / 32.0);          // the ramp begins and ends at whole pairs
        if (turns > 32.0 * one_pair) CHECK(std::fabs(ratio - 1) < 1e-12);
        if (turns * one_pair < 1.0 || (i == 0 && turns < 1.0)) CHECK(std::fabs(ratio - 8) < 1e-9);
      }
    }
  return 0;
}

// Chunks of very long units: what the merge's LDS holds, and as many as a case of tests/test_gpu_operators.py wants.
int many_chunks() {
  for (int dtype : {HACK_BF16, HACK_F32})
    for (int units : {1, 2, kH})
      for (int64_t len : {140001LL, 1000000LL, 16000000LL, 200000000LL, 2147483647LL})
        for (int N : {1, 5, 16, 40}) {
          Context c(dtype, units, units);
          std::vector<int64_t> off(units, 0);
          std::vector<int32_t> l(units, (int32_t)len);
          const hack_packed_cache kv{at(0x100000000000), at(0x200000000000), nullptr, (len + 63) / 64 * 64, off.data(), l.data()};
          stub::attentions.clear();
          CHECK(hack_attn_packed(c.ctx, 1, N, at(0x50000000), &kv, 0.1f, at(0x60000000), kStream) == HACK_OK && stub::attentions.size() == 1);
          const auto& a = stub::attentions[0];
          CHECK(a.n_chunks <= kMostChunks && (int64_t)a.chunk * a.n_chunks >= (len + 63) / 64);
          if (units == 1 && N <= 16) CHECK(a.n_chunks >= 200);
        }
  return 0;
}

// Rotations: every row once in fewer than 2^32 threads, or a refusal.
int large_rotations() {
  double freq[64];
  CHECK(hack_rope_freqs(16, 1, HACK_ROPE_PLAIN, 10000.0, 1.0, 0.0, freq, nullptr) == HACK_OK);
  const hack_rope rope{HACK_ROPE_HALF, 16, 1, 1.f, freq};
  struct Call { int B, heads, N; bool fits; };
  for (const Call& x : {Call{1, 1, 1, true}, Call{64, 40, 1, true}, Call{2, 16, 4096, true}, Call{1, 1, 32 * ((1 << 24) - 1), true}, Call{1, 1, 32 * ((1 << 24) - 1) + 1, false},
                        Call{1, 1, INT32_MAX, false}, Call{1, 3, INT32_MAX, false}, Call{(1 << 24) - 1, 1, 1, true}, Call{1 << 24, 1, 1, false}, Call{1, 1 << 30, 1, true}, Call{1, (1 << 30) + 1, 1, false},
                        Call{8, INT32_MAX, 1, false}, Call{INT32_MAX, 1, 1, false}}) {
    hack_ctx ctx;   // no workspace is used
    ctx.cfg = hack_config{0, 1, kD, HACK_BF16, INT32_MAX, 64, INT32_MAX, 32};
    const hack_rows r{at(0x100000000000), at(0x600000000000), x.heads, (int64_t)x.heads * x.N * kD, (int64_t)x.N * kD, kD, nullptr, 0};
    stub::rotations.clear();
    const hack_status st = hack_rotate(&ctx, x.B, x.N, &r, &rope, nullptr, 0, 0, kStream);
    CHECK(st == (x.fits ? HACK_OK : HACK_ECAPACITY) && stub::rotations.size() == (x.fits ? 1 : 0));
    if (!x.fits) continue;
    const RotateArgs& a = stub::rotations[0];
    CHECK((int64_t)a.groups[1] * x.B < (1 << 24) && a.groups[0] == a.groups[1]);
    const int64_t across = (kRotateThreads / 8) >> a.t[0].tokens_log2, rows = 1 << a.t[0].tokens_log2, parts = a.groups[0] / a.t[0].tiles;
    CHECK(parts * a.t[0].tiles == a.groups[0] && a.t[0].tiles * rows >= x.N && (a.t[0].tiles - 1) * rows < x.N);
    CHECK(parts * across * a.steps >= x.heads && (parts - 1) * across * a.steps < x.heads);
  }
  return 0;
}

int pack_refusals() {
  Context c;
  CHECK(hack_packed_bytes(96, 64, nullptr) == HACK_EINVAL);
  int64_t n = 0;
  CHECK(hack_packed_bytes(96, 64, &n) == HACK_EINVAL && hack_packed_bytes(128, -1, &n) == HACK_EINVAL);
  CHECK(hack_packed_bytes(128, 65, &n) == HACK_OK && n == 2 * 64 * (64 + 4));
  CHECK(hack_packed_bytes(64, 0, &n) == HACK_OK && n == 0);
  CHECK(hack_packed_bytes(64, (int64_t)INT32_MAX * 64, &n) == HACK_OK && hack_packed_bytes(64, (int64_t)INT32_MAX * 64 + 1, &n) == HACK_EINVAL);

  const int64_t in_off[kH] = {0, 96, 192, 288}, off[kH] = {0, 128, 256, 384};
  const int32_t in_len[kH] = {90, 0, 5, 33}, len[kH] = {100, 10, 15, 43}, first[kH] = {100, 0, 15, 43};
  const hack_cache in{at(kA), at(kB), nullptr, 400, in_off, in_len};
  const hack_packed_cache out{at(kC), at(kE), nullptr, 512, off, len};
  auto pack = [&](const hack_cache* i, const void* k, const void* v, const int32_t* kept, int64_t stride, const int32_t* f, const hack_packed_cache* o, int N = 10) {
    return hack_pack(c.ctx, 1, N, i, k, v, 0, kept, stride, f, o, kStream);
  };
  uint8_t *const k = at(0x50000000), *const v = at(0x60000000);
  int32_t* const kept = at<int32_t>(0x70000000);
  CHECK(pack(&in, k, v, nullptr, 0, nullptr, &out) == HACK_OK && stub::packs.size() == 1);
  const stub::Pack& a = stub::packs[0];
  CHECK(a.unit.size() == 4 && a.unit[3].row0 == 288 && a.unit[3].len_in == 33 && a.unit[3].block == 6 && a.unit[3].first == 0 && a.unit[3].n == 43 && a.n_new == 10);
  CHECK(pack(nullptr, k, v, nullptr, 0, first, &out) == HACK_OK && stub::packs.back().unit[0].n == 0 && stub::packs.back().unit[1].n == 10);
  CHECK(pack(&in, k, v, kept, 100, nullptr, &out) == HACK_OK);
  REFUSED(HACK_ECAPACITY, pack(&in, k, v, kept, 99, nullptr, &out));
  REFUSED(HACK_EINVAL, pack(&in, k, v, at<int32_t>(0x70000002), 100, nullptr, &out));
  REFUSED(HACK_EINVAL, hack_pack(nullptr, 1, 10, &in, k, v, 0, nullptr, 0, nullptr, &out, kStream));
  REFUSED(HACK_EINVAL, pack(nullptr, nullptr, nullptr, nullptr, 0, nullptr, &out));
  REFUSED(HACK_EINVAL, pack(&in, k, nullptr, nullptr, 0, nullptr, &out));
  REFUSED(HACK_EINVAL, pack(&in, nullptr, v, nullptr, 0, nullptr, &out));
  REFUSED(HACK_EINVAL, pack(&in, k + 8, v, nullptr, 0, nullptr, &out));
  REFUSED(HACK_EINVAL, pack(&in, nullptr, nullptr, nullptr, 0, nullptr, &out));   // more rows than are cached
  REFUSED(HACK_EINVAL, pack(&in, k, v, nullptr, 0, nullptr, nullptr));
  REFUSED(HACK_EINVAL, pack(&in, k, v, nullptr, 0, nullptr, &out, 0));
  REFUSED(HACK_ECAPACITY, pack(&in, k, v, nullptr, 0, nullptr, &out, 513));
  const int32_t bad_first[2][kH] = {{101, 0, 0, 0}, {0, -1, 0, 0}};
  for (const auto& f : bad_first) REFUSED(HACK_EINVAL, pack(&in, k, v, nullptr, 0, f, &out));
  const int64_t bad_off[4][kH] = {{0, 130, 256, 384}, {0, -64, 256, 384}, {0, 128, 256, 512}, {64, 128, 256, 384}};   // the last: unit 0 runs into unit 1
  for (const auto& o : bad_off) {
    hack_packed_cache p = out;
    p.off = o;
    REFUSED(HACK_EINVAL, pack(&in, k, v, nullptr, 0, nullptr, &p));
  }
  for (int i = 0; i < 8; ++i) {
    hack_packed_cache p = out;
    if (i == 0) p.k = nullptr;
    if (i == 1) p.v = nullptr;
    if (i == 2) p.off = nullptr;
    if (i == 3) p.len = nullptr;
    if (i == 4) p.rows = 500;
    if (i == 5) p.rows = 448 - 64;
    if (i == 6) p.k = at(kC + 4);
    if (i == 7) p.pos = at<int32_t>(2);
    REFUSED(HACK_EINVAL, pack(&in, k, v, nullptr, 0, nullptr, &p));
  }
  // units in any order, and no rows at all
  const int64_t turned[kH] = {384, 256, 128, 0};
  hack_packed_cache p = out;
  p.off = turned;
  const int32_t full[kH] = {100, 10, 15, 43};
  CHECK(pack(&in, k, v, nullptr, 0, nullptr, &p) == HACK_OK);
  REFUSED(HACK_OK, pack(&in, k, v, nullptr, 0, full, &p));

  hack_cache back{at(kA), at(kB), nullptr, 512, off, len};
  const hack_packed_cache src = out;
  CHECK(hack_unpack(c.ctx, 1, &src, nullptr, &back, kStream) == HACK_OK && stub::unpacks.back().unit[3].row0 == 384);
  REFUSED(HACK_EINVAL, hack_unpack(nullptr, 1, &src, nullptr, &back, kStream));
  REFUSED(HACK_EINVAL, hack_unpack(c.ctx, 1, nullptr, nullptr, &back, kStream));
  REFUSED(HACK_EINVAL, hack_unpack(c.ctx, 1, &src, nullptr, nullptr, kStream));
  const int32_t some[kH] = {1, 0, 0, 0}, most[kH] = {99, 10, 15, 43}, beyond[kH] = {101, 0, 0, 0};
  REFUSED(HACK_EINVAL, hack_unpack(c.ctx, 1, &src, some, &back, kStream));
  REFUSED(HACK_EINVAL, hack_unpack(c.ctx, 1, &src, beyond, &back, kStream));
  back.len = most;
  CHECK(hack_unpack(c.ctx, 1, &src, some, &back, kStream) == HACK_OK && stub::unpacks.back().unit[0].first == 1 && stub::unpacks.back().unit[0].n == 99);
  const int64_t shared[kH] = {0, 96, 256, 384};
  back.off = shared;
  REFUSED(HACK_EINVAL, hack_unpack(c.ctx, 1, &src, some, &back, kStream));
  stub::device = 1;
  back.off = off;
  REFUSED(HACK_EINVAL, hack_unpack(c.ctx, 1, &src, some, &back, kStream));
  REFUSED(HACK_EINVAL, pack(&in, k, v, nullptr, 0, nullptr, &out));
  stub::device = 0;
  return 0;
}

// Outputs that share memory with inputs, or K with V.
int shared_memory() {
  Context c;
  const int64_t off[kH] = {0, 64, 128, 192};
  const int32_t len[kH] = {40, 40, 40, 40};
  uint8_t *const k = at(0x50000000), *const v = at(0x60000000), *const q = at(0x70000000);
  constexpr int64_t kPlain = 256 * kD * 2, kPacked = 4 * 34 * kD, kNew = kH * 40 * kD * 2;   // bytes
  const auto plain = [&](uint8_t* a, uint8_t* b, int32_t* pos = nullptr) { return hack_cache{a, b, pos, 256, off, len}; };
  const auto packed = [&](uint8_t* a, uint8_t* b, int32_t* pos = nullptr) { return hack_packed_cache{a, b, pos, 256, off, len}; };
  const auto pack = [&](const hack_cache& i, const hack_packed_cache& p, const int32_t* kept = nullptr) {
    return hack_pack(c.ctx, 1, 40, &i, k, v, 0, kept, 40, nullptr, &p, kStream);
  };
  const auto unpack = [&](const hack_packed_cache& p, const hack_cache& r) { return hack_unpack(c.ctx, 1, &p, nullptr, &r, kStream); };
  const auto attn = [&](uint8_t* x, const hack_packed_cache& p, uint8_t* out) { return hack_attn_packed(c.ctx, 1, 40, x, &p, 0.5f, out, kStream); };
  int32_t *const pos = at<int32_t>(0x40000000), *const kept = at<int32_t>(0x48000000);
  // side by side is apart
  CHECK(pack(plain(at(kA), at(kA + kPlain)), packed(at(kC), at(kC + kPacked)), kept) == HACK_OK);
  CHECK(pack(plain(at(kC + 2 * kPacked), at(kA)), packed(at(kC), at(kC + kPacked))) == HACK_OK);
  CHECK(unpack(packed(at(kC), at(kC + kPacked), pos), plain(at(kA), at(kA + kPlain), pos + 256)) == HACK_OK);
  CHECK(attn(q, packed(at(kC), at(kE)), q + kNew) == HACK_OK);
  CHECK(pack(plain(at(kC), at(kA)), packed(at(kC + kPlain - 16), at(kE))) == HACK_EINVAL);
  CHECK(pack(plain(at(kB), at(kA)), packed(at(kE), at(kA + kPlain - 16))) == HACK_EINVAL);
  CHECK(pack(plain(at(kA), at(kB)), packed(at(kC), at(kC + kPacked - 16))) == HACK_EINVAL);
  CHECK(pack(plain(at(kA), at(kB)), packed(k + kNew - 16, at(kE))) == HACK_EINVAL);
  CHECK(pack(plain(at(kA), at(kB)), packed(at(kE), v)) == HACK_EINVAL);
  CHECK(pack(plain(at(kA), at(kB), pos), packed(at(kC), at(kE), pos + 255)) == HACK_EINVAL);
  CHECK(pack(plain(at(kA), at(kB)), packed(at(kC), at(kE), kept + 159), kept) == HACK_EINVAL);
  CHECK(unpack(packed(at(kC), at(kE)), plain(at(kA), at(kA + kPlain - 16))) == HACK_EINVAL);
  CHECK(unpack(packed(at(kC), at(kE)), plain(at(kC + kPacked - 16), at(kA))) == HACK_EINVAL);
  CHECK(unpack(packed(at(kC), at(kE), pos), plain(at(kB), at(kA), pos + 255)) == HACK_EINVAL);
  CHECK(attn(q, packed(at(kC), at(kE)), q + kNew - 16) == HACK_EINVAL);
  CHECK(stub::packs.size() == 2 && stub::unpacks.size() == 1);
  return 0;
}

// Every unit once, whatever their number.
int many_units() {
  constexpr int n = 3000;
  Context c(HACK_BF16, 10, n);
  std::vector<int64_t> off(n);
  std::vector<int32_t> len(n), first(n, 0);
  int64_t rows = 0;
  for (int u = 0; u < n; ++u) {
    off[u] = rows;
    len[u] = 1 + u * 37 % 200;
    rows += (len[u] + 63) / 64 * 64;
  }
  const hack_packed_cache out{at(kC), at(kE), nullptr, rows, off.data(), len.data()};
  std::vector<int64_t> in_off(n);
  for (int u = 0; u < n; ++u) in_off[u] = off[u];
  const hack_cache in{at(kA), at(kB), nullptr, rows, in_off.data(), len.data()};
  CHECK(hack_pack(c.ctx, n / 10, 1, &in, nullptr, nullptr, 0, nullptr, 0, nullptr, &out, kStream) == HACK_OK);
  int u = 0;
  for (const auto& a : stub::packs)
    for (size_t i = 0; i < a.unit.size(); ++i, ++u) CHECK(a.unit[i].row0 == off[u] && a.unit[i].n == len[u] && a.unit[i].block == off[u] / 64);
  CHECK(u == n);
  CHECK(hack_attn_packed(c.ctx, n / 10, 5, at(0x50000000), &out, 0.1f, at(0x60000000), kStream) == HACK_OK);
  std::vector<int> seen(n, 0);
  CHECK(stub::attentions.size() == (n + kAttnPackedUnits - 1) / kAttnPackedUnits);
  for (const auto& a : stub::attentions) {
    CHECK(a.n_units >= 1 && a.n_units <= kAttnPackedUnits);
    for (const AttnPackedUnit& x : a.unit) {
      CHECK(x.unit >= 0 && x.unit < n && x.len == len[x.unit] && x.block == off[x.unit] / 64);
      ++seen[x.unit];
    }
  }
  for (int i = 0; i < n; ++i) CHECK(seen[i] == 1);
  return 0;
}

int attn_plan() {
  Context c, f32(HACK_F32);
  std::vector<int64_t> off(8);
  std::vector<int32_t> len(8);
  auto cache = [&](std::vector<int32_t> l) {
    int64_t rows = 0;
    for (size_t u = 0; u < l.size(); ++u) {
      off[u] = rows;
      len[u] = l[u];
      rows += (l[u] + 63) / 64 * 64;
    }
    return hack_packed_cache{at(kC), at(kE), nullptr, rows, off.data(), len.data()};
  };
  uint8_t *const q = at(0x50000000), *const out = at(0x60000000);
  auto attn = [&](const hack_packed_cache& kv, int N, float scale = 0.1f, const void* qq = nullptr, void* o = nullptr, hack_ctx* ctx = nullptr) {
    return hack_attn_packed(ctx ? ctx : c.ctx, 1, N, qq ? qq : q, &kv, scale, o ? o : out, kStream);
  };
  hack_packed_cache kv = cache({100, 1, 5, 43});
  CHECK(attn(kv, 7) == HACK_OK);
  CHECK(attn(kv, 7, 0.1f, nullptr, nullptr, f32.ctx) == HACK_OK && stub::queries.back() == 16);
  REFUSED(HACK_EINVAL, attn(kv, 7, 0.1f, q, q + 4 * 7 * kD * 4 - 16, f32.ctx));
  REFUSED(HACK_EINVAL, hack_attn_packed(nullptr, 1, 7, q, &kv, 0.1f, out, kStream));
  REFUSED(HACK_EINVAL, hack_attn_packed(c.ctx, 1, 7, nullptr, &kv, 0.1f, out, kStream));
  REFUSED(HACK_EINVAL, hack_attn_packed(c.ctx, 1, 7, q, nullptr, 0.1f, out, kStream));
  REFUSED(HACK_EINVAL, hack_attn_packed(c.ctx, 1, 7, q, &kv, 0.1f, nullptr, kStream));
  REFUSED(HACK_EINVAL, attn(kv, 0));
  REFUSED(HACK_ECAPACITY, attn(kv, 513));
  REFUSED(HACK_EINVAL, attn(kv, 7, 0.f));
  REFUSED(HACK_EINVAL, attn(kv, 7, NAN));
  REFUSED(HACK_EINVAL, attn(kv, 7, 0.1f, q + 8));
  REFUSED(HACK_EINVAL, attn(kv, 7, 0.1f, q, out + 8));
  REFUSED(HACK_EINVAL, attn(kv, 7, 0.1f, q, q));
  REFUSED(HACK_EINVAL, attn(kv, 7, 0.1f, q, q + 4 * 7 * kD * 2 - 16));
  CHECK(attn(kv, 7, 0.1f, q, q + 4 * 7 * kD * 2) == HACK_OK);
  len[1] = 0;
  REFUSED(HACK_EINVAL, attn(kv, 7));
  len[1] = -1;
  REFUSED(HACK_EINVAL, attn(kv, 7));
  len[1] = 1;
  stub::device = 1;
  REFUSED(HACK_EINVAL, attn(kv, 7));
  stub::device = 0;
  // Partial results fit the workspace, chunks cover the longest unit, and none is empty for it.
  const std::vector<std::vector<int32_t>> sets = {{1, 1, 1, 1}, {64, 65, 1, 3}, {100000, 1, 7, 700}, {2000000000, 1, 1, 1}, {511, 512, 513, 2}, {131071, 131071, 131071, 131071}};
  for (hack_ctx* ctx : {c.ctx, f32.ctx}) for (const auto& s : sets)
    for (int N : {1, 16, 17, 33, 500}) {
      kv = cache(s);
      stub::attentions.clear();
      stub::queries.clear();
      CHECK(attn(kv, N, 0.1f, nullptr, nullptr, ctx) == HACK_OK && stub::attentions.size() == 1);
      const auto& a = stub::attentions[0];
      const int64_t queries = stub::queries[0], longest = (*std::max_element(s.begin(), s.end()) + 63LL) / 64;
      CHECK(a.q_tiles == (N + queries - 1) / queries && a.chunk >= 1 && a.n_chunks >= 1);
      CHECK((int64_t)a.chunk * a.n_chunks >= longest && (int64_t)a.chunk * (a.n_chunks - 1) < longest);
      const size_t rows = (size_t)a.n_units * a.q_tiles * a.n_chunks * queries;
      if (a.n_chunks > 1) CHECK(stub::owned(a.part_o, rows * kD * 4) && stub::owned(a.part_ml, rows * 8));
    }
  return 0;
}

int no_exceptions() {
  const int64_t off[kH] = {384, 128, 256, 0};
  const int32_t len[kH] = {100, 10, 15, 43};
  const hack_packed_cache out{at(kC), at(kE), nullptr, 512, off, len};
  const hack_cache in{at(kA), at(kB), nullptr, 512, off, len};
  for (int call = 0; call < 2; ++call)
    for (long n = 0; n < 20; ++n) {
      Context c;
      stub::allocations_left = n;
      stub::allocation_failed = false;
      const hack_status st = call == 0 ? hack_pack(c.ctx, 1, 1, &in, nullptr, nullptr, 0, nullptr, 0, nullptr, &out, kStream) : hack_unpack(c.ctx, 1, &out, nullptr, &in, kStream);
      stub::allocations_left = -1;
      CHECK(st == (stub::allocation_failed ? HACK_EHIP : HACK_OK));
      if (!stub::allocation_failed) break;
    }
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  const std::map<std::string, int (*)()> checks = {{"rotate_refusals", rotate_refusals}, {"rope_freqs", rope_freqs}, {"pack_refusals", pack_refusals},
                                                   {"shared_memory", shared_memory}, {"many_units", many_units}, {"attn_plan", attn_plan}, {"no_exceptions", no_exceptions},
                                                   {"backward_frequencies", backward_frequencies}, {"chunk_rows", chunk_rows}, {"large_launches", large_launches},
                                                   {"rotation_shared_memory", rotation_shared_memory}, {"far_lists", far_lists}, {"rope_parts_ends", rope_parts_ends},
                                                   {"many_chunks", many_chunks}, {"large_rotations", large_rotations}};
  const auto it = argc > 1 ? checks.find(argv[1]) : checks.end();
  if (it == checks.end()) return 2;
  const int rc = it->second();
  if (rc == 0) puts("ok");
  return rc;
}
