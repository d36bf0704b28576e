// Host-only checks of latent attention (csrc/kvx_latent_host.cpp), built by
// tests/test_latent_host.py with the sanitizers.  The argument names the check.  Nothing is
// launched: a call whose arguments were accepted ends with KVX_EHIP where there is no device.

#include "kvx_latent_host.cpp"

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <string>
#include <tuple>

namespace kvx {
static std::string g_message;
int report(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_message = buf;
  return code;
}
#define KVX_STUB(name, ...) \
  hipError_t name(__VA_ARGS__) { std::exit(4); }
KVX_STUB(launch_store_latent, const LatentStoreParams&, int64_t, int, bool, bool, hipStream_t)
KVX_STUB(launch_load_latent, const LatentLoadParams&, int64_t, int, bool, hipStream_t)
KVX_STUB(launch_latent_attention, const LatentAttnParams&, int64_t, const LatentSmallPlan*, const LatentRowPlan*, int,
         bool, int, hipStream_t)
KVX_STUB(launch_latent_merge, const LatentMergeParams&, int64_t, const LatentSmallPlan*, const LatentRowPlan*, int,
         int, hipStream_t)
KVX_STUB(launch_latent_absorb, const LatentProjParams&, int64_t, int, int, hipStream_t)
KVX_STUB(launch_latent_output, const LatentProjParams&, int64_t, int, int, hipStream_t)
KVX_STUB(launch_latent_expand, const LatentExpandParams&, int64_t, int, int, bool, hipStream_t)
KVX_STUB(launch_latent_prefill, const LatentPrefillParams&, int64_t, int, hipStream_t)
KVX_STUB(launch_latent_tile_merge, const LatentTileMergeParams&, int64_t, int, hipStream_t)
}  // namespace kvx

#define CHECK(cond)                                                           \
  do {                                                                        \
    if (!(cond)) {                                                            \
      std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #cond, kvx::g_message.c_str()); \
      std::exit(3);                                                           \
    }                                                                         \
  } while (0)

namespace {

struct TestBatch {
  std::vector<int32_t> P, E, indptr{0};
  int32_t ids = 0;
  kvx_batch b{};
  void add(int32_t p, int32_t e) {
    P.push_back(p);
    E.push_back(e);
    indptr.push_back(indptr.back() + (int32_t)(((int64_t)p + e + 15) / 16));
  }
  const kvx_batch* get() {
    b = kvx_batch{(int32_t)P.size(), P.data(), E.data(), indptr.data(), &ids};
    return &b;
  }
};

void* addr(uintptr_t a) { return (void*)a; }

// ---------------------------------------------------------------- refusals

void refusals() {
  kvx_latent_pool* out = nullptr;
  CHECK(latent_pool_create(10, 16, 512, 64, 0, nullptr) == KVX_EINVAL);
  CHECK(latent_pool_create(0, 16, 512, 64, 0, &out) == KVX_EINVAL);
  CHECK(latent_pool_create(1ll << 31, 16, 512, 64, 0, &out) == KVX_EINVAL);
  CHECK(latent_pool_create(10, 32, 512, 64, 0, &out) == KVX_EUNSUPPORTED);
  CHECK(latent_pool_create(10, 16, 384, 64, 0, &out) == KVX_EUNSUPPORTED);
  CHECK(latent_pool_create(10, 16, 512, 32, 0, &out) == KVX_EUNSUPPORTED);
  CHECK(latent_pool_create(10, 16, 512, 64, 2, &out) == KVX_EINVAL);
  CHECK(out == nullptr);
  CHECK(latent_pool_destroy(nullptr) == KVX_OK);
  kvx_latent_layout lay;
  CHECK(latent_pool_layout(nullptr, &lay) == KVX_EINVAL);

  kvx_latent_pool pool;
  pool.num_pages = 100;
  pool.latent_dim = 512;
  pool.page_bytes = 18432;
  CHECK(latent_pool_layout(&pool, nullptr) == KVX_EINVAL);
  CHECK(latent_pool_layout(&pool, &lay) == KVX_OK && lay.key_offset == 1024 && lay.scale_offset == 0);
  CHECK(latent_pool_set_split_keys(&pool, 63) == KVX_EINVAL);
  CHECK(latent_pool_set_split_keys(&pool, -64) == KVX_EINVAL);
  CHECK(latent_pool_set_split_keys(nullptr, 64) == KVX_EINVAL);

  TestBatch one, none, bad;
  one.add(20, 3);
  none.add(20, 0);
  bad.add(20, 3);
  bad.indptr.back() = 1;  // 23 tokens need two pages
  void* kv = addr(0x10000);
  const int64_t ok = 576;
  CHECK(store_latent(nullptr, one.get(), kv, ok, nullptr) == KVX_EINVAL);
  CHECK(store_latent(&pool, nullptr, kv, ok, nullptr) == KVX_EINVAL);
  CHECK(store_latent(&pool, bad.get(), kv, ok, nullptr) == KVX_EINVAL);
  CHECK(store_latent(&pool, one.get(), nullptr, ok, nullptr) == KVX_EINVAL);
  CHECK(store_latent(&pool, one.get(), addr(0x10008), ok, nullptr) == KVX_EINVAL);
  for (int64_t stride : {(int64_t)0, ok - 8, ok + 4, (int64_t)-576, ((int64_t)1 << 40) + 8})
    CHECK(store_latent(&pool, one.get(), kv, stride, nullptr) == KVX_EINVAL);
  CHECK(store_latent(&pool, none.get(), nullptr, ok, nullptr) == KVX_OK);
  CHECK(load_latent(&pool, one.get(), nullptr, ok, nullptr) == KVX_EINVAL);
  CHECK(load_latent(&pool, one.get(), addr(0x10004), ok, nullptr) == KVX_EINVAL);
  CHECK(load_latent(&pool, one.get(), kv, 575, nullptr) == KVX_EINVAL);
  CHECK(load_latent(&pool, none.get(), nullptr, ok, nullptr) == KVX_OK);

  kvx_rope rope{10000.0, nullptr, 64, KVX_ROPE_HALF, nullptr, nullptr, 1e-6f};
  auto with = [&](const kvx_rope* r, const void* q, int32_t hq, int32_t qd, void* qo) {
    return store_latent_rope(&pool, one.get(), r, q, hq, qd, qo, kv, ok, nullptr);
  };
  void *q = addr(0x100000), *qo = addr(0x200000);
  CHECK(with(nullptr, q, 4, 192, qo) == KVX_EINVAL);
  kvx_rope r = rope;
  r.rotary_dim = 32;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  r = rope, r.style = 2;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  r = rope, r.theta = 0.0;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  r = rope, r.norm_eps = -1.0f;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  r = rope, r.norm_eps = NAN;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  r = rope, r.q_norm = q;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  r = rope, r.k_norm = addr(0x10002);
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  double rates[32] = {};
  rates[31] = -1.0;
  r = rope, r.inv_freq = rates;
  CHECK(with(&r, q, 4, 192, qo) == KVX_EINVAL);
  CHECK(with(&rope, q, -1, 192, qo) == KVX_EINVAL);
  CHECK(with(&rope, q, 1025, 192, qo) == KVX_EINVAL);
  CHECK(with(&rope, nullptr, 4, 192, qo) == KVX_EINVAL);
  CHECK(with(&rope, q, 4, 192, nullptr) == KVX_EINVAL);
  for (int qd : {56, 196, 4104, 0}) CHECK(with(&rope, q, 4, qd, qo) == KVX_EINVAL);
  CHECK(with(&rope, addr(0x100008), 4, 192, qo) == KVX_EINVAL);
  CHECK(with(&rope, q, 4, 192, addr(0x100000 + 16)) == KVX_EINVAL);                  // overlaps
  CHECK(with(&rope, q, 4, 192, addr(0x100000 + 3 * 4 * 192 * 2 - 16)) == KVX_EINVAL);
  const int free_ = with(&rope, q, 4, 192, addr(0x100000 + 3 * 4 * 192 * 2));        // side by side
  const int same = with(&rope, q, 4, 192, q);
  CHECK(free_ != KVX_EINVAL && same != KVX_EINVAL);

  auto attend = [&](const kvx_batch* b, const void* qq, int32_t hq, float sc, void* o) {
    return latent_attention(&pool, b, qq, hq, sc, o, nullptr, nullptr);
  };
  CHECK(latent_attention(nullptr, one.get(), q, 16, 0.1f, qo, nullptr, nullptr) == KVX_EINVAL);
  for (int hq : {0, -1, 1025}) CHECK(attend(one.get(), q, hq, 0.1f, qo) == KVX_EINVAL);
  for (float sc : {0.0f, -1.0f, 3e38f, INFINITY, NAN}) CHECK(attend(one.get(), q, 16, sc, qo) == KVX_EINVAL);
  CHECK(attend(one.get(), nullptr, 16, 0.1f, qo) == KVX_EINVAL);
  CHECK(attend(one.get(), q, 16, 0.1f, nullptr) == KVX_EINVAL);
  CHECK(attend(one.get(), addr(0x100002), 16, 0.1f, qo) == KVX_EINVAL);
  CHECK(attend(none.get(), nullptr, 16, 0.1f, nullptr) == KVX_OK);
  TestBatch huge;
  huge.add(0, 1 << 22);
  CHECK(attend(huge.get(), q, 1024, 0.1f, qo) == KVX_EUNSUPPORTED);

  TestBatch far;
  far.add((1ll << 31) - (1 << 23), 1);
  CHECK(attend(far.get(), q, 1, 0.1f, qo) == KVX_EUNSUPPORTED);

  kvx_latent_proj proj{addr(0x300000), addr(0x400000), 16, 128, 128};
  auto extend = [&](const kvx_latent_proj* p, int form) {
    return latent_extend_attention(&pool, one.get(), p, q, 0.1f, qo, nullptr, form, nullptr);
  };
  CHECK(extend(nullptr, 0) == KVX_EINVAL);
  CHECK(extend(&proj, 3) == KVX_EINVAL);
  CHECK(extend(&proj, -1) == KVX_EINVAL);
  kvx_latent_proj p = proj;
  p.nope_dim = 96;
  CHECK(extend(&p, 0) == KVX_EUNSUPPORTED);
  p = proj, p.v_dim = 64;
  CHECK(extend(&p, 0) == KVX_EUNSUPPORTED);
  p = proj, p.num_q_heads = 0;
  CHECK(extend(&p, 0) == KVX_EINVAL);
  p = proj, p.w_uk = nullptr;
  CHECK(extend(&p, 0) == KVX_EINVAL);
  p = proj, p.w_uv = addr(0x400001);
  CHECK(extend(&p, 0) == KVX_EINVAL);
  CHECK(latent_extend_attention(&pool, none.get(), &proj, nullptr, 0.1f, nullptr, nullptr, 0, nullptr) == KVX_OK);
}

// ---------------------------------------------------------------- plans

TestBatch random_batch(std::mt19937& rng, int kind) {
  auto pick = [&](int a, int b) { return std::uniform_int_distribution<int>(a, b)(rng); };
  TestBatch t;
  const int n = kind == 3 ? pick(129, 300) : pick(1, kind == 0 ? 12 : 40);
  for (int i = 0; i < n; i++) {
    int p = pick(0, 3) == 0 ? pick(0, 70) : pick(0, kind == 1 ? 60000 : 5000);
    int e = kind == 1 || kind == 3 ? 1 : pick(0, 5) == 0 ? 0 : pick(1, kind == 2 ? 400 : 7);
    t.add(p, e);
  }
  return t;
}

// Every (row, key that it sees) is covered exactly once, by ranges that start at multiples of
// 64; parts of a tile are numbered as its merge says.
void absorbed_plans() {
  std::mt19937 rng(7);
  int seen_rows = 0, seen_small = 0, seen_memory = 0, seen_parts = 0;
  for (int round = 0; round < 400; round++) {
    TestBatch t = random_batch(rng, round % 4);
    const int Hq = (int[]){1, 5, 16, 33, 128}[rng() % 5];
    const int split = rng() % 3 == 0 ? 64 * (1 + (int)(rng() % 40)) : 0;
    const kvx_batch* b = t.get();
    std::vector<Member> members;
    int64_t row = 3;
    for (int r = 0; r < b->num_reqs; r++)
      if (b->extend_lens[r] > 0) {
        members.push_back({r, row});
        row += b->extend_lens[r] + rng() % 2;
      }
    if (members.empty()) continue;
    AbsorbedPlan plan;
    plan_absorbed(b, members, Hq, 512, split, plan);
    // the units, as the kernels take them
    std::vector<LatentUnit> units;
    std::vector<LatentMerge> merges;
    if (plan.in_args && plan.rows.n > 0) {
      seen_rows++;
      const kvx::LatentRowPlan& rp = plan.rows;
      CHECK(rp.n <= kvx::kLatRowReqs);
      for (int i = 0; i < rp.n_units; i++) {
        int r = 0;
        while (r + 1 < kvx::kLatRowReqs && rp.first[r + 1] <= i) r++;
        const int c = i - rp.first[r], end = rp.prefix[r] + rp.extend[r];
        units.push_back({0, rp.extend[r] * Hq, rp.qo[r], rp.prefix[r], rp.page_base[r], c * rp.len[r],
                         std::min(end, (c + 1) * rp.len[r]), end > rp.len[r] ? rp.part0[r] + c : -1});
        if (i > 0) CHECK(rp.len[r] <= rp.len[0]);
      }
      for (int r = 0; r < rp.n; r++) {
        const int end = rp.prefix[r] + rp.extend[r];
        if (end > rp.len[r])
          merges.push_back({0, rp.extend[r] * Hq, rp.qo[r], rp.part0[r], (end + rp.len[r] - 1) / rp.len[r], 0});
      }
      CHECK(merges.empty() == plan.merges.empty());
    } else if (plan.in_args) {
      seen_small++;
      CHECK(plan.small.n_tiles <= kvx::kLatSmallTiles && plan.small.n_units <= kvx::kLatSmallUnits);
      for (int i = 0; i < plan.small.n_units; i++) {
        const uint16_t code = plan.small.code[i];
        if (code == kvx::kLatNoUnit) continue;
        CHECK((code >> 10) < plan.small.n_tiles);
        const kvx::LatentSmallTile& s = plan.small.tile[code >> 10];
        const int c = code & (kvx::kLatSmallParts - 1);
        units.push_back({s.row0, s.nrows, s.qo, s.prefix, s.page_base, c * s.len, std::min(s.key_end, (c + 1) * s.len),
                         s.key_end > s.len ? s.part0 + c : -1});
      }
      merges = plan.merges;
    } else {
      seen_memory++;
      CHECK(plan.units.size() % 8 == 0 || plan.units.back().nrows > 0);
      for (const LatentUnit& u : plan.units)
        if (u.nrows > 0) units.push_back(u);
      merges = plan.merges;
    }
    const int M = 16 * plan.row_blocks;
    std::map<std::pair<int, int>, std::vector<LatentUnit>> tiles;  // (qo, row0)
    std::vector<char> used((size_t)plan.n_parts, 0);
    for (const LatentUnit& u : units) {
      CHECK(u.nrows >= 1 && u.nrows <= M && u.row0 % M == 0 && u.key_begin % 64 == 0 && u.key_begin < u.key_end);
      if (u.part >= 0) {
        CHECK(u.part < plan.n_parts && !used[(size_t)u.part]);
        used[(size_t)u.part] = 1;
        seen_parts++;
      }
      tiles[{u.qo, u.row0}].push_back(u);
    }
    CHECK((int64_t)plan.n_parts * M * 513 * 4 <= kMaxPartBytes);
    std::map<std::pair<int, int>, LatentMerge> by_tile;
    for (const LatentMerge& m : merges) CHECK(by_tile.emplace(std::make_pair(m.qo, m.row0), m).second);
    size_t n_tiles = 0;
    for (const Member& m : members) {
      const int64_t P = b->prefix_lens[m.req], rows = (int64_t)b->extend_lens[m.req] * Hq;
      for (int64_t r0 = 0; r0 < rows; r0 += M, n_tiles++) {
        auto& us = tiles[{(int)m.row, (int)r0}];
        CHECK(!us.empty());
        std::sort(us.begin(), us.end(), [](const LatentUnit& a, const LatentUnit& c) { return a.key_begin < c.key_begin; });
        const int64_t nrows = std::min<int64_t>(M, rows - r0);
        int64_t key = 0;
        for (size_t i = 0; i < us.size(); i++) {
          const LatentUnit& u = us[i];
          CHECK(u.key_begin == key && u.nrows == nrows && u.prefix == P && u.page_base == b->page_indptr[m.req]);
          key = u.key_end;
          if (us.size() == 1) {
            CHECK(u.part == -1);
          } else {
            const LatentMerge& mg = by_tile.at({(int)m.row, (int)r0});
            CHECK(mg.nparts == (int)us.size() && u.part == mg.part0 + (int)i && mg.nrows == u.nrows);
          }
        }
        CHECK(key == P + (r0 + nrows - 1) / Hq + 1);
      }
    }
    CHECK(tiles.size() == n_tiles);
  }
  CHECK(seen_rows > 10 && seen_small > 10 && seen_memory > 10 && seen_parts > 100);
}

void expanded_plans() {
  std::mt19937 rng(11);
  int seen_parts = 0;
  for (int round = 0; round < 200; round++) {
    TestBatch t = random_batch(rng, round % 2 ? 2 : 0);
    const int heads = (int[]){1, 3, 16}[rng() % 3];
    const kvx_batch* b = t.get();
    std::vector<int64_t> qo;
    CHECK(check_batch(b, qo) == KVX_OK);
    std::vector<int32_t> reqs;
    for (int r = 0; r < b->num_reqs; r++)
      if (b->extend_lens[r] > 0 && rng() % 4) reqs.push_back(r);
    if (reqs.empty()) continue;
    std::vector<LatentExpandUnit> x;
    std::vector<int64_t> x_row;
    const int64_t x_rows = expand_units(b, reqs, x, x_row);
    std::vector<char> row_of((size_t)x_rows, 0);
    for (const LatentExpandUnit& u : x) {
      CHECK(u.nrows > 0 && u.nrows <= 256 && u.nrows % 64 == 0 && u.key0 < u.key_end && u.x_row + u.nrows <= x_rows);
      for (int i = 0; i < u.nrows; i++) CHECK(!row_of[(size_t)(u.x_row + i)]++);
    }
    for (char c : row_of) CHECK(c);
    ExpandedPlan plan;
    plan_expanded(b, qo, reqs, x_row, heads, 128, plan);
    std::map<std::tuple<int, int>, std::vector<LatentTile>> tiles;
    std::vector<char> used((size_t)plan.n_parts, 0);
    for (const LatentTile& u : plan.units) {
      if ((u.head_ntok & 0xFFFF) == 0) continue;
      CHECK(u.key_begin % 64 == 0 && u.key_begin < u.key_end && (u.head_ntok >> 16) < heads);
      if (u.part >= 0) {
        CHECK(u.part < plan.n_parts && !used[(size_t)u.part]);
        used[(size_t)u.part] = 1;
        seen_parts++;
      }
      tiles[{u.qo_row, u.head_ntok >> 16}].push_back(u);
    }
    size_t n = 0;
    for (size_t i = 0; i < reqs.size(); i++) {
      const int r = reqs[i];
      const int64_t P = b->prefix_lens[r], E = b->extend_lens[r];
      for (int h = 0; h < heads; h++)
        for (int64_t t0 = 0; t0 < E; t0 += kvx::kLatTileTok, n++) {
          auto& us = tiles[{(int)(qo[(size_t)r] + t0), h}];
          CHECK(!us.empty());
          std::sort(us.begin(), us.end(), [](const LatentTile& a, const LatentTile& c) { return a.key_begin < c.key_begin; });
          int64_t key = 0;
          for (const LatentTile& u : us) {
            CHECK(u.key_begin == key && (u.head_ntok & 0xFFFF) == std::min<int64_t>(kvx::kLatTileTok, E - t0));
            CHECK(u.pos0 == P + t0 && u.x_row == x_row[i] && u.x_row + (u.key_end + 63) / 64 * 64 <= x_rows);
            CHECK((us.size() == 1) == (u.part == -1));
            key = u.key_end;
          }
          CHECK(key == P + std::min<int64_t>(E, t0 + kvx::kLatTileTok));
        }
    }
    CHECK(tiles.size() == n);
    for (const LatentTileMerge& m : plan.merges) {
      const auto& us = tiles.at({m.qo_row, m.head_ntok >> 16});
      CHECK((int)us.size() == m.nparts);
      for (size_t i = 0; i < us.size(); i++) CHECK(us[i].part == m.part0 + (int)i);
    }
  }
  CHECK(seen_parts > 100);
}

// Launch orders hold every unit once and give no XCD more units than CUs while there are enough.
void orders() {
  std::mt19937 rng(3);
  for (int round = 0; round < 300; round++) {
    std::vector<Group> groups;
    int32_t units = 0;
    const int n = 1 + (int)(rng() % 60);
    for (int i = 0; i < n; i++) {
      const int32_t c = 1 + (int32_t)(rng() % 9);
      groups.push_back({1.0 + (double)(rng() % 50), units, c});
      units += c;
    }
    const std::vector<int32_t> order = spread(groups);
    std::vector<char> seen((size_t)units, 0);
    size_t on[8] = {};
    for (size_t i = 0; i < order.size(); i++)
      if (order[i] >= 0) {
        CHECK(order[i] < units && !seen[(size_t)order[i]]++);
        on[i % 8]++;
      }
    for (char c : seen) CHECK(c);
    if (units <= 256)
      for (size_t c : on) CHECK(c <= 32);
  }
}

// The forms: single tokens go absorbed, a long prompt expanded, whatever the heads.
void forms() {
  for (int hq : {4, 16, 128}) {
    TestBatch one, prompt, both;
    for (int i = 0; i < 64; i++) one.add(8000, 1);
    prompt.add(0, 8000);
    for (int i = 0; i < 64; i++) both.add(30000, 1);
    both.add(20000, 4000);
    const std::vector<bool> a = choose_forms(one.get(), hq, 512, 128), p = choose_forms(prompt.get(), hq, 512, 128),
                            m = choose_forms(both.get(), hq, 512, 128);
    for (int i = 0; i < 64; i++) CHECK(a[(size_t)i] && m[(size_t)i]);
    CHECK(!p[0] && !m[64]);
  }
}

}  // namespace

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "refusals") refusals();
  else if (what == "absorbed") absorbed_plans();
  else if (what == "expanded") expanded_plans();
  else if (what == "orders") orders();
  else if (what == "forms") forms();
  else return 2;
  std::printf("%s passed\n", what.c_str());
  return 0;
}
