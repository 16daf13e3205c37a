// The same as host_harness.cpp, whose stand-in runtime and checks it takes, for the entry points on a cache in
// pages: their whole host logic at ordinary, smallest and largest sizes and at refusals.
#define main host_harness_main
#include "host_harness.cpp"
#undef main

namespace {
struct PagesShape {
  int64_t Tq;
  int S, prefixes, Hq, Hk, D, page_size, columns, count;
};

void pages_path(const PagesShape& x, tdq_dtype dt) {
  char tag[160];
  snprintf(tag, sizeof tag, "pages Tq=%lld S=%d G=%d %d/%d D=%d P=%d columns=%d count=%d dt=%d", (long long)x.Tq, x.S,
           x.prefixes, x.Hq, x.Hk, x.D, x.page_size, x.columns, x.count, (int)dt);
  const std::string t = tag;
  const tdq_heads Q = {dev<void>(0), (int64_t)x.Hq * x.D, x.D}, K = {dev<void>((size_t)1 << 36), (int64_t)x.Hk * x.D, x.D};
  const tdq_heads lo = {dev<void>((size_t)2 << 36), (int64_t)x.Hk * x.D, x.D}, hi = {dev<void>((size_t)3 << 36), (int64_t)x.Hk * x.D, x.D};
  const int64_t row = (int64_t)x.Hk * x.D;
  const tdq_pages Kc = {dev<void>((size_t)4 << 36), row * x.page_size, row, x.D}, Vc = {dev<void>((size_t)5 << 36), row * x.page_size, row, x.D};
  const int32_t* ints = dev<int32_t>((size_t)6 << 36);
  const tdq_sequences seq = {ints, ints, ints, x.columns, x.S, x.columns, 1 << 20, x.page_size};
  const tdq_sequences pre = {ints, ints, ints, x.columns, x.prefixes, x.columns, 1 << 20, x.page_size};
  const tdq_sequences all = {nullptr, ints, ints, x.columns, x.S, x.columns, 1 << 20, x.page_size};
  float* f = dev<float>((size_t)7 << 36);
  int32_t* chosen = dev<int32_t>((size_t)8 << 36);
  char* work = dev<char>((size_t)9 << 36);
  const int first = x.count > 1, last = x.count > 2;

  if (x.Hq + 2 * x.Hk <= 4096) {
    for (const int R : {0, 8, x.D})
      expect_ok((t + " append").c_str(), tdq_cache_append(&Q, &K, &K, dt, x.Tq, &seq, x.Hq, x.Hk, x.D, f, nullptr, 1e-6f, R, R == 8,
                                                          nullptr, 0, 0, nullptr, R ? f : nullptr, &Q, &Kc, &Vc, nullptr));
    expect_ok((t + " append, no queries").c_str(), tdq_cache_append(nullptr, &K, &K, dt, x.Tq, &seq, 0, x.Hk, x.D, nullptr, f, 0.f, x.D, 0,
                                                                    ints, x.Tq, 1, ints, f, nullptr, &Kc, &Vc, nullptr));
  }
  expect_ok((t + " bounds").c_str(), tdq_page_bounds(&Kc, dt, x.Tq, &seq, x.Hk, x.D, &lo, &hi, nullptr));
  expect_ok((t + " bounds of all").c_str(), tdq_page_bounds(&Kc, dt, 0, &all, x.Hk, x.D, &lo, &hi, nullptr));

  size_t need = tdq_select_pages_workspace_bytes(x.Tq, x.Hk, x.columns);
  if (need != (size_t)x.Tq * x.Hk * x.columns * 4) fail("%s: workspace of the choice %zu", tag, need);
  auto choice = [&](void* w, size_t n) {
    return tdq_select_pages(&Q, &lo, &hi, dt, x.Tq, &seq, x.Hq, x.Hk, x.D, 1, first, last, x.count, chosen, w, n, nullptr);
  };
  expect_ok((t + " choice").c_str(), choice(work, need));
  expect_err((t + " choice, small workspace").c_str(), choice(work, need - 1), TDQ_ERR_WORKSPACE);
  expect_err((t + " choice, misaligned workspace").c_str(), choice(work + 128, need), TDQ_ERR_WORKSPACE);

  need = tdq_attention_selected_workspace_bytes(x.Tq, x.Hq, x.Hk, x.D, x.page_size, x.count);
  auto selected = [&](void* w, size_t n) {
    return tdq_attention_selected(&Q, &Kc, &Vc, dt, x.Tq, &seq, x.Hq, x.Hk, x.D, 0.1f, 1, chosen, x.count, &Q, f, w, n, nullptr);
  };
  expect_ok((t + " chosen").c_str(), selected(need ? work : nullptr, need));
  if (need) {
    // two numbers and a row for each part
    if (need % ((size_t)x.Tq * x.Hq) == 0 && need / ((size_t)x.Tq * x.Hq) < 2u * (x.D + 2) * 4) fail("%s: parts", tag);
    expect_err((t + " chosen, no workspace").c_str(), selected(nullptr, need), TDQ_ERR_WORKSPACE);
    expect_err((t + " chosen, small workspace").c_str(), selected(work, need - 1), TDQ_ERR_WORKSPACE);
  }

  size_t without = 0;
  for (const int prefixes : {0, x.prefixes}) {
    need = tdq_attention_paged_workspace_bytes(x.Tq, x.S, prefixes, x.Hq, x.Hk, x.D);
    if (need == 0 || need < without || need % 256) fail("%s: workspace of the attention %zu", tag, need);
    if (prefixes && need - without < (size_t)x.Tq * x.Hq * 2 * (x.D + 2) * 4) fail("%s: no room for whole rows", tag);
    without = need;
    auto paged = [&](void* w, size_t n) {
      return tdq_attention_paged(&Q, &Kc, &Vc, dt, x.Tq, &seq, prefixes ? &pre : nullptr, x.Hq, x.Hk, x.D, -0.1f, 1, &Q, f, w, n,
                                 nullptr);
    };
    expect_ok((t + " paged").c_str(), paged(work, need));
    if (prefixes == 0 && x.prefixes == 0) break;
    expect_err((t + " paged, small workspace").c_str(), paged(work, need - 1), TDQ_ERR_WORKSPACE);
    expect_err((t + " paged, misaligned workspace").c_str(), paged(work + 8, need), TDQ_ERR_WORKSPACE);
  }
}
}  // namespace

int main() {
  g_dev = static_cast<unsigned char*>(
      mmap(nullptr, kDevSpan, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
  if (g_dev == MAP_FAILED) {
    perror("mmap");
    return 2;
  }
  g_symbol_mem = g_dev + ((size_t)15 << 36);
  // single tokens, prompts, the smallest, the most heads, sequences, tokens, columns and chosen pages
  const PagesShape shapes[] = {
      {16, 16, 1, 32, 8, 128, 64, 500, 64},      {2257, 4, 3, 32, 8, 128, 16, 600, 32},  {1, 1, 0, 1, 1, 8, 16, 1, 1},
      {5000, 7, 100, 16, 2, 256, 1024, 1200, 3}, {300, 300, 299, 7, 7, 96, 32, 20, 20},  {3, 2, 1, 4096, 4096, 8, 16, 9, 4},
      {3, 2, 1, 4096, 1, 256, 16, 9, 4},         {1 << 20, 1 << 20, 1 << 20, 2, 1, 64, 16, 8, 2},
      {1 << 30, 1, 1, 2, 1, 8, 1024, 16, 1},     {1, 1, 1, 1, 1, 200, 16, 1 << 26, 1 << 20},
      {1 << 30, 9, 0, 1, 1, 40, 64, 64, 64},     {40, 40, 1, 24, 1, 184, 128, 1 << 20, 7},
  };
  for (const PagesShape& s : shapes)
    for (const tdq_dtype dt : {TDQ_F16, TDQ_BF16}) pages_path(s, dt);
  printf("%d calls checked, %d failures\n", g_calls, g_fail);
  return g_fail ? 1 : 0;
}
