// The launches of the rows to the experts and of the losses on given answers, noted as in host_launch_driver.cpp, from which the stand-in for the
// HIP runtime comes: grids within their limits at the largest sizes, and workgroups that make up the whole of a job.
// Built and run by tests/test_host_answers_rows.py.
#define main launches_of_the_other_entry_points
#include "host_launch_driver.cpp"
#undef main

static std::map<std::string, int64_t> noted(const char* what) {
  std::map<std::string, int64_t> blocks;
  for (const Launch& l : launches)
    for (const char* n : {"answers_kernel", "pairs_kernel", "count_rows_kernel", "place_rows_kernel", "copy_rows_kernel", "dispatch_few_rows_kernel",
                          "dispatch_many_rows_kernel", "combine_rows_kernel", "combine_rows_backward_kernel"})
      if (l.kernel.find(n) != std::string::npos) blocks[n] += l.grid.x;
  check(what);
  return blocks;
}

int main() {
  auto at = [](int64_t i) { return (void*)((uintptr_t)(i + 1) << 44); };   // never read
  auto f = [&](int64_t i) { return (float*)at(i); };
  auto n32 = [&](int64_t i) { return (int32_t*)at(i); };
  auto n64 = [&](int64_t i) { return (int64_t*)at(i); };
  const size_t room = ~(size_t)0;

  // ---- losses: rows of every workgroup size, as many as there can be
  for (moep_dtype dt : {MOEP_F32, MOEP_BF16})
    for (int64_t T : {(int64_t)1, (int64_t)7, (int64_t)600, ((int64_t)1 << 22) - 1, ((int64_t)1 << 22) + 1001, (int64_t)1 << 30})
      for (int64_t V : {1, 3, 4096, 8000, 50000, 131072, 1000000, 1 << 28}) {
        char what[96];
        std::snprintf(what, sizeof what, "losses of %" PRId64 " rows of %" PRId64 " logits, dtype %d", T, V, (int)dt);
        EXPECT(moe_policy_loss(at(1), V, n64(2), f(3), f(4), f(5), T, V, dt, .2f, .2f, .1f, 1.f, f(6), f(7), f(8), f(9), nullptr, 0, nullptr) == MOEP_OK);
        EXPECT(noted(what)["answers_kernel"] == T);
        EXPECT(moe_policy_loss(at(1), V, n64(2), f(3), f(4), f(5), T, V, dt, .2f, .2f, .1f, 1.f, f(6), f(7), f(8), f(9), at(10), V, nullptr) == MOEP_OK);
        EXPECT(noted(what)["answers_kernel"] == T);
        EXPECT(moe_policy_loss_backward(at(1), V, n64(2), f(3), f(4), T, V, dt, 1.f, at(10), V, nullptr) == MOEP_OK);
        int64_t n = noted(what)["answers_kernel"];
        EXPECT(n % T == 0 && n >= T && (n == T || n <= 1024));
        for (int64_t pairs : {(int64_t)0, (int64_t)1, (int64_t)1 << 22}) {
          EXPECT(moe_preference_loss(at(1), V, n64(2), n64(3), f(4), T, V, pairs, dt, .1f, 0.f, 1, f(5), f(6), f(7), f(8), f(9), at(10), V, nullptr) == MOEP_OK);
          auto b = noted(what);
          EXPECT(b["pairs_kernel"] == pairs && b["answers_kernel"] == T + (pairs ? n : 0));
        }
      }

  // ---- rows
  for (moep_dtype dt : {MOEP_F32, MOEP_BF16})
    for (int k : {1, 2, 7, 16})
      for (int64_t T : {(int64_t)0, (int64_t)1, (int64_t)64, (int64_t)300, (int64_t)512, (int64_t)8192, (int64_t)100001, ((int64_t)1 << 30) / k})
        for (int H : {64, 4096, 1 << 24})
          for (int E : {1, 32}) {
            char what[96];
            std::snprintf(what, sizeof what, "%" PRId64 " tokens of %d, k %d, E %d, dtype %d", T, H, k, E, (int)dt);
            const int64_t chunks = (int64_t)H * (dt == MOEP_BF16 ? 2 : 4) / 16, R = T * k;
            const size_t ws = moe_dispatch_rows_workspace(T, k, E);
            EXPECT((ws > 0) == (R > 8192) && ws <= 8192 * 4);
            EXPECT(moe_dispatch_rows(at(1), n32(2), n32(3), T, k, E, H, dt, at(4), n32(5), n32(6), at(7), room, nullptr) == MOEP_OK);
            auto b = noted(what);
            if (R <= 256) EXPECT(b["dispatch_few_rows_kernel"] == (T ? T : 1));
            else if (R <= 8192) EXPECT(b["dispatch_many_rows_kernel"] <= 512 && b["dispatch_many_rows_kernel"] * up(T, 512) >= T && up(T, 512) * k <= 64);
            else EXPECT(b["place_rows_kernel"] == b["count_rows_kernel"] && b["place_rows_kernel"] * E * 4 == (int64_t)ws && b["copy_rows_kernel"] * 256 >= T * chunks);
            if (!T) continue;
            EXPECT(moe_dispatch_rows_backward(at(1), n32(2), T, k, H, R, dt, at(3), nullptr) == MOEP_OK);
            EXPECT(noted(what)["combine_rows_kernel"] * 256 >= T * chunks);
            EXPECT(moe_combine_rows(at(1), n32(2), f(3), T, k, H, R, dt, at(4), nullptr) == MOEP_OK);
            EXPECT(noted(what)["combine_rows_kernel"] * 256 >= T * chunks);
            EXPECT(moe_combine_rows_backward(at(1), at(2), n32(3), f(4), T, k, H, R, dt, at(5), f(6), nullptr) == MOEP_OK);
            const int64_t n = noted(what)["combine_rows_backward_kernel"];
            EXPECT(n == T || (n * 4 >= up(T, 8) && chunks < 256));
          }
  if (!failures) std::printf("all checks passed\n");
  return failures != 0;
}
