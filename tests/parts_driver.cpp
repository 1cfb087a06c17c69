// Host checks of csrc/sfmp_parts.h: the parts of every total follow each other without a gap from 0 to the end, no part exceeds
// an equal share or the least one, and every page is in the workgroup that workgroup_of names.
#include <cstdio>
#include <cstdlib>

#include "../paper_2602_01027_amd/csrc/sfmp_parts.h"

static void fail(const char* what, int total, int workgroups, int waves, int least) {
  std::printf("%s: %d pages, %d x %d wavefronts, least %d\n", what, total, workgroups, waves, least);
  std::exit(1);
}

static void check(int total, int workgroups, int waves, int least) {
  const sfmp::Parts p(total, workgroups, waves, least);
  const int64_t n = (int64_t)workgroups * waves, share = (total + n - 1) / n > least ? (total + n - 1) / n : least;
  int64_t at = 0;
  for (int g = 0; g < workgroups; ++g) {
    const sfmp::Part whole = p.whole(g);
    if (whole.begin != at) fail("workgroup's first page", total, workgroups, waves, least);
    for (int w = 0; w < waves; ++w) {
      const sfmp::Part part = p.part(g, w);
      if (part.begin != at || part.end < part.begin || part.end > total) fail("gap or overlap", total, workgroups, waves, least);
      if (part.end - part.begin > share || (part.end < total && part.end - part.begin != share)) fail("share", total, workgroups, waves, least);
      at = part.end;
    }
    if (whole.end != at) fail("workgroup's end", total, workgroups, waves, least);
    if (whole.end > whole.begin && (p.workgroup_of(whole.begin) != g || p.workgroup_of(whole.end - 1) != g))
      fail("workgroup of a page", total, workgroups, waves, least);
  }
  if (at != total) fail("end", total, workgroups, waves, least);
}

int main() {
  const int forms[][3] = {{256, 8, 1}, {256, 4, 1}, {512, 1, 4}, {512, 1, 8}, {256, 1, 4}, {256, 1, 8}};
  for (const auto& f : forms) {
    for (int total = 0; total < 5000; ++total) check(total, f[0], f[1], f[2]);
    for (int back = 0; back < 5000; ++back) check(INT32_MAX - back, f[0], f[1], f[2]);
    for (int64_t total = 5000; total < INT32_MAX; total = total * 5 / 4 + 1) check((int)total, f[0], f[1], f[2]);
  }
  std::printf("ok\n");
}
