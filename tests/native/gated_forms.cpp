// Prints the form that each gated call on stdin takes, by the library's own rules:
//   f <type 0|1> <rows> <k> <k2> <n> <lead>
//   b <type> <rows> <k> <k2> <n> <lead> <ask: letters of x, 2, w, b>
// lead: elements by which x (and x2) lie behind an aligned place. For the
// gradients: how dz is made, dw's tiles, its parts (the steps of one and the rows
// of its last step) and its join, dx's tiles, its parts and their join.
#include <cstdio>
#include <cstring>

#include "../../paper_2410_22697_amd/csrc/gated_rules.hpp"

int main() {
  char line[256];
  while (std::fgets(line, sizeof line, stdin)) {
    char what, ask[16] = "";
    int type, k, k2, n, lead;
    long long rows;
    if (std::sscanf(line, "%c %d %lld %d %d %d %d %15s", &what, &type, &rows, &k, &k2, &n, &lead, ask) < 7) return 1;
    const char* at = (const char*)4096;  // aligned, and never followed
    const char* x = at + lead * ms::gated_size(type);
    const char* x2 = k2 ? x : nullptr;
    if (what == 'f') {
      massive_gated_args a = {};
      a.x = x, a.x_second = x2, a.w = at, a.rows = rows, a.x_stride = k, a.x_second_stride = k2, a.w_stride = k + k2;
      a.n = n, a.k = k, a.k_second = k2, a.type = type;
      if (ms::gated_few(&a)) std::printf("few\n");
      else std::printf("%s %s\n", ms::gated_narrow(&a) ? "narrow" : "wide", ms::gated_direct(&a) ? "direct" : "registers");
      continue;
    }
    massive_gated_grads a = {};
    a.x = x, a.x_second = x2, a.w = at, a.rows = rows, a.x_stride = k, a.x_second_stride = k2, a.w_stride = k + k2;
    a.n = n, a.k = k, a.k_second = k2, a.type = type;
    char* there = (char*)at;
    if (std::strchr(ask, 'x')) a.dx = there;
    if (std::strchr(ask, '2')) a.dx_second = there;
    if (std::strchr(ask, 'w')) a.dw = there;
    if (std::strchr(ask, 'b')) a.dbias = there;
    const ms::GatedPlan p = ms::gated_plan(&a);
    const int step = ms::kTileStepBytes / ms::gated_size(type);
    const bool made = ms::gated_dw_made(&a, p);
    std::printf("%s", made ? "made" : a.dbias && p.in_units ? "sums" : "dz");
    if (a.dw) {
      const int64_t part = rows < p.dw.part ? rows : p.dw.part, last = rows - (p.dw.parts - 1) * p.dw.part;
      std::printf(" dw %s %s parts %lld steps %lld rest %lld ways %d", p.dw.nb == 2 ? "narrow" : "wide",
                  made || ms::gated_dw_direct(&a) ? "direct" : "registers", (long long)p.dw.parts, (long long)((part + step - 1) / step),
                  (long long)(last % step), ms::gated_ways(p.dw.parts, 2 * (int64_t)n * (k + k2)));
    }
    if (a.dx || a.dx_second) {
      const int64_t cols = (a.dx ? k : 0) + (a.dx_second ? k2 : 0);
      std::printf(" dx %s %s parts %lld ways %d", p.dx.nb == 2 ? "narrow" : "wide", ms::gated_dx_direct(&a) ? "direct" : "registers",
                  (long long)p.dx.parts, ms::gated_ways(p.dx.parts, rows * cols));
    }
    std::printf("\n");
  }
  return 0;
}
