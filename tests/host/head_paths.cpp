// Which tiles, remainders and shared contractions the calls of the head's loss take: reads lines "tokens width words tied" (dense rows at
// 16-byte positions) and prints a line of names for each.
#include <cstdio>
#include <set>
#include <string>

#include "../../paper_2607_19058_amd/csrc/head_plan.h"

using namespace moe;
typedef std::set<std::string> Names;

static void logits(Names &n, const std::string &what, int mode, const HeadProduct &p) {
  const LogitsChoice c = choose_logits(mode, p);
  n.insert(what + "/" + std::to_string(c.tile));
  if (c.first < p.cols) n.insert(what + "/rest/" + std::to_string(c.rest));
}
static std::string choice(const ResultChoice &c, bool fold) { return std::to_string(c.tile) + (c.parts > 1 || fold ? "/shared" : "/one"); }
static void result(Names &n, const std::string &what, int mode, const HeadProduct &p, bool fold) {
  const ResultPlan s = plan_result(mode, p, fold);
  n.insert(what + "/" + choice(s.main, fold));
  if (s.rest.parts) n.insert(what + (s.rows < p.rows ? "/rows/" : "/columns/") + choice(s.rest, fold));
}

int main() {
  long long T, d, V;
  int by_row;
  while (scanf("%lld %lld %lld %d", &T, &d, &V, &by_row) == 4) {
    skew_head_desc h = {};
    h.x = h.w = h.targets = reinterpret_cast<const void *>(4096);
    h.tokens = T;
    h.d = d;
    h.vocab = V;
    h.ldx = d;
    h.ldw = by_row ? d : V;
    h.flags = by_row ? SKEW_TRANSPOSE : 0;
    h.target_bytes = 8;
    h.scale = 1.0f;
    Names n;
    const std::string layout = by_row ? "tied" : "untied";
    const ForwardPlan f = forward_plan(h);
    if (f.few) n.insert("few");
    for (int64_t t0 = 0; t0 < T && !f.few; t0 += f.run)
      for (int64_t v0 = 0; v0 < V; v0 += f.piece)
        logits(n, "loss/" + layout, mode_of(h), logits_of(h, f, nullptr, 0, std::min<int64_t>(f.run, T - t0), v0, nullptr));
    const BackwardPlan b = backward_plan(h);
    const std::string kind = std::string(b.split ? "two/" : "half/") + layout;
    for (int64_t v0 = 0; v0 < V; v0 += b.piece) {
      logits(n, "G/" + kind, mode_of(h), logits_of(h, b, nullptr, 0, T, v0, nullptr));
      result(n, "dx/" + kind + (v0 ? "/more" : ""), dx_mode(h), dx_of(h, b, nullptr, nullptr, v0), b.split);
      result(n, "dw/" + kind, kOuter, dw_of(h, b, nullptr, nullptr, v0), false);
    }
    for (const std::string &s : n) printf("%s ", s.c_str());
    printf("\n");
  }
  return 0;
}
