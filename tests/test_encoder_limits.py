"""CPU-side checks of the attention's work lists at their limits."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_03199_amd", "csrc")


def _run(tmp_path, name, text):
    src, exe = tmp_path / (name + ".cpp"), tmp_path / name
    src.write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout


FIT = r'''
#include <stdio.h>
#include "attn_plan.h"
using namespace sieve;
#define NEED(x) \
  do { if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)
static std::vector<int64_t> each(int64_t n, int64_t length) {
  std::vector<int64_t> o(n + 1);
  for (int64_t i = 0; i <= n; ++i) o[i] = i * length;
  return o;
}
// a launch of `items` work-groups of 256 threads has fewer than 2^32 threads
static bool launches(int64_t items) { return items * 256 < (int64_t(1) << 32); }
static bool fits(const std::vector<int64_t>& qo, const std::vector<int64_t>& ko, int kvh, int G) {
  const int64_t n = (int64_t)qo.size() - 1;
  return lists_fit(count_items(qo.data(), ko.data(), n, kvh, G), (int64_t)kvh * G);
}
int main() {
  AttnLists p;
  // one query over 1.5 million documents, 12 key heads: 18 million work-groups
  const auto one = each(1500000, 1), ten = each(1500000, 10);
  NEED(!make_lists(one.data(), ten.data(), 1500000, 12, 1, false, &p));
  NEED(p.fwd.empty() && p.dkv.empty());
  // the forward list alone, and that of dK and dV with the work-groups for the bias's gradient
  const auto none = each(1, 0);
  for (int64_t n : {(int64_t(1) << 24) - 2, (int64_t(1) << 24) - 1, int64_t(1) << 24}) {
    const std::vector<int64_t> rows{0, n * 128}, keys{0, n * 128};
    NEED(fits(rows, none, 1, 1) == launches(n));
    NEED(fits(none, keys, 1, 1) == launches(n + 1));
    NEED(fits(none, keys, 1, 4) == launches(n + 4));
    const std::vector<int64_t> odd{0, n * 128 - 127};  // the last tile has one row
    NEED(fits(odd, none, 1, 1) == launches(n));
  }
  // tiles are counted as they are cut: 32 rows where no sequence has more, else 128
  const auto short_ = each(700000, 32), longer = each(700000, 40);
  AttnCounts c = count_items(short_.data(), short_.data(), 700000, 2, 1);
  NEED(c.fwd == 1400000 && c.dq == 1400000 && c.dkv == 1400000);
  c = count_items(longer.data(), longer.data(), 700000, 2, 4);
  NEED(!c.few && c.fwd == 2800000 && c.dq == 2800000 && c.dkv == 1400000);
  // and the lists have these sizes where nothing is shared out
  const auto q = each(3000, 150);
  NEED(make_lists(q.data(), q.data(), 3000, 2, 2, true, &p));
  c = count_items(q.data(), q.data(), 3000, 2, 2);
  NEED((int64_t)p.fwd.size() == c.fwd && (int64_t)p.dq.size() == c.dq);
  NEED((int64_t)p.dkv.size() == c.dkv);
  printf("ok\n");
}
'''


def test_lists_that_no_launch_takes_are_refused(tmp_path):
    """Before any part of them runs: a plan's lists are launched one work-group an item."""
    _run(tmp_path, "fit", FIT)


DEVICES = r'''
#include <stdio.h>
#include "once_per_device.h"
using namespace sieve;
#define NEED(x) \
  do { if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)
int main() {
  std::atomic<uint64_t> done{0};
  int calls = 0, answer = 0;
  auto ask = [&] { ++calls; return answer; };
  NEED(once_per_device(done, 0, ask) == 0 && calls == 1);
  NEED(once_per_device(done, 0, ask) == 0 && calls == 1);  // known
  NEED(once_per_device(done, 1, ask) == 0 && calls == 2);  // another device
  NEED(once_per_device(done, 63, ask) == 0 && calls == 3);
  answer = 5;
  NEED(once_per_device(done, 2, ask) == 5 && calls == 4);  // a failure is not remembered
  answer = 0;
  NEED(once_per_device(done, 2, ask) == 0 && calls == 5);
  NEED(once_per_device(done, 2, ask) == 0 && calls == 5);
  NEED(once_per_device(done, 64, ask) == 0 && once_per_device(done, 64, ask) == 0 && calls == 7);
  printf("ok\n");
}
'''


def test_large_lds_is_asked_for_on_every_device(tmp_path):
    """A process may have plans on several devices; what one was asked for does not hold for
    another."""
    _run(tmp_path, "devices", DEVICES)


FEW = r'''
#include <stdio.h>
#include "attn_plan.h"
using namespace sieve;
#define NEED(x) \
  do { if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)
static bool few(int64_t rows, int64_t keys, int G) {
  const std::vector<int64_t> qo{0, rows, 2 * rows}, ko{0, 1, 1 + keys};
  AttnLists p;
  if (!make_lists(qo.data(), ko.data(), 2, 2, G, false, &p)) return false;
  return p.few;
}
int main() {
  NEED(!few(32, 32, 1) && !few(1, 64, 1) && !few(1, 64, 8));  // short texts, short contexts
  NEED(few(1, 65, 1) && few(32, 65, 1) && few(4, 20000, 8));
  NEED(!few(33, 20000, 1) && !few(5, 20000, 8));              // rows: queries times their group
  printf("ok\n");
}
'''


def test_waves_share_keys_only_where_there_are_some(tmp_path):
    """Tiles of few rows share the keys among four waves: a batch of short texts has none to
    share, whatever its rows."""
    _run(tmp_path, "few", FEW)
