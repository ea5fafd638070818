"""CPU-side checks of the text-encoder operators: C layouts, argument errors before any HIP call,
the relative position buckets, the cut of a batch into work items, and the oracle's gradients
against differences."""
import ctypes
import os
import subprocess

import pytest
import torch

from encoder_reference import attention, bucket, norm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_03199_amd", "csrc")


@pytest.fixture(scope="module")
def enc():
    import paper_2608_03199_amd as ps
    if not os.path.exists(ps.LIB_PATH):
        from paper_2608_03199_amd import build
        build.build()
    from paper_2608_03199_amd import encoder
    return encoder


def _compile(tmp_path, name, text, cc="g++"):
    src, exe = tmp_path / (name + (".c" if cc == "gcc" else ".cpp")), tmp_path / name
    src.write_text(text)
    flags = ["-std=c++17", "-O2"] if cc == "g++" else []
    subprocess.run([cc, *flags, "-Wall", "-Werror", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), str(src), "-o", str(exe), "-lm"], check=True)
    return str(exe)


@pytest.mark.parametrize("name, c_name", [("_Desc", "sieve_attn_desc"), ("_Heads", "sieve_heads")])
def test_struct_layouts_match_c(enc, tmp_path, name, c_name):
    mirror = getattr(enc, name)
    fields = [f for f, _ in mirror._fields_]
    exe = _compile(tmp_path, name, '#include <stdio.h>\n#include <stddef.h>\n#include "sieve.h"\n'
                   'int main(void){printf("%zu", sizeof(' + c_name + '));' +
                   "".join(f'printf(" %zu", offsetof({c_name}, {f}));' for f in fields) +
                   "return 0;}\n", "gcc")
    vals = [int(x) for x in subprocess.run([exe], capture_output=True, text=True,
                                           check=True).stdout.split()]
    assert vals == [ctypes.sizeof(mirror)] + [getattr(mirror, f).offset for f in fields]


def test_norm_argument_errors_without_a_gpu(enc):
    lib = enc._library()
    p = ctypes.c_void_p(0x1000)
    none = None

    def forward(x=p, xs=8, r=none, rs=0, w=p, b=none, dt=1, wdt=1, rows=4, n=8, eps=1e-5,
                y=ctypes.c_void_p(0x2000), h=none, mean=none, rstd=none):
        return lib.sieve_norm_forward(x, xs, r, rs, w, b, dt, wdt, rows, n, eps, y, h, mean, rstd,
                                      none)

    assert forward(dt=3) == -1 and b"dtype" in lib.sieve_last_error()
    assert forward(dt=1, wdt=2) == -1 and b"wdtype" in lib.sieve_last_error()
    assert forward(rows=-1) == -1
    assert forward(n=0) == -1
    assert forward(n=65537, xs=65537) == -4
    assert forward(eps=float("nan")) == -1 and forward(eps=-1.0) == -1
    assert forward(x=none) == -1 and forward(w=none) == -1 and forward(y=none) == -1
    assert forward(r=p, rs=8) == -1 and b"residual" in lib.sieve_last_error()
    assert forward(r=p, rs=8, h=ctypes.c_void_p(0x2000)) == -1  # y and h
    assert forward(xs=7) == -1 and b"stride" in lib.sieve_last_error()
    assert forward(mean=p) == -1
    assert forward(rows=0, x=none, y=none) == 0
    assert lib.sieve_norm_workspace(4, 0) == -1
    assert lib.sieve_norm_workspace(1 << 40, 768) > 0

    def backward(dy=p, dys=8, h=p, hs=8, w=p, mean=p, rstd=p, rows=100, dx=p, ws=none, size=0):
        return lib.sieve_norm_backward(dy, dys, h, hs, w, mean, rstd, none, 1, 0, rows, 8, dx, p,
                                       p, ws, size, none)

    assert backward(w=none) == -1 and backward(mean=none) == -1 and backward(dx=none) == -1
    assert backward(dys=7) == -1
    assert backward() == -1 and b"workspace" in lib.sieve_last_error()
    assert backward(ws=ctypes.c_void_p(0x1008), size=1 << 30) == -1  # not aligned


def _create(enc, q_offsets, k_offsets=None, **over):
    args = dict(dtype=1, heads=4, kv_heads=2, head_dim=64, causal=0, num_buckets=0,
                max_distance=0, scale=0.125)
    args.update(over)
    qo = torch.tensor(q_offsets, dtype=torch.int64)
    ko = None if k_offsets is None else torch.tensor(k_offsets, dtype=torch.int64)
    d = enc._Desc(args["dtype"], args["heads"], args["kv_heads"], args["head_dim"],
                  args["causal"], args["num_buckets"], args["max_distance"], args["scale"],
                  args.get("nseq", len(q_offsets) - 1), qo.data_ptr(),
                  None if ko is None else ko.data_ptr())
    out = ctypes.c_void_p()
    rc = enc._library().sieve_attn_create(ctypes.byref(d), None, ctypes.byref(out))
    assert not out.value or rc == 0
    return rc


@pytest.mark.parametrize("over, code", [
    (dict(dtype=3), -1), (dict(kv_heads=3), -1), (dict(heads=0), -1), (dict(head_dim=0), -1),
    (dict(head_dim=129), -4), (dict(causal=2), -1), (dict(scale=0.0), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(num_buckets=2), -1),
    (dict(num_buckets=7), -1), (dict(num_buckets=258), -1),
    (dict(num_buckets=32, max_distance=8), -1), (dict(num_buckets=32, max_distance=800), -4),
    (dict(causal=1, num_buckets=32, max_distance=16), -1), (dict(nseq=-1), -1),
    (dict(heads=65536, kv_heads=1), -4)])
def test_attention_description_errors_without_a_gpu(enc, over, code):
    assert _create(enc, [0, 5], **over) == code
    assert enc._library().sieve_last_error()


@pytest.mark.parametrize("offsets, code", [
    ([1, 5], -1), ([0, 5, 4], -1), ([0, 1 << 31], -4), ([0, (1 << 30) - 1], -4),
    ([0] + [i << 29 for i in range(1, 2050)], -4)])
def test_attention_offset_errors_without_a_gpu(enc, offsets, code):
    assert _create(enc, offsets) == code
    assert enc._library().sieve_last_error()


def test_attention_call_errors_without_a_gpu(enc):
    lib = enc._library()
    assert lib.sieve_attn_workspace(None, 0) == -1
    assert lib.sieve_attn_forward(None, None, None, None, None, None, None, None, None, 0, None) == -1
    assert lib.sieve_attn_backward(None, None, None, None, None, None, None, None, None, None,
                                   None, None, None, None, 0, None) == -1
    assert b"plan" in lib.sieve_last_error()
    lib.sieve_attn_free(None)


SETS = [(32, 128), (16, 40), (8, 20), (4, 2), (32, 1024), (64, 1475), (256, 777), (12, 77)]


@pytest.mark.parametrize("buckets, distance", SETS)
@pytest.mark.parametrize("causal", [False, True])
def test_buckets_are_exact(tmp_path, buckets, distance, causal):
    if distance <= (buckets if causal else buckets // 2) // 2:
        pytest.skip("no such table")
    exe = _compile(tmp_path, "buckets", '#include <stdio.h>\n#include "attn_plan.h"\n'
                   'int main(){for(int r=-%d;r<=%d;++r)printf("%%d ",sieve::bucket_of(r,%d,%d,%s));}'
                   % (2 * distance, 2 * distance, buckets, distance, "true" if causal else "false"))
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True,
                                          check=True).stdout.split()]
    want = [bucket(r, buckets, distance, causal) for r in range(-2 * distance, 2 * distance + 1)]
    assert got == want


LISTS = r'''
#include <stdio.h>
#include <map>
#include <set>
#include <tuple>
#include "attn_plan.h"
using namespace sieve;
#define NEED(x) do { if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)
static int run(const std::vector<int64_t>& qo, const std::vector<int64_t>& ko, int kvh, int G,
               bool causal) {
  AttnLists p;
  const int64_t n = (int64_t)qo.size() - 1;
  const bool fits = (ko[n] / kAttnKeys + n) * kvh <= kMaxItems;
  NEED(make_lists(qo.data(), ko.data(), n, kvh, G, causal, &p) == fits);
  if (!fits) return 0;
  // forward and dq: each row tile once, its keys covered once from 0 to the last seen one
  for (int which = 0; which < 2; ++which) {
    std::map<std::tuple<int64_t, int, int>, std::vector<std::pair<int, int>>> tiles;
    std::set<int> parts;
    for (const AttnItem& x : which ? p.dq : p.fwd) {
      NEED(x.lo >= 0 && x.lo <= x.hi && x.hi <= x.nk && x.row >= 0 && (int64_t)x.row < (int64_t)x.nq * G);
      NEED(x.row % (which || !p.few ? kAttnRows : kAttnFewRows) == 0);
      tiles[{x.q0, x.kvh, x.row}].push_back({x.lo, x.hi});
      if (which) NEED(x.part >= 0 && x.part < p.row_tiles && x.part == x.tile0 + x.row / kAttnRows);
      if (x.part >= 0 && !which) NEED(x.part < p.parts && parts.insert(x.part).second);
    }
    size_t want = 0;
    const int tile = which || !p.few ? kAttnRows : kAttnFewRows;
    for (int64_t s = 0; s < n; ++s) {
      const int64_t rows = (qo[s + 1] - qo[s]) * G, nk = ko[s + 1] - ko[s], nq = qo[s + 1] - qo[s];
      for (int64_t r = 0; r < rows; r += tile)
        for (int h = 0; h < kvh; ++h) {
          ++want;
          auto& v = tiles[{qo[s], h, (int)r}];
          std::sort(v.begin(), v.end());
          NEED(!v.empty() && v[0].first == 0);
          for (size_t i = 1; i < v.size(); ++i) NEED(v[i].first == v[i - 1].second);
          int64_t last = std::min(r + tile, rows) - 1, end = nk;
          if (causal) end = std::max<int64_t>(0, std::min(nk, last / G + nk - nq + 1));
          NEED(v.back().second == end);
        }
    }
    NEED(want == tiles.size());
  }
  size_t fwd_parts = 0;
  for (const AttnJoin& j : p.joins) fwd_parts += j.parts;
  NEED((int)fwd_parts == p.parts);
  // dk and dv: each key tile once, its rows covered once from the first that sees it
  std::map<std::tuple<int64_t, int, int>, std::vector<std::pair<int, int>>> tiles;
  std::set<int> parts;
  for (const AttnItem& x : p.dkv) {
    NEED(x.lo >= 0 && x.lo <= x.hi && (int64_t)x.hi <= (int64_t)x.nq * G && x.row % kAttnKeys == 0);
    NEED(x.lo % G == 0 || x.part >= 0);
    if (x.part >= 0) NEED(x.part < p.kv_parts && parts.insert(x.part).second);
    tiles[{x.k0, x.kvh, x.row}].push_back({x.lo, x.hi});
  }
  size_t want = 0;
  for (int64_t s = 0; s < n; ++s) {
    const int64_t nk = ko[s + 1] - ko[s], nq = qo[s + 1] - qo[s], rows = nq * G;
    for (int64_t k = 0; k < nk; k += kAttnKeys)
      for (int h = 0; h < kvh; ++h) {
        ++want;
        auto& v = tiles[{ko[s], h, (int)k}];
        std::sort(v.begin(), v.end());
        const int64_t from = causal ? std::max<int64_t>(0, std::min(rows, (k - (nk - nq)) * G)) : 0;
        NEED(!v.empty() && v[0].first == from && v.back().second == rows);
        for (size_t i = 1; i < v.size(); ++i) NEED(v[i].first == v[i - 1].second);
      }
  }
  NEED(want == tiles.size() && (int)parts.size() == p.kv_parts);
  return 0;
}
static std::vector<int64_t> offsets(std::vector<int64_t> lens, int64_t start = 0) {
  std::vector<int64_t> o{0};
  for (int64_t l : lens) o.push_back(o.back() + l);
  (void)start;
  return o;
}
int main() {
  const std::vector<std::vector<int64_t>> lens = {
      {}, {0}, {1}, {5, 0, 7}, {128}, {129, 127, 64, 1}, {3000, 17, 900}, {12007}, {33, 32, 31},
      {2000000000, 5, 1900000000, 2000000000}};
  for (const auto& l : lens)
    for (int kvh : {1, 3})
      for (int G : {1, 3, 4, 16})
        for (bool causal : {false, true}) {
          if (l.size() == 4 && l[0] > 1000000000 && (G > 1 || kvh > 1)) continue;
          const auto o = offsets(l);
          if (l.empty() || l[0] < 1000000000)
            if (run(o, o, kvh, G, causal)) { printf("self %zu\n", l.size()); return 1; }
          std::vector<int64_t> few, many;
          for (int64_t x : l) { few.push_back(x > 2 ? 2 : x); many.push_back(x / 2); }
          if (run(offsets(few), o, kvh, G, causal)) { printf("few\n"); return 1; }
          if (l.empty() || l[0] < 1000000000)
            if (run(o, offsets(many), kvh, G, causal)) { printf("many\n"); return 1; }
        }
  std::vector<int64_t> ones(2000, 1);
  if (run(offsets(ones), offsets(ones), 12, 1, false)) return 1;
  AttnLists p;
  const auto big = offsets(std::vector<int64_t>(40, 2000000000));
  NEED(!make_lists(big.data(), big.data(), 40, 8, 1, false, &p));
  printf("ok\n");
}
'''


def test_work_items_cover_every_pair_once(tmp_path):
    exe = _compile(tmp_path, "lists", LISTS)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip().endswith("ok"), out.stdout


def test_oracle_gradients_against_differences():
    """The formulas of the oracle: directional derivatives of its own forward pass."""
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, dy = rnd(5, 9), rnd(9), rnd(9), rnd(5, 9)
    args = {"x": x, "w": w, "b": b}
    UNIT64 = __import__("encoder_reference")
    UNIT64.UNIT[torch.float64] = UNIT64.TINY[torch.float64] = 0.0
    try:
        val, _ = norm(x, w, b, 1e-5, None, dy)
        for name, grad in (("x", "dx"), ("w", "dweight"), ("b", "dbias")):
            v, e = rnd(*args[name].shape), 1e-5
            f = [float((norm(*[args[n] + (s * e * v if n == name else 0) for n in "xwb"], 1e-5)[0]["y"]
                        * dy).sum()) for s in (1, -1)]
            assert abs((f[0] - f[1]) / (2 * e) - float((val[grad] * v).sum())) < 1e-7
        qo, ko = [0, 7, 7, 11], [0, 5, 8, 13]
        mask = torch.rand(13, generator=g) > 0.2
        args = {"q": rnd(11, 4, 6), "k": rnd(13, 2, 6), "v": rnd(13, 2, 6), "bias": rnd(8, 4)}
        dout = rnd(11, 4, 6)

        def call(a, dout=None):
            return attention(a["q"], a["k"], a["v"], qo, ko, True, None, mask, a["bias"], 9, dout)[0]

        val = call(args, dout)
        for name in args:
            v, e = rnd(*args[name].shape), 1e-5
            f = [float((call({**args, name: args[name] + s * e * v})["out"] * dout).sum())
                 for s in (1, -1)]
            assert abs((f[0] - f[1]) / (2 * e) - float((val["d" + name] * v).sum())) < 1e-7
    finally:
        del UNIT64.UNIT[torch.float64], UNIT64.TINY[torch.float64]
