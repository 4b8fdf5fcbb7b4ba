// The optimizer step's planner (csrc/optim_api.cu) without a GPU: over random
// lists of tensors, sizes and addresses, every launch's tables are walked as the
// kernels walk them, and every element must come up exactly once, at its
// address, with what moves as vectors on its boundary; refusals launch nothing.
#include <cassert>
#include <cstdio>
#include <map>
#include <random>
#include <set>

#include "fake_cuda.h"

#include "api.cu"
#include "optim_api.cu"

namespace {
std::vector<std::pair<StepClass, StepParams>> steps;
std::vector<ClipParams> clips;
std::vector<ConvertParams> converts;
}  // namespace

namespace frk {
cudaError_t launch_step(const StepClass& c, const StepParams& p, cudaStream_t) { steps.emplace_back(c, p); return cudaSuccess; }
cudaError_t launch_clip(const ClipParams& p, cudaStream_t) { clips.push_back(p); return cudaSuccess; }
cudaError_t launch_convert(const ConvertParams& p, cudaStream_t) { converts.push_back(p); return cudaSuccess; }
}  // namespace frk

namespace {

#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

// The tensor of block b, from t on, as tensor_of finds it.
uint32_t find(const OptWork& w, uint32_t t, uint32_t b) {
  CHECK(t < w.n_tensors && w.tensors[t].first <= b);
  while (b - w.tensors[t].first >= w.tensors[t].n_blocks) CHECK(++t < w.n_tensors);
  return t;
}

// The tensor that a warp starts its blocks from b on with, as first_tensor finds it.
uint32_t first(const OptWork& w, uint32_t group, uint32_t warp, int warps, uint32_t b) {
  if (!w.start_of_warps) return find(w, w.start[group], b);
  const uint32_t t = w.start[group * warps + warp];
  CHECK(find(w, t, b) == t);
  return t;
}

using Seen = std::map<uint32_t, std::vector<uint8_t>>;  // per tensor of the plan, how often each element came up

void see(Seen& seen, const std::vector<fr_opt_tensor>& list, const OptDesc& d, uint32_t block, bool vectors) {
  const fr_opt_tensor& x = list[d.tensor];
  const uint64_t first = static_cast<uint64_t>(block) * kOptBlock, stop = std::min(first + kOptBlock, d.n);
  CHECK(first < d.n && d.skipped + stop <= x.n);
  auto here = [&](const void* mine, const void* theirs, uint32_t dtype) {
    CHECK(mine == static_cast<const uint8_t*>(theirs) + (theirs ? d.skipped * type_bytes(dtype) : 0));
    if (vectors && theirs) CHECK(reinterpret_cast<uintptr_t>(mine) % (8 * type_bytes(dtype)) == 0);
  };
  here(d.weight, x.weight, x.weight_dtype);
  here(d.grad, x.grad, x.grad_dtype);
  here(d.master, x.master, FR_DT_F32);
  here(d.m, x.m, x.state_dtype);
  here(d.v, x.v, x.state_dtype);
  CHECK(d.m_exp == x.m_exp && d.v_exp == x.v_exp && (d.skipped == 0 || x.state_dtype == FR_DT_F32));
  auto& s = seen[d.tensor];
  s.resize(x.n);
  for (uint64_t i = first; i < stop; ++i) CHECK(++s[d.skipped + i] == 1);
}

void all_seen(const Seen& seen, const std::vector<fr_opt_tensor>& list, const std::set<uint32_t>& which) {
  for (uint32_t t : which) {
    if (list[t].n == 0) continue;
    auto it = seen.find(t);
    CHECK(it != seen.end() && it->second.size() == list[t].n);
    for (uint8_t c : it->second) CHECK(c == 1);
  }
}

void walk_step(Seen& seen, const std::vector<fr_opt_tensor>& list, const StepClass& c, const StepParams& p) {
  const uint32_t per_warp = c.eight ? p.work.per_warp : 1;
  CHECK(c.eight || p.work.per_warp == 1);
  for (uint32_t cta = 0; cta < p.work.n_groups; ++cta)
    for (uint32_t warp = 0; warp < kOptWarps; ++warp) {
      uint32_t b = (cta * kOptWarps + warp) * per_warp;
      const uint32_t end = std::min(b + per_warp, p.work.n_blocks);
      if (b >= end) continue;
      for (uint32_t t = first(p.work, cta, warp, kOptWarps, b); b < end; ++b) {
        t = find(p.work, t, b);
        const OptDesc& d = p.work.tensors[t];
        const bool vectors = d.aligned && b - d.first < d.n / kOptBlock;
        if (vectors && c.weight == kWeightBf16) CHECK(d.skipped % 2 == 0);
        see(seen, list, d, b - d.first, vectors);
      }
    }
  CHECK(static_cast<uint64_t>(p.work.n_groups) * kOptWarps * per_warp >= p.work.n_blocks);
}

void walk_clip(Seen& seen, const std::vector<fr_opt_tensor>& list, const ClipParams& p) {
  const uint32_t n_ctas = std::max(1u, std::min(p.work.n_groups, kClipCtas)), per_warp = p.work.per_warp;
  CHECK(per_warp >= 1 && per_warp <= kClipMost);
  CHECK(*p.done == 0);
  for (uint32_t cta = 0; cta < n_ctas; ++cta) {
    p.partials[cta] = {};  // (there is one for each)
    for (uint32_t k = cta; k < p.work.n_groups; k += n_ctas)
      for (uint32_t warp = 0; warp < kClipWarps; ++warp) {
        uint32_t b = (k * kClipWarps + warp) * per_warp;
        const uint32_t end = std::min(b + per_warp, p.work.n_blocks);
        if (b >= end) continue;
        for (uint32_t t = first(p.work, k, warp, kClipWarps, b);; ++t) {  // on to the next tensor, without a search
          const OptDesc& d = p.work.tensors[t];
          CHECK(t < p.work.n_tensors && b >= d.first && b - d.first < d.n_blocks);
          for (; b < std::min(end, d.first + d.n_blocks); ++b) see(seen, list, d, b - d.first, false);
          if (b >= end) break;
        }
      }
  }
}

void walk_convert(Seen& seen, const std::vector<fr_opt_tensor>& list, const ConvertParams& p, bool src) {
  for (uint32_t cta = 0; cta < p.src.n_groups; ++cta)
    for (uint32_t warp = 0; warp < kOptWarps; ++warp) {
      uint32_t b = (cta * kOptWarps + warp) * kConvertBlocks;
      const uint32_t end = std::min(b + kConvertBlocks, p.src.n_blocks);
      if (b >= end) continue;
      for (uint32_t t = first(p.src, cta, warp, kOptWarps, b); b < end; ++b) {
        t = find(p.src, t, b);
        const OptDesc &s = p.src.tensors[t], &d = p.dst.tensors[t];
        CHECK(s.first == d.first && s.n == d.n && s.tensor == d.tensor);
        see(seen, list, src ? s : d, b - s.first, false);
        const OptDesc& mine = src ? s : d;
        if (mine.aligned) {
          const uint64_t v = 8 * type_bytes(list[mine.tensor].state_dtype);
          CHECK(reinterpret_cast<uintptr_t>(mine.m) % v == 0 && reinterpret_cast<uintptr_t>(mine.v) % v == 0);
        }
      }
    }
}

fr_opt make(const std::vector<fr_opt_tensor>& list) {
  fr_opt p = nullptr;
  CHECK(fr_opt_create(list.data(), list.size(), &p) == FR_OK);
  return p;
}

}  // namespace

int main() {
  std::mt19937_64 rng(5);
  auto below = [&](uint64_t n) { return rng() % n; };
  for (int round = 0; round < 300; ++round) {
    std::vector<fr_opt_tensor> list, other;
    std::set<uint32_t> whole;
    const uint64_t n_tensors = below(4) == 0 ? below(400) : below(12), most = below(3) == 0 ? 9 : below(2) ? 3000 : 200000;
    uint64_t at = 1 << 20;
    auto place = [&](uint64_t bytes, uint64_t element, uint64_t off) {  // an address, `off` elements from a boundary
      void* p = reinterpret_cast<void*>(at + off * element);
      at += (bytes + 1024) / 512 * 512 + 512;
      return p;
    };
    for (uint64_t t = 0; t < n_tensors; ++t) {
      fr_opt_tensor x = {}, y = {};
      x.n = below(10) == 0 ? 0 : below(most) + 1;
      x.weight_dtype = below(2) ? FR_DT_BF16 : FR_DT_F32;
      x.grad_dtype = below(2) ? FR_DT_BF16 : FR_DT_F32;
      x.state_dtype = below(2) ? FR_DT_BYTES : FR_DT_F32;
      x.lr_scale = x.decay_scale = 1.0f;
      const uint64_t common = below(10);
      auto off = [&] { return below(6) ? common : below(10); };
      x.weight = place(4 * x.n, type_bytes(x.weight_dtype), off());
      x.grad = place(4 * x.n, type_bytes(x.grad_dtype), off());
      if (x.weight_dtype == FR_DT_BF16 && below(2)) x.master = static_cast<float*>(place(4 * x.n, 4, off()));
      x.m = place(4 * x.n, type_bytes(x.state_dtype), off());
      x.v = place(4 * x.n, type_bytes(x.state_dtype), off());
      if (x.state_dtype == FR_DT_BYTES) {
        x.m_exp = static_cast<uint8_t*>(place(x.n / 256 + 1, 1, off()));
        x.v_exp = static_cast<uint8_t*>(place(x.n / 256 + 1, 1, off()));
      }
      list.push_back(x);
      whole.insert(static_cast<uint32_t>(t));
    }
    fr_opt p = make(list);
    uint64_t nt, ne, nb, want = 0;
    CHECK(fr_opt_info(p, &nt, &ne, &nb) == FR_OK);
    for (const fr_opt_tensor& x : list) want += x.n;
    CHECK(nt == n_tensors && ne == want);
    fr_adamw h = {1e-3, 0.9, 0.95, 1e-8, 0.1, 3, 7, FR_ROUND_RANDOM, 0};
    steps.clear();
    CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_OK);
    fake::finish_all();
    Seen seen;
    std::set<int> classes;
    for (auto& s : steps) {
      CHECK(classes.insert(s.first.index()).second && s.second.work.n_blocks > 0 && !s.second.exact && s.second.random);
      walk_step(seen, list, s.first, s.second);
    }
    all_seen(seen, list, whole);
    clips.clear();
    fr_clip record;
    CHECK(fr_grad_clip(p, 1.0f, 1.0f, &record, nullptr) == FR_OK && clips.size() == 1);
    seen.clear();
    walk_clip(seen, list, clips[0]);
    all_seen(seen, list, whole);
    fr_opt_destroy(p);
    // moments alone, 32 bits to 8 and back
    std::vector<fr_opt_tensor> a, b;
    for (const fr_opt_tensor& x : list) {
      fr_opt_tensor f = {}, e = {};
      f.n = e.n = x.n;
      f.state_dtype = FR_DT_F32;
      e.state_dtype = FR_DT_BYTES;
      f.m = place(4 * x.n, 4, below(10));
      f.v = place(4 * x.n, 4, below(2) * 8);
      e.m = place(x.n, 1, below(2) * 8);
      e.v = place(x.n, 1, below(10));
      e.m_exp = static_cast<uint8_t*>(place(x.n / 256 + 1, 1, 1));
      e.v_exp = static_cast<uint8_t*>(place(x.n / 256 + 1, 1, 3));
      a.push_back(f);
      b.push_back(e);
    }
    fr_opt pa = make(a), pb = make(b);
    converts.clear();
    CHECK(fr_opt_convert(pa, pb, FR_ROUND_NEAREST, 1, nullptr) == FR_OK && fr_opt_convert(pb, pa, FR_ROUND_NEAREST, 1, nullptr) == FR_OK);
    CHECK(converts.size() == (want ? 2u : 0u));
    fake::finish_all();
    for (size_t k = 0; k < converts.size(); ++k)
      for (int src = 0; src < 2; ++src) {
        seen.clear();
        walk_convert(seen, (k == 0) == (src == 1) ? a : b, converts[k], src == 1);
        all_seen(seen, a, whole);
      }
    CHECK(fr_adamw_step(pa, &h, nullptr, nullptr) == (want ? FR_ERR_INVALID_ARG : FR_OK));
    CHECK(fr_grad_clip(pa, 1.0f, 1.0f, &record, nullptr) == (want ? FR_ERR_INVALID_ARG : FR_OK));
    fr_opt_destroy(pa);
    fr_opt_destroy(pb);
  }

  // a list whose tables go by CTA: 2^18 blocks of one tensor and more, small ones around it
  for (uint32_t dtype : {FR_DT_F32, FR_DT_BYTES}) {
    std::vector<fr_opt_tensor> list;
    std::set<uint32_t> whole;
    uint64_t at = 1ull << 30;
    for (uint64_t n : {5ull, 300ull, (1ull << 27) + 77, 9ull, 70000ull, 1ull}) {
      fr_opt_tensor x = {};
      x.n = n;
      x.weight_dtype = x.grad_dtype = FR_DT_BF16;
      x.state_dtype = dtype;
      x.lr_scale = x.decay_scale = 1.0f;
      auto place = [&](uint64_t bytes) { void* q = reinterpret_cast<void*>(at); at += (bytes + 1023) / 512 * 512; return q; };
      x.weight = place(2 * n), x.grad = place(2 * n), x.m = place(4 * n), x.v = place(4 * n);
      if (dtype == FR_DT_BYTES) x.m_exp = static_cast<uint8_t*>(place(n / 256 + 1)), x.v_exp = static_cast<uint8_t*>(place(n / 256 + 1));
      whole.insert(static_cast<uint32_t>(list.size()));
      list.push_back(x);
    }
    fr_opt p = make(list);
    fr_adamw h = {1e-3, 0.9, 0.95, 1e-8, 0.1, 3, 7, FR_ROUND_RANDOM, 0};
    fr_clip record;
    steps.clear(), clips.clear();
    CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_OK && steps.size() == 1 && fr_grad_clip(p, 1.0f, 1.0f, &record, nullptr) == FR_OK);
    CHECK(steps[0].second.work.start_of_warps == (dtype == FR_DT_BYTES) && clips[0].work.start_of_warps);
    Seen seen;
    walk_step(seen, list, steps[0].first, steps[0].second);
    all_seen(seen, list, whole);
    seen.clear();
    walk_clip(seen, list, clips[0]);
    all_seen(seen, list, whole);
    fr_opt_destroy(p);
  }

  // sizes near the limits: what follows from them stays in 32 bits
  for (uint64_t n : {1ull, 4863ull, 4864ull, 4865ull, 77824ull, 77825ull, 3921936ull, 1ull << 31, (1ull << 32) - 2}) {
    CHECK(clip_blocks(n) >= 1 && clip_blocks(n) <= kClipMost);
    CHECK(step_blocks(false, n) == 1 && step_blocks(true, n) >= 1 && step_blocks(true, n) <= 8);
  }

  // refusals launch nothing
  steps.clear(), clips.clear(), converts.clear();
  fr_opt_tensor x = {};
  x.n = 1000;
  x.weight = x.m = reinterpret_cast<void*>(1 << 20);
  x.v = reinterpret_cast<void*>(1 << 21);
  x.grad = reinterpret_cast<void*>(1 << 22);
  x.weight_dtype = x.grad_dtype = x.state_dtype = FR_DT_F32;
  x.lr_scale = x.decay_scale = 1.0f;
  fr_opt p = make({x});
  fr_adamw good = {1e-3, 0.9, 0.95, 1e-8, 0.1, 1, 0, 0, 0}, h = good;
  h.eps = 1e-20;
  CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_OK && steps.back().second.exact == 1);
  steps.clear();
  h = good, h.beta2 = 1.0;
  CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  for (double bad : {1e300, -1.0, HUGE_VAL, static_cast<double>(NAN)}) {
    h = good, h.lr = bad;
    CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG);
    h = good, h.weight_decay = bad;
    CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG);
    h = good, h.eps = bad;
    CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  }
  h = good, h.step = 0;
  CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_adamw_step(p, &good, reinterpret_cast<fr_clip*>(4), nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_adamw_step(nullptr, &good, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_grad_clip(p, 0.0f, 1.0f, reinterpret_cast<fr_clip*>(8), nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_grad_clip(p, 1.0f, 1.0f, reinterpret_cast<fr_clip*>(4), nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_opt_convert(p, p, 0, 0, nullptr) == FR_ERR_INVALID_ARG);
  fr_opt q = nullptr;
  fr_opt_tensor big = x;
  big.n = 1ull << 46;
  CHECK(fr_opt_create(&big, 1, &q) == FR_ERR_INVALID_ARG && q == nullptr);
  big = x, big.m = static_cast<uint8_t*>(x.m) + 2;
  CHECK(fr_opt_create(&big, 1, &q) == FR_ERR_ALIGNMENT && q == nullptr);
  CHECK(steps.empty() && clips.empty() && converts.empty());
  fr_opt_destroy(p);
  fr_opt_destroy(nullptr);
  std::printf("opt_plan ok\n");
  return 0;
}
