// Randomised checks of the optimizer's host code (fr_adamw_state_table,
// fr_adamw_query), built with AddressSanitizer and
// UndefinedBehaviorSanitizer by tests/test_adamw_cpu.py (g++, CPU only; no
// device code is built or run):
//   1. states laid out for random sizes and widths are accepted, with the
//      sums that the sizes give;
//   2. random and adversarial descriptors get the answer of a plain
//      restatement of the header's rules.
#include <cstdio>
#include <random>
#include <vector>

#include "flashrestore.h"

static std::mt19937_64 rng(977);
static uint64_t U(uint64_t n) { return n ? rng() % n : 0; }

static uint64_t bytes(const fr_tensor_desc& d) { return d.numel * (d.dtype == FR_F32 ? 4 : 2); }

// The rules, one after the other; -100: more than one is broken (any of their codes will do).
static int expect(const std::vector<fr_tensor_desc>& t, const std::vector<fr_adamw_tensor>& a, uint32_t groups,
                  uint64_t grad_bytes) {
  bool inval = false, align = false, range = false, over = false;
  std::vector<int> named;
  for (const fr_adamw_tensor& d : a) {
    if (d.reserved || d.flags > 1 || d.group >= groups || (d.grad_dtype != FR_F32 && d.grad_dtype != FR_BF16)) inval = true;
    if (d.grad_offset % 16) align = true;
    if ((d.m_scale < 0) != (d.v_scale < 0)) inval = true;
    if (d.master < 0 || d.master >= int(t.size())) {
      inval = true;
      continue;
    }
    const uint64_t n = t[d.master].numel, mom = d.m_scale >= 0 ? (n + 3) / 4 : n, bl = (n + 255) / 256;
    const int e[6] = {d.param, d.master, d.m, d.v, d.m_scale, d.v_scale};
    const uint64_t want[6] = {n, n, mom, mom, bl, bl};
    for (int j = 0; j < 6; j++) {
      if (e[j] == -1 && (j == 0 || (j >= 4 && d.m_scale < 0))) continue;
      if (e[j] < 0 || e[j] >= int(t.size()) || t[e[j]].dtype != (j ? FR_F32 : FR_BF16) || t[e[j]].numel != want[j]) {
        inval = true;
        continue;
      }
      named.push_back(e[j]);
    }
    const uint64_t gb = n * (d.grad_dtype == FR_F32 ? 4 : 2);
    if (d.grad_offset > grad_bytes || gb > grad_bytes - d.grad_offset) range = true;
  }
  for (size_t i = 0; i < named.size(); i++)
    for (size_t j = 0; j < i; j++) {
      const fr_tensor_desc &x = t[named[i]], &y = t[named[j]];
      if (named[i] == named[j]) over = true;
      if (bytes(x) && bytes(y) && x.src_offset < y.src_offset + bytes(y) && y.src_offset < x.src_offset + bytes(x)) over = true;
    }
  const int k = inval + align + range + over;
  if (k > 1) return -100;
  return inval ? FR_E_INVAL : align ? FR_E_ALIGN : range ? FR_E_RANGE : over ? FR_E_OVERLAP : FR_OK;
}

int main() {
  uint64_t accepted = 0, refused = 0, wrong = 0;
  for (int it = 0; it < 20000; it++) {
    const uint32_t n = uint32_t(U(6)), gdt = U(2) ? FR_F32 : FR_BF16;
    std::vector<uint64_t> numel(n);
    std::vector<uint8_t> bits(n);
    for (uint32_t k = 0; k < n; k++) {
      numel[k] = U(3) ? U(3000) : U(2) ? 0 : 256 * U(9);
      bits[k] = U(2) ? 8 : 32;
    }
    uint32_t ne = 0;
    uint64_t ab = 0, gb = 0;
    if (fr_adamw_state_table(numel.data(), bits.data(), n, gdt, nullptr, 0, &ne, nullptr, &ab, &gb) != FR_OK) wrong++;
    std::vector<fr_tensor_desc> t(ne);
    std::vector<fr_adamw_tensor> a(n);
    if (ne && fr_adamw_state_table(numel.data(), bits.data(), n, gdt, t.data(), ne - 1, &ne, a.data(), &ab, &gb) != FR_E_RANGE) wrong++;
    if (fr_adamw_state_table(numel.data(), bits.data(), n, gdt, t.data(), ne, &ne, a.data(), &ab, &gb) != FR_OK) wrong++;
    const uint64_t C = uint64_t(16) << U(12);
    fr_adamw_info info;
    if (fr_adamw_query(t.data(), ne, C, ab, a.data(), n, 1, gb, &info) != FR_OK) wrong++;
    uint64_t el = 0, e8 = 0, ctr = 0;
    for (uint32_t k = 0; k < n; k++) {
      el += numel[k];
      e8 += bits[k] == 8 ? numel[k] : 0;
      ctr += (numel[k] + 1023) / 1024 * 1024;
    }
    if (info.n_elements != el || info.n_elements_8bit != e8 || info.n_counters != ctr) wrong++;
    // adversarial: some fields changed
    uint32_t groups = 1;
    for (uint64_t c = U(4); c && n; c--) {
      fr_adamw_tensor& d = a[U(n)];
      const int32_t some = U(3) ? int32_t(U(ne + 1)) : U(2) ? -1 : int32_t(rng());
      switch (U(12)) {
        case 0: d.grad_offset = U(2) ? rng() : 16 * U(gb / 8 + 2); break;
        case 1: d.grad_dtype = uint32_t(U(4)); break;
        case 2: d.group = uint32_t(U(3)); break;
        case 3: d.param = some; break;
        case 4: d.master = some; break;
        case 5: d.m = some; break;
        case 6: d.v = some; break;
        case 7: d.m_scale = some; break;
        case 8: d.v_scale = some; break;
        case 9: d.flags = uint32_t(U(3)); break;
        case 10: groups = uint32_t(U(3)); break;
        case 11:
          if (ne > 1) {  // sender ranges may overlap in a table
            const uint32_t x = uint32_t(U(ne));
            t[x].src_offset = t[U(ne)].src_offset;
            if (t[x].src_offset + bytes(t[x]) > ab) ab = t[x].src_offset + bytes(t[x]);
          }
      }
    }
    const int rc = fr_adamw_query(t.data(), ne, C, ab, a.data(), n, groups, gb, &info), want = expect(t, a, groups, gb);
    if (want == -100 ? rc == FR_OK : rc != want) wrong++;
    (rc == FR_OK ? accepted : refused)++;
  }
  std::printf("%llu accepted, %llu refused, %llu wrong\n", (unsigned long long)accepted, (unsigned long long)refused,
              (unsigned long long)wrong);
  return wrong != 0 || accepted < 1000 || refused < 1000;
}
