/* The short division of the optimizer step, q + (m - d q) y with y = 1 / d and
 * q = m y, each operation rounded once (fused where written so), on the
 * quotients of 24-bit numbers that come nearest to a border: a number of 24
 * bits, or halfway between two.  Where a 2^k = e (mod b), k = 24 + (a < b) bits
 * put the quotient between 2^24 and 2^25, e / b from a whole number: an even
 * one is a number of 24 bits, an odd one lies between two.  All b of 24 bits,
 * |e| <= 4 (times the powers of two that divide b), all a of 24 bits for which
 * that holds.  Built with gcc -O3 -march=native -ffp-contract=off -fopenmp. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

static int wrong(float a, float b) {
  const float y = 1.0f / b, q = a * y;
  return fmaf(fmaf(-b, q, a), y, q) != a / b;
}

/* x 2^-k modulo the odd b */
static int64_t halved(int64_t x, int k, int64_t b) {
  for (; k; k--) x = (x & 1 ? x + b : x) >> 1;
  return x;
}

int main(void) {
  const int64_t lo = 1 << 23, hi = 1 << 24;
  uint64_t n = 0, bad = 0;
#pragma omp parallel for reduction(+ : n, bad) schedule(dynamic, 4096)
  for (int64_t b = lo; b < hi; b++) {
    const int twos = __builtin_ctzll((unsigned long long)b);
    const int64_t odd = b >> twos;
    if (odd == 1) continue; /* a power of two: every quotient is exact */
    for (int k = 24; k <= 25; k++) {
      if (k < twos) continue;
      for (int64_t e = -4; e <= 4; e++) {
        /* a 2^(k - twos) = e (mod odd) */
        const int64_t a0 = halved((e % odd + odd) % odd, k - twos, odd);
        int left = 64; /* (of a small odd part many; they repeat what the others show) */
        for (int64_t a = a0 + (lo - a0 + odd - 1) / odd * odd; a < hi && left; a += odd, left--) {
          if ((a < b) != (k == 25)) continue;
          n++;
          bad += (uint64_t)wrong((float)a, (float)b);
        }
      }
    }
  }
  printf("%llu quotients, %llu wrong\n", (unsigned long long)n, (unsigned long long)bad);
  return bad != 0 || n < 50000000;
}
