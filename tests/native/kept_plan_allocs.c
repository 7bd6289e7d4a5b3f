/* Host allocations of a call whose plan the thread keeps: none.
 *
 * A serving program calls every layer of a step with the same lengths, and asks for the
 * workspace with them too; finding the kept plan compares the lengths and builds nothing.
 * Counts malloc (which C++'s operator new uses) around 1000 repeated workspace queries
 * of each kind.  Needs no GPU.  Prints "ok" and exits 0 on success. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "cw.h"
#include "cw_layer.h"

extern void* __libc_malloc(size_t n);
static _Thread_local long mallocs;
void* malloc(size_t n) {
  ++mallocs;
  return __libc_malloc(n);
}

enum { SEQS = 5, CALLS = 1000 };
static const int32_t kLp[SEQS] = {900, 40, 333, 0, 7000}, kLs[SEQS] = {1, 200, 1, 64, 1};

static size_t step(void) { return cw_step_workspace_bytes(kLp, kLs, SEQS, 4, 3, 128, 16, CW_KV_BF16); }
static size_t extend(void) { return cw_extend_workspace_bytes(kLp, kLs, SEQS, 4, 3, 128, 16); }
static size_t diff(void) { return cw_diff_workspace_bytes(kLp, kLs, SEQS, 2, 3, 128, 16, CW_KV_BF16); }

static int check(const char* name, size_t (*query)(void)) {
  const size_t want = query();
  if (query() != want || want == 0) {
    fprintf(stderr, "FAIL %s: sizes differ\n", name);
    return 1;
  }
  const long before = mallocs;
  for (int i = 0; i < CALLS; ++i)
    if (query() != want) return 1;
  const long n = mallocs - before;
  if (n != 0) fprintf(stderr, "FAIL %s: %ld allocations in %d calls with a kept plan\n", name, n, CALLS);
  return n != 0;
}

int main(void) {
  free(malloc(16));
  if (mallocs == 0) {
    fprintf(stderr, "FAIL malloc is not counted\n");
    return 1;
  }
  const int bad = check("extend", extend) + check("step", step) + check("diff", diff);
  if (bad == 0) printf("ok\n");
  return bad != 0;
}
