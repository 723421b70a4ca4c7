"""What the decoder's operators ask of the CUDA runtime, checked without a GPU: their host code, compiled against stand-ins
for the calls that launch a kernel, set its limit of shared memory and look up the driver's tensor maps, which write down what
they are given."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_20305_b200", "csrc")

STANDINS = r"""
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdio>
#include <map>
#include <set>
std::map<const void*, std::set<int>> limits;      // of a kernel: what its limit of shared memory was set to
std::map<const void*, size_t> most;               // the most that a launch asked for
int launches = 0, fails_from = 1 << 30;           // launches so far; the first one that is refused
extern "C" cudaError_t recorded_limit(const void* kernel, cudaFuncAttribute, int bytes) {
  limits[kernel].insert(bytes);
  return cudaSuccess;
}
void look(const void* kernel, void** arguments);
extern "C" cudaError_t recorded_launch(const cudaLaunchConfig_t* config, const void* kernel, void** arguments) {
  look(kernel, arguments);
  if (config->dynamicSmemBytes > most[kernel]) most[kernel] = config->dynamicSmemBytes;
  return ++launches >= fails_from ? cudaErrorLaunchOutOfResources : cudaSuccess;
}
// (a tensor map that holds nothing but the address of its tensor)
static CUresult address_as_map(CUtensorMap* map, CUtensorMapDataType, cuuint32_t, void* address, const cuuint64_t*, const cuuint64_t*,
                               const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                               CUtensorMapFloatOOBfill) {
  *reinterpret_cast<void**>(map) = address;
  return CUDA_SUCCESS;
}
extern "C" cudaError_t recorded_entry(const char*, void** fn, unsigned long long, cudaDriverEntryPointQueryResult* found) {
  *fn = reinterpret_cast<void*>(&address_as_map);
  *found = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
#include "%s"
namespace psa {
psa_status_t check_last_cuda_error(const char*) { return launches >= fails_from ? PSA_ERR_CUDA : PSA_OK; }
}  // namespace psa
void* const P = reinterpret_cast<void*>(4096);
#define FLOATS reinterpret_cast<float*>(4096)
#define INTS reinterpret_cast<int*>(4096)
%s
int main() {
%s
  return 0;
}
"""


def run(tmp_path, source, body, look="void look(const void*, void**) {}"):
    """The output of a program that has `source`'s host code with the stand-ins, and `body` as its main function.  `look` is
    called at every launch."""
    (tmp_path / "host.cu").write_text(STANDINS % (source, look, body))
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    # (no machine code for the kernels: nothing here runs them)
    done = subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=compute_100a", "-DcudaLaunchKernelExC=recorded_launch",
                           "-DcudaFuncSetAttribute=recorded_limit", "-DcudaGetDriverEntryPoint=recorded_entry", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o",
                           str(tmp_path / "host"), str(tmp_path / "host.cu")], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    done = subprocess.run([str(tmp_path / "host")], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    return done.stdout


def test_a_kernels_limit_of_shared_memory_does_not_depend_on_the_call(tmp_path):
    """The limit belongs to the kernel, not to the call, and host threads share it: one that lowered it between another
    one's setting and launch would have that launch refused."""
    out = run(tmp_path, "psa_norm.cu", r"""
  for (int hidden = 1; hidden <= 16384; ++hidden)
    for (long long tokens : {1LL, 300LL, 5000LL, 200000LL})
      for (int types = 0; types < 3; ++types)
        for (void* d_total : {(void*)nullptr, P}) {
          const int x = types == 2 ? PSA_DTYPE_F32 : PSA_DTYPE_BF16, w = types == 0 ? PSA_DTYPE_BF16 : PSA_DTYPE_F32;
          if (psa_norm_bwd(P, P, P, FLOATS, d_total, x, w, tokens, hidden, 0, P, P, P, P, nullptr, nullptr) != PSA_OK) return 1;
        }
  for (auto& l : limits) {
    printf("%zu %zu", l.second.size(), most[l.first]);
    for (int bytes : l.second) printf(" %d", bytes);
    printf("\n");
  }""")
    kernels = [[int(v) for v in line.split()] for line in out.splitlines()]
    assert len(kernels) >= 12
    for n, most, *values in kernels:
        assert n == 1 and most <= values[0] <= 227 * 1024, (n, most, values[:5])


@pytest.mark.parametrize("source,call,n", [
    ("psa_embed.cu", "psa_embed_bwd(P, INTS, PSA_DTYPE_BF16, PSA_DTYPE_BF16, 1000, 500, 72, 1.0f, 0, P, P, nullptr, nullptr)", 3),
    ("psa_norm.cu", "psa_norm_bwd(P, P, P, FLOATS, P, PSA_DTYPE_BF16, PSA_DTYPE_BF16, 1000, 72, 0, P, P, P, P, nullptr, nullptr)", 2)])
def test_nothing_is_launched_behind_a_refused_launch(tmp_path, source, call, n):
    """The sums of the embedding's gradient take token numbers and ids as addresses from what the launch before them wrote."""
    out = run(tmp_path, source, r"""
  for (int first = 1; first <= %d; ++first) {
    launches = 0;
    fails_from = first;
    const int rc = %s;
    printf("%%d %%d\n", rc == PSA_ERR_CUDA, launches);
  }""" % (n + 1, call))
    assert out.split("\n")[:-1] == ["1 %d" % k for k in range(1, n + 1)] + ["0 %d" % n]


LOOK = r"""
std::set<const void*> written;      // by the call's launches so far
int call_launches = 0, early = 0, wrong = 0;
void look(const void*, void** arguments) {
  const psa::ProductList& list = *static_cast<const psa::ProductList*>(arguments[0]);
  for (int i = 0; i < list.n_products; ++i) {
    if (!list.p[i].early) continue;
    ++early;
    wrong += call_launches == 0;      // nothing is known of what the stream holds before the call
    for (const psa::OperandMaps& b : list.maps[i].b)
      if (const void* from = *reinterpret_cast<const void* const*>(&b.flat)) wrong += int(written.count(from));
  }
  for (int i = 0; i < list.n_products; ++i)
    for (const void* to : list.p[i].out) written.insert(to);
  written.insert(list.h);
  written.erase(nullptr);
  ++call_launches;
}
"""


def test_weights_are_requested_early_only_where_no_launch_that_may_still_run_writes_them(tmp_path):
    """ffn_small_kernel loads the B operand of an `early` product before behind_wait(): a launch before it in the same call must
    have waited for all that came before the call, and none of the call may write the operand."""
    out = run(tmp_path, "psa_ffn.cu", r"""
  char* at = reinterpret_cast<char*>(1 << 20);
  auto next = [&] { return static_cast<void*>(at += 4096); };
  for (long long tokens : {1LL, 60LL, 200LL, 700LL, 1815LL, 3000LL, 16215LL})
    for (int hidden : {64, 256, 2048, 4096})
      for (int ffn : {72, 704, 5632, 14336}) {
        void *x = next(), *wg = next(), *wu = next(), *wd = next(), *y = next(), *g = next(), *u = next(), *ws = next();
        written.clear();
        call_launches = 0;
        if (psa_ffn(x, wg, wu, wd, tokens, hidden, ffn, y, g, u, ws, nullptr, nullptr) != PSA_OK) return 1;
        written.clear();
        call_launches = 0;
        at += 1LL << 32;
        void* scratch = next();
        at += 1LL << 32;
        if (psa_ffn_bwd(y, x, wg, wu, wd, g, u, tokens, hidden, ffn, next(), next(), next(), next(), scratch, nullptr, nullptr) != PSA_OK)
          return 1;
      }
  printf("%d %d %d\n", launches, early, wrong);""", LOOK)
    launches, early, wrong = map(int, out.split())
    assert launches >= 7 * 16 * 4 and early >= 7 * 16 * 2 and wrong == 0


def test_kernels_of_the_feed_forward_block_wait_before_they_let_the_next_one_start():
    source = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "psa_ffn.cu")).read())
    calls = re.findall(r"behind_(wait|go)\(\)", source)
    assert len(calls) == 6 and calls == ["wait", "go"] * 3
