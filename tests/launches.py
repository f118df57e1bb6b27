"""Which kernels a call of kvr_attend_shared launches, found without a GPU: a host program that puts its own launch calls and
registration of kernels before the runtime's, so that nothing is launched and every launch is named.  Test infrastructure."""
import os
import subprocess

from paper_2512_17917_amd import build as B

PROBE = r"""
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include "kvr_launch.h"
static size_t asked;
static std::map<const void*, std::string>& names() {          // (the library's kernels register before main's statics are there)
  static std::map<const void*, std::string> x;
  return x;
}
extern "C" void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[f] = name; }
static int device;
static std::map<std::pair<int, const void*>, int> limit;
extern "C" hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute a, int value) {
  if (a == hipFuncAttributeMaxDynamicSharedMemorySize) limit[{device, f}] = value;
  return hipSuccess;
}
extern "C" hipError_t hipGetDevice(int* dev) { *dev = device; return hipSuccess; }
extern "C" hipError_t hipLaunchKernel(const void* f, dim3, dim3, void**, size_t lds, hipStream_t) {
  std::printf(" %s:%zu:%d", names()[f].c_str(), lds, limit.count({device, f}) ? limit[{device, f}] : 65536);
  return hipSuccess;
}
extern "C" hipError_t __hipPushCallConfiguration(dim3, dim3, size_t lds, hipStream_t) { asked = lds; return hipSuccess; }
extern "C" hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, hipStream_t* st) {
  *g = dim3(1); *b = dim3(1); *lds = asked; *st = nullptr;
  return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }
int main() {
  int f32, B, Hq, Hkv, rows, by_start, page, cols, window, sink, groups, scores;
  while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d %d %d", &f32, &B, &Hq, &Hkv, &rows, &by_start, &page, &cols, &window, &sink, &groups, &scores, &device) == 13) {
    kvr::DevDesc d = {};
    d.B = B; d.Hq = Hq; d.Hkv = Hkv; d.G = Hq / Hkv; d.scale = 1.f;
    static int32_t x[4];                     // no kernel runs: never read
    kvr::SharedArgs s;
    std::memset(&s, 0, sizeof(s));
    kvr_pages p = {};
    p.k = p.v = x; p.table = x; p.n_pages = 1; p.page_size = page; p.table_cap = cols;
    s.a.pages = kvr::dev_pages(p);
    s.a.q = s.a.out = x; s.a.n_ctx = x; s.a.ws = x;
    s.a.n_rows = rows; s.a.q_start = by_start ? x : nullptr;
    s.a.vis.window = window; s.a.vis.n_sink = sink;
    s.a.scores = scores ? (float*)x : nullptr; s.a.n_cap = scores ? s.a.pages.cap : 0;
    s.start = s.n_shared = x; s.n_groups = groups;
    const hipError_t e = kvr::launch_attend_shared(d, f32 ? KVR_F32 : KVR_BF16, s, nullptr);
    std::printf(" %d\n", (int)e);
  }
}
"""


def build_probe(folder):
    """-> ask(list of dicts) -> a list of kernels' names (mangled) each; dicts: f32, B, Hq, Hkv, rows, by_start, page, cols, window,
    sink, groups, scores, device (0 if left out).  ask.lds: for each call its launches' dynamic LDS and the limit there."""
    src, exe = str(folder / "launches.hip"), str(folder / "launches")
    open(src, "w").write(PROBE)
    subprocess.run([B._hipcc(), "--offload-host-only", "-std=c++17", "-I", B.CSRC, src, "-L", os.path.dirname(B.OUT),
                    "-l:" + os.path.basename(B.OUT), f"-Wl,-rpath,{os.path.dirname(B.OUT)}", "-o", exe], check=True, capture_output=True)
    order = "f32 B Hq Hkv rows by_start page cols window sink groups scores device".split()

    def ask(calls):
        out = subprocess.run([exe], input="".join(" ".join(str(int(c.get(k, 0))) for k in order) + "\n" for c in calls), capture_output=True, text=True,
                             check=True).stdout.splitlines()
        assert len(out) == len(calls)
        got, ask.lds = [], []
        for c, line in zip(calls, out):
            *kernels, rc = line.split()
            assert rc == "0", (c, line)
            got.append([k.split(":")[0] for k in kernels])
            ask.lds.append([tuple(map(int, k.split(":")[1:])) for k in kernels])
        return got
    return ask


def call_of(b, dtype_is_f32, window=0, sink=0, scores=True):
    """The call that tests.test_gpu_shared.Batch.check makes."""
    return dict(f32=dtype_is_f32, B=b.B, Hq=b.Hq, Hkv=b.Hkv, rows=b.rows, by_start=b.q_start is not None, page=b.page, cols=b.table.shape[1],
                window=window, sink=sink, groups=len(b.common), scores=scores)
