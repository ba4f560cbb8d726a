"""lmt.h's calls on a device that only notes what is launched on it (tests/fake_device), and from a C program."""
import os
import subprocess

import pytest

import fake_device
import paper_2402_02447_amd as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

LIB = """
from ctypes import *
L = CDLL(B.library_path())
for f in ("lmt_embed_grad_workspace", "lmt_matmul_workspace"):
    getattr(L, f).restype = c_uint64
P, U, D = (lambda x: c_void_p(x)), c_uint64, c_double
GB = 1 << 33
def embed(tokens, width, vocab=1000, dt=0, odt=0):
    return L.lmt_embed(P(GB), dt, U(vocab), U(width), U(width), P(GB), 6, U(tokens), D(1), P(GB), odt, U(width), None, None)
def grad(tokens, width, vocab=1000, dt=0, gdt=0, flags=0):
    ws = L.lmt_embed_grad_workspace(U(tokens), U(vocab), U(width))
    return L.lmt_embed_grad(P(GB), dt, U(width), P(GB), 6, U(tokens), D(1), c_int64(-1), P(GB), gdt, U(vocab), U(width), U(width), flags, None, P(GB), U(ws), None)
def quantize(rows, cols, t=True):
    return L.lmt_quantize(P(GB), 2, U(rows), U(cols), U(cols), 3, 0, P(GB), P(GB), P(GB if t else 0), P(GB if t else 0), None)
def matmul(m, n, k, cdt=2, flags=0):
    ws = L.lmt_matmul_workspace(U(m), U(n), U(k))
    return L.lmt_matmul(P(GB), 3, P(GB), P(GB), 3, P(GB), U(m), U(n), U(k), P(GB), cdt, U(n), flags, P(GB), U(ws), None)
def loss(rows, classes, dt=2):
    return L.lmt_cross_entropy(P(GB), dt, U(rows), U(classes), U(classes), P(GB), 6, c_int64(-100), None, P(GB), P(GB), P(GB), U(classes), None, None)
"""


@pytest.fixture(scope="module")
def device(tmp_path_factory):
    return fake_device.build(tmp_path_factory.mktemp("fake"))


def test_a_grid_never_has_more_threads_than_32_bits_count(device):
    """Every kernel has 1024 threads or fewer; the sizes are ones that 288 GB of memory hold, up to LMT_MAX_ROWS."""
    fake_device.run(device, LIB + """
MOST = 0x7fffff00
for call, launched in ((lambda: loss(MOST, 3), -(-MOST // 4)), (lambda: loss(1 << 26, 1000), 1 << 24), (lambda: loss((1 << 24) + 5, 2000), (1 << 24) + 5),
                       (lambda: loss(1 << 21, 60000), 1 << 21), (lambda: loss((1 << 21) + 1, 60000), (1 << 21) + 1)):
    assert call() == 0
    seen = kernels()
    assert sum(g for _, g in seen) == launched and max(g for _, g in seen) << 10 < 1 << 32, seen
    assert all(g > 0 for _, g in seen)
for call in (lambda: embed(MOST, 8), lambda: embed(MOST, 60), lambda: quantize(1 << 30, 1, False), lambda: quantize(1 << 23, 1000, False), lambda: quantize((1 << 23) - 1, 8000),
             lambda: matmul(MOST, 1, 100), lambda: matmul(1, MOST, 100), lambda: matmul(1, 1 << 30, 128), lambda: matmul(1 << 18, 1 << 18, 1 << 10),
             lambda: matmul(MOST, 64, 0, 0), lambda: grad(MOST, 1), lambda: grad(MOST, 20), lambda: grad(1 << 23, 8000), lambda: grad(3, 20, vocab=MOST),
             lambda: grad(70000, 20, vocab=MOST), lambda: grad(0, 20, vocab=MOST)):
    assert call() == 0
    seen = kernels()
    threads = {"k_quantize": 512, "k_matmul": 256, "k_embed": 256, "k_token_none": 256, "k_token_sums": 256}
    assert seen and all(0 < g and g * threads.get(k, 1024) < 1 << 32 for k, g in seen), seen
""")


def test_what_a_call_enqueues(device):
    """Few launches, no memory of its own, and none for empty work."""
    fake_device.run(device, LIB + """
before = fake.fake_device_allocations()
fake.fake_fail_host_allocations(1)
for call, names in ((lambda: embed(100, 64), ["k_embed"]), (lambda: quantize(100, 200), ["k_quantize"]), (lambda: loss(19, 30522), ["k_cross_entropy"]),
                    (lambda: loss(1, 1 << 20), ["k_cross_entropy_long"]),
                    (lambda: grad(1, 64), ["k_token_sort", "k_token_sums"]), (lambda: grad(500, 64), ["k_token_sort", "k_token_sums", "k_token_joins"]),
                    (lambda: grad(16384, 64), ["k_token_sort", "k_token_sums", "k_token_joins"]),
                    (lambda: grad(16385, 64), ["k_token_counts", "k_token_move", "k_token_sums", "k_token_joins"]),
                    (lambda: grad(16385, 64, vocab=30522), 2 * ["k_token_counts", "k_token_move"] + ["k_token_sums", "k_token_joins"]),
                    (lambda: grad(0, 64), ["k_token_none"]), (lambda: grad(0, 64, flags=1), []),
                    (lambda: matmul(37, 1024, 1024), ["k_matmul_few"]), (lambda: matmul(2432, 30522, 1024), ["k_matmul"]),
                    (lambda: matmul(1024, 1024, 4096, 0), ["k_matmul", "k_matmul_join"]), (lambda: matmul(3, 4, 0, flags=1), []),
                    (lambda: embed(0, 8), []), (lambda: embed(8, 0), []), (lambda: quantize(0, 8), []), (lambda: matmul(0, 8, 8), []), (lambda: loss(0, 8), [])):
    code = call()
    seen = [k for k, _ in kernels()]
    fake.fake_fail_host_allocations(0)
    assert code == 0 and seen == names, (seen, names)
    fake.fake_fail_host_allocations(1)
fake.fake_fail_host_allocations(0)
assert fake.fake_device_allocations() == before
""")


def test_c99_program_builds_against_the_header_and_runs(tmp_path):
    (tmp_path / "check.c").write_text("""
#include <stdio.h>
#include <string.h>
#include "lmt.h"
int main(void) {
  float x[4] = {0};
  int32_t t[1] = {0};
  if (lmt_fp8_row_bytes(129) != 256 || lmt_scale_row_bytes(513) != 8 || lmt_embed_grad_workspace(0, 5, 5) != 0) return 1;
  if (lmt_embed(x, LMT_F32, 1, 4, 3, t, LMT_I32, 1, 1.0, x, LMT_F32, 4, NULL, NULL) != LMT_ERR_ARG || !strstr(lmt_last_error(), "stride")) return 2;
  if (lmt_embed_grad(x, LMT_F32, 4, t, LMT_I32, 1, 1.0, -1, x, LMT_F32, 1, 4, 4, LMT_ACCUMULATE, NULL, x, 0, NULL) >= 0) return 3;
  if (lmt_quantize(x, LMT_F32, 1, 4, 4, LMT_E4M3, 0, NULL, NULL, NULL, NULL, NULL) != LMT_ERR_NULL) return 4;
  if (lmt_matmul(x, LMT_F32, NULL, x, LMT_E5M2, NULL, 1, 1, 1, x, LMT_F32, 1, 0, NULL, 0, NULL) != LMT_ERR_ARG) return 5;
  if (lmt_cross_entropy(x, LMT_F32, 1, 0, 4, t, LMT_I32, -100, NULL, x, NULL, NULL, 0, NULL, NULL) != LMT_ERR_ARG) return 6;
  puts("lmt ok");
  return 0;
}
""")
    lib, exe = B.library_path(), str(tmp_path / "check")
    libdir = os.path.dirname(lib)
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "check.c"),
                    "-o", exe, "-L", libdir, "-l:libbca.so", f"-Wl,-rpath,{libdir}", "-Wl,--allow-shlib-undefined"], check=True)
    import torch
    env = dict(os.environ, LD_LIBRARY_PATH=os.path.join(os.path.dirname(torch.__file__), "lib") + ":" + os.environ.get("LD_LIBRARY_PATH", ""))
    r = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert r.returncode == 0 and "lmt ok" in r.stdout, r.stdout + r.stderr
