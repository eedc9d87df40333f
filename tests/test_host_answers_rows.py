"""What the entry points of the rows to the experts and of the losses on given answers refuse, their workspaces, and what the compiler made
of their kernels.  Nothing is launched here."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2402_14800_amd as pkg
from paper_2402_14800_amd import binding, build

LIB = binding._lib
P = ctypes.c_void_p
ONE = P(1 << 20)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
BAD = (float("nan"), float("inf"), -1.0)


def dispatch(x=ONE, ids=ONE, used=None, T=4, k=2, E=8, H=64, dt=1, rows=ONE, slots=ONE, off=ONE, ws=None, n=0):
    return LIB.moe_dispatch_rows(x, ids, used, T, k, E, H, dt, rows, slots, off, ws, n, None)


def dispatch_back(d=ONE, slots=ONE, T=4, k=2, H=64, R=8, dt=1, dx=ONE):
    return LIB.moe_dispatch_rows_backward(d, slots, T, k, H, R, dt, dx, None)


def combine(y=ONE, slots=ONE, w=ONE, T=4, k=2, H=64, R=8, dt=1, out=ONE):
    return LIB.moe_combine_rows(y, slots, w, T, k, H, R, dt, out, None)


def combine_back(d=ONE, y=ONE, slots=ONE, w=ONE, T=4, k=2, H=64, R=8, dt=1, dy=ONE, dw=ONE):
    return LIB.moe_combine_rows_backward(d, y, slots, w, T, k, H, R, dt, dy, dw, None)


@pytest.mark.parametrize("call", [dispatch, dispatch_back, combine, combine_back])
def test_rows_refusals(call):
    assert call(dt=2) == EINVAL and call(T=-1) == EINVAL and call(T=(1 << 29) + 1) == EINVAL and call(k=0) == EINVAL and call(k=17) == EINVAL
    assert call(H=0) == EINVAL and call(H=96) == EUNSUPPORTED and call(H=6, dt=0) == EUNSUPPORTED and call(H=(1 << 24) + 64) == EINVAL
    assert call(slots=None) == EINVAL and call(slots=P((1 << 20) + 2)) == EUNSUPPORTED
    if call is dispatch:
        assert call(E=0) == EINVAL and call(E=33) == EINVAL
        for name in ("x", "ids", "rows", "off"):
            assert call(**{name: None}) == EINVAL
        assert call(x=P((1 << 20) + 8)) == EUNSUPPORTED and call(rows=P((1 << 20) + 4)) == EUNSUPPORTED
        assert call(used=P((1 << 20) + 1)) == EUNSUPPORTED and call(off=P((1 << 20) + 1)) == EUNSUPPORTED
        assert call(T=0, off=None) == EINVAL
        big = dict(T=100000, k=2)
        need = binding.moe_dispatch_rows_workspace(100000, 2, 8)
        assert call(**big) == EWORKSPACE and call(ws=ONE, n=need - 1, **big) == EWORKSPACE and call(ws=P((1 << 20) + 128), n=need, **big) == EWORKSPACE
    else:
        assert call(R=-1) == EINVAL and call(R=(1 << 30) + 1) == EINVAL
        assert call(T=0, slots=None) == OK
    if call is dispatch_back:
        assert call(d=None) == EINVAL and call(dx=None) == EINVAL and call(d=P((1 << 20) + 8)) == EUNSUPPORTED and call(dx=P((1 << 20) + 8)) == EUNSUPPORTED
    if call is combine:
        assert call(y=None) == EINVAL and call(out=None) == EINVAL and call(w=P((1 << 20) + 2)) == EUNSUPPORTED and call(out=P((1 << 20) + 8)) == EUNSUPPORTED
    if call is combine_back:
        assert call(d=None) == EINVAL and call(y=None) == EINVAL and call(dy=None) == EINVAL
        assert call(dw=P((1 << 20) + 1)) == EUNSUPPORTED and call(y=P((1 << 20) + 8)) == EUNSUPPORTED and call(dy=P((1 << 20) + 8)) == EUNSUPPORTED


def test_dispatch_workspaces():
    ws = binding.moe_dispatch_rows_workspace
    assert ws(0, 2, 8) == 0 and ws(1, 16, 32) == 0 and ws(4096, 2, 8) == 0 and ws(512, 16, 32) == 0
    assert ws(4097, 2, 8) > 0 and ws(-1, 2, 8) == 0 and ws(10, 17, 8) == 0 and ws(10, 2, 33) == 0 and ws(1 << 30, 2, 8) == 0
    for T in (5000, 32768, 100001, 1 << 20, (1 << 26) - 1):
        for k, E in ((16, 32), (2, 8), (1, 32), (16, 1)):
            assert (0 < ws(T, k, E) <= 8192 * 4) if T * k > 8192 else ws(T, k, E) == 0


def policy(z=ONE, ld=100, tok=ONE, old=ONE, adv=ONE, ref=ONE, T=4, V=100, dt=1, lo=0.2, hi=0.2, kl=0.1, tau=1.0, w=None, loss=ONE, lp=ONE,
           stats=ONE, grad=ONE, ldg=100):
    f = ctypes.c_float
    return LIB.moe_policy_loss(z, ld, tok, old, adv, ref, T, V, dt, f(lo), f(hi), f(kl), f(tau), w, loss, lp, stats, grad, ldg, None)


def policy_back(z=ONE, ld=100, tok=ONE, stats=ONE, gl=ONE, T=4, V=100, dt=1, tau=1.0, grad=ONE, ldg=100):
    return LIB.moe_policy_loss_backward(z, ld, tok, stats, gl, T, V, dt, ctypes.c_float(tau), grad, ldg, None)


def preference(z=ONE, ld=100, tok=ONE, off=ONE, ref=ONE, T=4, V=100, pairs=2, dt=1, beta=0.1, ls=0.0, avg=0, w=None, loss=ONE, rew=ONE, lp=ONE,
               stats=ONE, grad=ONE, ldg=100):
    f = ctypes.c_float
    return LIB.moe_preference_loss(z, ld, tok, off, ref, T, V, pairs, dt, f(beta), f(ls), avg, w, loss, rew, lp, stats, grad, ldg, None)


def preference_back(z=ONE, ld=100, tok=ONE, off=ONE, stats=ONE, gl=ONE, T=4, V=100, pairs=2, dt=1, grad=ONE, ldg=100):
    return LIB.moe_preference_loss_backward(z, ld, tok, off, stats, gl, T, V, pairs, dt, grad, ldg, None)


@pytest.mark.parametrize("call", [policy, policy_back, preference, preference_back])
def test_loss_refusals(call):
    assert call(dt=7) == EINVAL and call(T=-1) == EINVAL and call(T=(1 << 30) + 1) == EINVAL
    assert call(V=0) == EINVAL and call(V=(1 << 28) + 1, ld=1 << 30, ldg=1 << 30) == EINVAL and call(ld=99) == EINVAL and call(ldg=99) == EINVAL
    assert call(z=P((1 << 20) + 1)) == EUNSUPPORTED and call(grad=P((1 << 20) + 1)) == EUNSUPPORTED and call(grad=P((1 << 20) + 2), dt=0) == EUNSUPPORTED
    assert call(z=None) == EINVAL and call(tok=None) == EINVAL and call(stats=None) == EINVAL
    assert call(tok=P((1 << 20) + 4)) == EUNSUPPORTED and call(stats=P((1 << 20) + 2)) == EUNSUPPORTED
    if call in (policy, policy_back):
        assert call(T=0, z=None, tok=None, stats=None) == OK
        for tau in (0.0, 2.0 ** -61, 2.0 ** 61) + BAD:
            assert call(tau=tau) == EINVAL
    if call is policy:
        for name in ("old", "adv", "loss", "lp"):
            assert call(**{name: None}) == EINVAL
        assert call(ref=None) == EINVAL                                                   # a KL term without a reference
        for x in BAD:
            assert call(lo=x) == EINVAL and call(hi=x) == EINVAL and call(kl=x) == EINVAL
        assert call(lo=1.5) == EINVAL and call(hi=2.0 ** 61) == EINVAL and call(kl=2.0 ** 61) == EINVAL
        assert call(w=P((1 << 20) + 2)) == EUNSUPPORTED and call(old=P((1 << 20) + 2)) == EUNSUPPORTED and call(lp=P((1 << 20) + 2)) == EUNSUPPORTED
    if call is policy_back:
        assert call(gl=None) == EINVAL and call(grad=None) == EINVAL
    if call is preference:
        for name in ("off", "ref", "loss", "rew", "lp"):
            assert call(**{name: None}) == EINVAL
        for x in BAD:
            assert call(beta=x) == EINVAL and call(ls=x) == EINVAL
        assert call(beta=0.0) == EINVAL and call(beta=2.0 ** 61) == EINVAL and call(ls=1.0) == EINVAL and call(avg=2) == EINVAL
        assert call(off=P((1 << 20) + 4)) == EUNSUPPORTED and call(rew=P((1 << 20) + 2)) == EUNSUPPORTED
        assert call(T=0, pairs=0, z=None, tok=None, ref=None, stats=None, lp=None, loss=None, rew=None) == OK
    if call is preference_back:
        assert call(gl=None) == EINVAL and call(grad=None) == EINVAL and call(off=None) == EINVAL
        assert call(T=0, z=None, tok=None) == OK and call(pairs=0, gl=None) == OK
    if call in (preference, preference_back):
        assert call(pairs=-1) == EINVAL and call(pairs=(1 << 22) + 1) == EINVAL


Z, I, S, F = torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.int64), torch.zeros(4)


@pytest.mark.parametrize("bad", [
    lambda: pkg.moe_dispatch_rows(Z, I, 8),                                               # (on the host)
    lambda: pkg.moe_dispatch_rows(Z, I.long(), 8),
    lambda: pkg.moe_dispatch_rows(Z, I[:3], 8),
    lambda: pkg.moe_dispatch_rows(Z, I, 8, used=F),
    lambda: pkg.moe_dispatch_rows(Z, I, 8, rows=Z),
    lambda: pkg.moe_dispatch_rows_backward(Z, I),
    lambda: pkg.moe_dispatch_rows_backward(Z[0], I),
    lambda: pkg.moe_combine_rows(Z, I),
    lambda: pkg.moe_combine_rows(Z, I, F),
    lambda: pkg.moe_combine_rows_backward(Z[:3], Z, I),
    lambda: pkg.moe_combine_rows_backward(Z, Z, I, dy=Z[:2]),
    lambda: pkg.moe_policy_loss(Z, S, F, F),
    lambda: pkg.moe_policy_loss(Z.t(), S, F, F),
    lambda: pkg.moe_policy_loss_backward(Z, S, Z, F),
    lambda: pkg.moe_preference_loss(Z, S, S, F),
    lambda: pkg.moe_preference_loss_backward(Z, S, S[:3], Z, F),
])
def test_binding_refuses_before_it_calls(bad):
    with pytest.raises(ValueError):
        bad()


def test_kernels_do_not_spill():
    usage = build.kernel_resource_usage("answers.hip")
    rows = {n: u for n, u in usage.items() if "answers_kernel" in n}
    # 2 types: the loss alone and the gradient alone by 3 workgroup sizes, both together by 5 and not held
    assert len(rows) == 24
    for name, u in rows.items():
        assert u["ScratchSize"] == 0 and u["VGPRs Spill"] == 0 and u["Occupancy"] >= 4, (name, u)
    for name, u in build.kernel_resource_usage("rows.hip").items():
        assert u["ScratchSize"] == 0 and u["VGPRs Spill"] == 0, (name, u)


def test_the_answer_of_a_row(tmp_path):
    """The search that the wavefronts make, run lane by lane on the CPU from its own source: the answer of every row, and for offsets in no
    order an end within the array."""
    text = open(os.path.join(build.CSRC, "answers.hip")).read()
    body = re.search(r"__device__ __forceinline__ int answer_of\(.*?\n}\n", text, re.S).group(0)
    body = body.replace("__device__ __forceinline__", "static").replace("const int lane = threadIdx.x & 63;", "")
    body = body.replace("__popcll(__ballot(at < hi && offsets[at] <= t))", "ballot").replace(", at = lo + (lane + 1) * step - 1;", ";")
    body = body.replace("const int k = ballot;", """int k = 0;
    for (int lane = 0; lane < 64; ++lane) {
      const int at = lo + (lane + 1) * step - 1;
      if (at < hi) { if (at < 0 || at >= n) std::abort(); k += offsets[at] <= t; }
    }
    if (++rounds > 4) std::abort();""")
    (tmp_path / "search.cpp").write_text("""#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>
using std::min;
static int rounds;
""" + body + """
int main() {
  std::srand(3);
  for (int round = 0; round < 3000; ++round) {
    const int n = 1 + 2 * (std::rand() % (round % 10 ? 70 : 6000)), T = 1 + std::rand() % 3000;
    std::vector<int64_t> o(n);
    for (auto& x : o) x = std::rand() % (T + 1);
    const bool sorted = round % 3;
    if (sorted) std::sort(o.begin(), o.end());
    for (int q = 0; q < 40; ++q) {
      const int64_t t = q < 2 ? (q ? T - 1 : 0) : std::rand() % T;
      rounds = 0;
      const int a = answer_of(o.data(), n, t);
      if (a < -1 || a >= n) return 1;
      if (sorted && a != std::upper_bound(o.begin(), o.end(), t) - o.begin() - 1) return 2;
    }
  }
  std::puts("ok");
}
""")
    exe = str(tmp_path / "search")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", str(tmp_path / "search.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_launches_keep_to_the_grid_limits(tmp_path):
    """Every launch at the largest sizes, noted by a program that stands in for the HIP runtime."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe, lib = str(tmp_path / "driver"), binding.library_path()
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-I", os.path.join(root, "include"),
                        os.path.join(root, "tests", "host_answers_rows_driver.cpp"), "-o", exe, lib, "-Wl,-rpath," + os.path.dirname(lib),
                        "-Wl,-rpath-link,/opt/rocm/lib", "-Wl,-rpath,/opt/rocm/lib", "-Wl,--unresolved-symbols=ignore-in-shared-libs"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "all checks passed", (r.stdout[-4000:], r.stderr[-2000:])
