"""What the entry points of the logits and of one expert's block refuse, and their workspaces, on the host; what the compiler made of
their kernels.  Nothing is launched here."""
import ctypes
import re

import pytest
import torch

import paper_2402_14800_amd as pkg
from paper_2402_14800_amd import binding, build
from tests.test_kernel_resources import k_loops

LIB = binding._lib
P = ctypes.c_void_p
ONE = P(1 << 20)
EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 3


def logprobs(logits=ONE, ld=100, tokens=ONE, T=4, V=100, dt=1, K=5, lp=ONE, ent=ONE, tlp=ONE, ids=ONE):
    return LIB.moe_token_logprobs(logits, ld, tokens, T, V, dt, K, lp, ent, tlp, ids, None)


def test_logprobs_refusals():
    assert logprobs(dt=2) == EINVAL
    assert logprobs(T=-1) == EINVAL and logprobs(T=(1 << 30) + 1) == EINVAL
    assert logprobs(V=0) == EINVAL and logprobs(V=(1 << 28) + 1, ld=1 << 30) == EINVAL
    assert logprobs(ld=99) == EINVAL
    assert logprobs(K=-1) == EINVAL and logprobs(K=129, V=1000, ld=1000) == EINVAL
    assert logprobs(K=8, V=7, ld=7) == EINVAL                # more alternatives than there are
    assert logprobs(logits=None) == EINVAL and logprobs(tokens=None) == EINVAL
    assert logprobs(lp=None) == EINVAL and logprobs(ent=None) == EINVAL
    assert logprobs(tlp=None) == EINVAL and logprobs(ids=None) == EINVAL
    assert logprobs(logits=P((1 << 20) + 1)) == EUNSUPPORTED and logprobs(logits=P((1 << 20) + 2), dt=0) == EUNSUPPORTED
    assert logprobs(T=0, logits=None, tokens=None) == 0


def distill(logits=ONE, ld=100, ids=ONE, teacher=ONE, T=4, V=100, K=5, dt=1, tau=1.0, w=None, loss=ONE, stats=ONE, grad=ONE, ldg=100):
    return LIB.moe_distill_topk(logits, ld, ids, teacher, T, V, K, dt, ctypes.c_float(tau), w, loss, stats, grad, ldg, None)


def backward(logits=ONE, ld=100, ids=ONE, teacher=ONE, stats=ONE, gl=ONE, T=4, V=100, K=5, dt=1, tau=1.0, grad=ONE, ldg=100):
    return LIB.moe_distill_topk_backward(logits, ld, ids, teacher, stats, gl, T, V, K, dt, ctypes.c_float(tau), grad, ldg, None)


@pytest.mark.parametrize("call", [distill, backward])
def test_distillation_refusals(call):
    assert call(dt=7) == EINVAL and call(T=-1) == EINVAL and call(V=0) == EINVAL and call(ld=99) == EINVAL and call(ldg=99) == EINVAL
    assert call(K=0) == EINVAL and call(K=129) == EINVAL
    for tau in (0.0, -1.0, float("nan"), float("inf")):
        assert call(tau=tau) == EINVAL
    for name in ("logits", "ids", "teacher", "stats"):
        assert call(**{name: None}) == EINVAL
    assert call(logits=P((1 << 20) + 1)) == EUNSUPPORTED and call(grad=P((1 << 20) + 1)) == EUNSUPPORTED
    assert call(T=0, logits=None, ids=None, teacher=None, stats=None) == 0
    if call is distill:
        assert call(loss=None) == EINVAL
    else:
        assert call(gl=None) == EINVAL and call(grad=None) == EINVAL


def test_expert_block_refusals():
    fw = lambda x=ONE, w1=ONE, w3=ONE, w2=ONE, T=64, H=64, F=128, dt=1, y=ONE, gu=None, ws=ONE, n=1 << 40: \
        LIB.expert_ffn_forward(x, w1, w3, w2, T, H, F, dt, y, gu, ws, n, None)  # noqa: E731
    bw = lambda dy=ONE, x=ONE, w1=ONE, w3=ONE, w2=ONE, gu=ONE, T=64, H=64, F=128, dt=1, dx=ONE, d1=ONE, d3=ONE, d2=ONE, ws=ONE, n=1 << 40: \
        LIB.expert_ffn_backward(dy, x, w1, w3, w2, gu, T, H, F, dt, dx, d1, d3, d2, ws, n, None)  # noqa: E731
    for f in (fw, bw):
        assert f(dt=5) == EINVAL and f(T=-1) == EINVAL and f(H=0) == EINVAL and f(F=0) == EINVAL
        assert f(H=96) == EUNSUPPORTED and f(F=100) == EUNSUPPORTED and f(H=6, dt=0) == EUNSUPPORTED and f(F=1 << 19) == EUNSUPPORTED
        assert f(w1=None) == EINVAL and f(w3=None) == EINVAL and f(w2=None) == EINVAL and f(x=None) == EINVAL
        assert f(ws=None) == EWORKSPACE and f(ws=P((1 << 20) + 16)) == EWORKSPACE and f(n=255) == EWORKSPACE
        for name in ("x", "w1", "w3", "w2", "gu"):
            assert f(**{name: P((1 << 20) + 8)}) == EUNSUPPORTED
    assert fw(y=None) == EINVAL and fw(T=0, x=None, y=None, ws=None, n=0) == 0
    assert bw(dy=None) == EINVAL and bw(gu=None) == EINVAL
    assert bw(d1=None) == EINVAL and bw(d3=None) == EINVAL and bw(d2=None) == EINVAL     # all of them or none
    assert bw(dx=None, d1=None, d3=None, d2=None, ws=None, n=0) == 0                     # nothing is wanted
    assert bw(dx=P((1 << 20) + 4)) == EUNSUPPORTED and bw(d3=P((1 << 20) + 2)) == EUNSUPPORTED


def test_expert_block_workspaces():
    fw, bw = binding.expert_ffn_forward_workspace, binding.expert_ffn_backward_workspace
    assert fw(0, 64, 64, 1) == 0 and bw(0, 64, 64, 1) == 0 and fw(0, 64, 64, 0, True) == 0
    assert fw(1, 65, 64, 1) == 0 and bw(10, 64, 64, 3) == 0 and bw(1 << 29, 4096, 14336, 1) > 0
    assert fw(1, 4096, 14336, 1) == 14336 * 2                                            # h of the one row
    for T in (1, 63, 64, 65, 777, 8192):
        for H, F in ((64, 64), (64, 14336), (4096, 64), (1024, 3584), (4096, 14336)):
            for dt, size in ((0, 4), (1, 2)):
                for save in (False, True):
                    assert fw(T, H, F, dt, save) >= T * F * size
                # dh, da | db, both weights transposed, x and dy along the tokens, da, db, h along the tokens
                assert bw(T, H, F, dt) >= T * F * 4 + 2 * T * F * size + 3 * H * F * size + 2 * T * H * size + 3 * T * F * size


def test_expert_block_plans_of_every_small_shape():
    """The plans divide by numbers of tiles and steps: none of them is zero."""
    for code, unit in ((binding.MOEP_BF16, 64), (binding.MOEP_F32, 4)):
        for T in (0, 1, 2, 31, 32, 33, 63, 64, 65, 777, 10 ** 6):
            for H in (unit, 2 * unit, 5 * unit, 64 * unit):
                for F in (unit, 2 * unit, 9 * unit, 64 * unit):
                    backward = binding.expert_ffn_backward_workspace(T, H, F, code)
                    forward = [binding.expert_ffn_forward_workspace(T, H, F, code, save) for save in (False, True)]
                    assert (backward > 0) == (T > 0) and all((n > 0) == (T > 0) for n in forward)


@pytest.mark.parametrize("bad", [
    lambda z, i, t: pkg.moe_token_logprobs(z, i[:, 0].long()),                           # (on the host)
    lambda z, i, t: pkg.moe_token_logprobs(z[0], i[0].long()),
    lambda z, i, t: pkg.moe_token_logprobs(z.t(), i[:, 0].long()),
    lambda z, i, t: pkg.moe_distill_topk(z, i, t),
    lambda z, i, t: pkg.expert_ffn_forward(z, z, z, z),
])
def test_binding_refuses_before_it_calls(bad):
    z, i, t = torch.zeros((4, 8)), torch.zeros((4, 3), dtype=torch.int32), torch.zeros((4, 3))
    with pytest.raises(ValueError):
        bad(z, i, t)


def test_logit_kernels_do_not_spill():
    """Rows are held in registers, 64 of them per lane: what spilled would wait behind every chunk in flight when it came back."""
    usage = build.kernel_resource_usage("logits.hip")
    kernels = {n: u for n, u in usage.items() if "token_logprobs_kernel" in n or "distill_topk_kernel" in n}
    assert len(kernels) == 44                                # 2 types: log probabilities by 4 workgroup sizes, 3 modes of the loss by 5, and not held
    for name, u in kernels.items():
        assert u["ScratchSize"] == 0 and u["VGPRs Spill"] == 0 and u["Occupancy"] >= 4, (name, u)


PLAN = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "tile_plan.h"
using namespace moep;
#define CHECK(x) do { if (!(x)) { std::printf("%s: line %d\n", #x, __LINE__); return 1; } } while (0)
int main() {
  std::srand(1);
  for (int round = 0; round < 20000; ++round) {              // every tile of every GEMM once
    const int n = 1 + std::rand() % 4;
    uint32_t end[4], total = 0;
    for (int i = 0; i < n; ++i) end[i] = total += 1 + std::rand() % (std::rand() % 2 ? 300 : 9);
    std::vector<int> seen(total, 0);
    for (uint32_t L = 0; L < total; ++L) {
      const SeveralTile t = tile_of_several(L, n, [&](int i) { return end[i]; });
      const uint32_t start = t.gemm ? end[t.gemm - 1] : 0;
      CHECK(t.gemm < n && t.tile < end[t.gemm] - start);
      ++seen[start + t.tile];
    }
    for (int s : seen) CHECK(s == 1);
  }
  for (int64_t tiles = 0; tiles < 400; ++tiles)
    for (int64_t units = 1; units < 300; units += 7)
      for (int any = 0; any < 2; ++any) {
        const int64_t r = k_ranges(tiles, 256, units, 8, any);
        CHECK(r >= 1 && (r == 1 || (r * 8 <= units && r * tiles <= 256 && (any || units % r == 0))));
      }
  for (int64_t T : {1, 63, 64, 65, 300, 777, 4096, 100000, 1000000})
    for (int64_t H : {64, 320, 1024, 4096, 65536})
      for (int64_t F : {64, 832, 3584, 14336, 262144}) {
        const BackwardCut c = cut_backward(T, H, F);
        CHECK(c.dx_ranges >= 1 && c.t_ranges >= 1 && (F / 32) % c.dx_ranges == 0);
        CHECK(!c.together || c.t_ranges <= (T + 63) / 64);
      }
  std::puts("ok");
}
"""


def test_plans_of_the_training_step(tmp_path):
    """The arithmetic that the kernels and the host share, run as a program of its own."""
    import os
    import subprocess

    csrc = os.path.join(os.path.dirname(build.__file__), "csrc")
    (tmp_path / "plan.cpp").write_text(PLAN)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", csrc, str(tmp_path / "plan.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_training_gemms_wait_for_the_loads_they_mean():
    """The properties of the 256-row GEMM that its waits rely on (the bodies are the same source), in the training step's instantiations."""
    usage = {n: u for n, u in build.kernel_resource_usage("gemm_train.hip").items() if "gemm_packed_kernel" in n}
    assert len(usage) == 4                                   # both branches kept, fp32 sums (2 weight layouts), several GEMMs
    for name, u in usage.items():
        assert u["ScratchSize"] == 0 and u["VGPRs Spill"] == 0 and u["SGPRs Spill"] == 0, (name, u)
        assert u["AGPRs"] == 256 and u["VGPRs"] <= 256 and u["Occupancy"] == 1, (name, u)
    text = build.device_assembly("gemm_train.hip").splitlines()
    starts = [i for i, line in enumerate(text) if re.match(r"_ZN\S*gemm_packed_kernel\S*:", line)]
    assert len(starts) == 4
    for start in starts:
        row_major = re.search(r"kernelILi\d+ELb[01]ELb([01])E", text[start]).group(1) == "1"
        bodies = set()
        for mfmas, ops in k_loops(text[start:next(i for i in range(start, len(text)) if ".Lfunc_end" in text[i])]):
            at = [i for i, o in enumerate(ops) if o == "s_barrier"]
            steps = [ops[b:e] for b, e in zip([0] + [i + 1 for i in at], at)]
            assert ops[-1] == "s_barrier" and len(steps) == (2 if row_major else 1), (text[start], ops)
            assert all(isinstance(s[-1], int) and not any(isinstance(o, int) for o in s[:-1]) for s in steps), (text[start], ops)
            loads, waits = [s[:-1] for s in steps], [s[-1] for s in steps]
            if row_major:                                    # weights by two lane offsets in turn, then the rows of A by a third
                w = max(i for i, o in enumerate(loads[0]) if o != loads[0][-1]) + 1
                a = len(loads[0]) - w
                for step in loads:
                    assert len(step) == w + a and len(set(step[0:w:2])) == len(set(step[1:w:2])) == len(set(step[w:])) == 1, (text[start], ops)
                assert waits == [w + 2 * a, 2 * (w + a)], (text[start], ops)
                assert mfmas == 2 * (2 * w) * (2 * a), (text[start], mfmas)
                bodies.add((2 * w, 2 * a))
            else:
                assert len(loads[0]) == 2 * waits[0], (text[start], ops)
                bodies.add((mfmas, waits[0]))
        tiles = [(ng, mg) for ng in (4, 8) for mg in (4, 6, 8)]
        assert bodies == ({*tiles} if row_major else {(2 * ng * mg, (ng + mg) // 2) for ng, mg in tiles}), (text[start], bodies)
