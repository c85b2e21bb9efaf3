"""Which kernels the serving operators' calls get, from the rules themselves
(serve_plan.h, built here for the host): the tests of each kernel reach it, and go on
doing so when the rules' measured times change."""
import ctypes
import os
import shutil
import subprocess

import pytest

from test_gpu_linear_kernels import FORMS
from test_gpu_selected_kernels import PICKS, SCORES
from test_gpu_shared_kernels import KINDS

from paper_2010_02164_amd import _native as N
from paper_2010_02164_amd import build

UNITS = 256   # compute units of an MI355X

SOURCE = """
#include <string.h>
#include "serve_plan.h"
template <class T> T of(const void *p) { T a; memcpy(&a, p, sizeof a); return a; }
extern "C" {
void linear(const void *p, int n_cu, int *out) {
  const sb::LinearPlan q = sb::linear_plan(of<sb_linear_args>(p), n_cu);
  out[0] = q.tile, out[1] = q.splits;
}
void shared(const void *p, int *out) {
  const sb::SharedKinds k = sb::shared_kinds(of<sb_shared_args>(p));
  out[0] = k.prefix, out[1] = k.own;
}
int many_scores(const void *p) { return sb::many_scores(of<sb_select_args>(p)); }
void pick(const void *p, int n_cu, int *out) {
  const sb_select_args a = of<sb_select_args>(p);
  const sb::PickPlan q = sb::pick_plan(sb::pages_between(a), (long long)a.n_tokens * a.kv_heads, n_cu);
  out[0] = q.threads, out[1] = q.per;
}
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, str(at / "plan.cpp"), "-o", str(at / "plan.so")], check=True)
    return ctypes.CDLL(os.path.join(str(at), "plan.so"))


def ask(fn, args, *more, n=2):
    out = (ctypes.c_int * n)()
    fn(args, *more, out)
    return tuple(out)


@pytest.mark.parametrize("form", sorted(FORMS))
def test_linear_shapes(rules, form):
    for M, N_, K in FORMS[form]:
        assert K % 16 == 0
        args = N.LINEAR_ARGS.pack(N.LINEAR_ARGS.size, 0, 0, 0, 0, 0, 0, K + 48, K + 48, N_, M, N_, K, N.SB_BF16)
        tile, splits = ask(rules.linear, args, UNITS)
        got = ("few_16" if M <= 16 else "few_32" if M <= 32 else "few_64") if tile == 0 else "split" if splits > 1 else f"tiles_{tile}"
        assert got == form, (M, N_, K)


@pytest.mark.parametrize("kinds", sorted(KINDS))
def test_shared_forms(rules, kinds):
    for members, Hq, Hkv, q in KINDS[kinds]:
        q_lens = [q[i % len(q)] for i in range(sum(members))]
        own = [0] * 7 + [0] * 11 + [sum(q_lens), len(q_lens), Hq, Hkv, 128, N.SB_BF16, 4, 16, 4, 0, 0, max(q_lens), 100, 0.1]
        args = N.SHARED_ARGS.pack(N.SHARED_ARGS.size, N.ATTENTION_ARGS.size, *own, 0, 0, 0, 4, len(members), 4, 100, 0)
        assert ask(rules.shared, args) == kinds


def select_args(tokens, requests, Hkv, page, top, first, last, max_kv):
    return N.SELECT_ARGS.pack(N.SELECT_ARGS.size, 0, 0, 0, 0, 0, 0, 0, 64, 64, 9, tokens, requests, Hkv, Hkv, 64, N.SB_BF16, 9, page, 9, top, first, last,
                              max_kv, 0)


@pytest.mark.parametrize("pick", sorted(PICKS))
def test_selection_lists(rules, pick):
    for B, q, Hkv, page, kv, max_kv, held in PICKS[pick]:
        threads, per = pick
        most = -(-max(kv) // page) - 2   # ranked for the longest request, of the first and last page apart
        assert ask(rules.pick, select_args(B * q, B, Hkv, page, 4, 1, 1, max(kv) if max_kv is None else max_kv), UNITS) == pick
        assert (most <= threads * per) == held


def test_selection_scores(rules):
    for many, forms in SCORES.items():
        for B, q in forms:
            assert bool(rules.many_scores(select_args(B * q, B, 1, 16, 4, 1, 1, 1000))) == many
