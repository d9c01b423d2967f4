"""CPU checks of windowed attention's entry points: refusals, workspace sizes, counted pairs, the tiles of keys and of queries that the
kernels go over, and the 64-bit formulas that the GPU tests compare with."""
import ctypes
import itertools
import os
import re
import subprocess
import types

import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from paper_2503_02356_amd import build
from tests import plain_window as W
from tests.test_build_checks import REPORT, accumulator_faults

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def params(dtype=B.CF_BF16, Hq=4, Hkv=2, D=128, T=100, Tk=150):
    p = B.AttnFwdParams()
    p.dtype, p.n_q_heads, p.n_kv_heads, p.head_dim, p.softmax_scale = dtype, Hq, Hkv, D, 0.1
    p.n_tokens, p.n_kv_tokens, p.n_segments = T, Tk, 1
    p.cu_seqlens_q = p.cu_seqlens_k = p.lse = 4096
    p.q = p.k = p.v = p.o = 1 << 20
    p.q_stride_tok = p.o_stride_tok = Hq * D
    p.kv_stride_tok = Hkv * D
    p.q_stride_head = p.kv_stride_head = p.o_stride_head = D
    return p


def bwd(p, nbytes=1 << 30):
    b = B.AttnBwdParams()
    b.f = p
    b.d_o = b.d_q = b.d_k = b.d_v = b.workspace = 1 << 20
    b.do_stride_tok = b.dq_stride_tok = p.q_stride_tok
    b.dkv_stride_tok = p.kv_stride_tok
    b.do_stride_head = b.dq_stride_head = b.dkv_stride_head = p.head_dim
    b.workspace_bytes = nbytes
    return b


def refused(code, what, call):
    with pytest.raises(B.CfError) as e:
        call()
    assert e.value.code == code and what in str(e.value), e.value


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 0), (1, -1), (-2**31, 0)])
def test_windows_that_are_none_are_refused(window, sinks):
    p = params()
    refused(B.CF_EINVAL, "window >= 1", lambda: B.cf_attn_window_fwd(p, window, sinks, stream=0))
    refused(B.CF_EINVAL, "window >= 1", lambda: B.cf_attn_window_bwd(bwd(p), window, sinks, stream=0))
    refused(B.CF_EINVAL, "window >= 1", lambda: B.cf_attn_window_bwd_workspace_bytes(p, window, sinks))
    refused(B.CF_EINVAL, "window >= 1", lambda: B.cf_count_window_pairs([0, 1], [0, 1], window, sinks))
    for call in (B.lib().cf_attn_window_fwd, B.lib().cf_attn_window_bwd):
        assert call(ctypes.byref(p if call is B.lib().cf_attn_window_fwd else bwd(p)), None, None) == B.CF_EINVAL
        assert call(None, ctypes.byref(B.AttnWindow(1, 0)), None) == B.CF_EINVAL


def test_what_the_calls_without_a_window_refuse_is_refused():
    for change, code in ((dict(Hq=5), B.CF_EINVAL), (dict(D=96), B.CF_EUNSUPPORTED), (dict(dtype=2), B.CF_EUNSUPPORTED), (dict(T=0), B.CF_EINVAL),
                         (dict(T=151), B.CF_EINVAL)):
        refused(code, "", lambda: B.cf_attn_window_fwd(params(**change), 8, 0, stream=0))
        refused(code, "", lambda: B.cf_attn_window_bwd(bwd(params(**change)), 8, 0, stream=0))
        refused(code, "", lambda: B.cf_attn_window_bwd_workspace_bytes(params(**change), 8, 0))
    for field, value in (("q", 0), ("k", 8), ("q_stride_tok", 4), ("kv_stride_head", 12), ("flags", 64), ("softmax_scale", float("nan"))):
        p = params()
        setattr(p, field, value)
        refused(B.CF_EINVAL, "cf_attn_window_fwd", lambda: B.cf_attn_window_fwd(p, 8, 0, stream=0))
    p = params()
    need = B.cf_attn_window_bwd_workspace_bytes(p, 8, 2)
    refused(B.CF_EINVAL, "workspace", lambda: B.cf_attn_window_bwd(bwd(p, 256), 8, 2, stream=0))
    assert need >= 4 * 4 * 100
    b = bwd(p)
    b.workspace += 16
    refused(B.CF_EINVAL, "aligned", lambda: B.cf_attn_window_bwd(b, 8, 2, stream=0))


def test_workspace_does_not_grow_with_a_prefix_that_nobody_sees():
    near, far = (B.cf_attn_window_bwd_workspace_bytes(params(Tk=n), 64, 4) for n in (5000, 1 << 30))
    assert near == far


def test_workspace_of_the_largest_calls():
    """Sizes whose products leave 63 bits: the far rows' sums are not asked for (delta is: 2^30 rows of 2^15 heads)."""
    p = params(dtype=B.CF_FP32, Hq=1 << 15, Hkv=1 << 15, D=64, T=1 << 30, Tk=1 << 30)
    p.n_segments = 512
    assert B.cf_attn_window_bwd_workspace_bytes(p, 1, 1 << 30) == 1 << 47


def test_windows_longer_than_the_field():
    """2^32 + 3 keys are all of them, not 3."""
    assert B.cf_count_window_pairs([0, 100], [0, 100], (1 << 32) + 3) == B.cf_count_pairs([0, 100], [0, 100]) == 5050
    assert B.cf_count_window_pairs([0, 100], [0, 100], 1, 1 << 40) == 5050
    refused(B.CF_EINVAL, "window >= 1", lambda: B.cf_count_window_pairs([0, 1], [0, 1], -(1 << 32) + 5))


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    there = types.SimpleNamespace(device=types.SimpleNamespace(index=1))
    p, paged, append = params(), B.AttnPagedParams(), B.KvAppendParams()
    b = bwd(p)
    b._keepalive, p._keepalive, paged._keepalive, append._keepalive = (p,), (there,), (there,), (there,)
    for call in (lambda: B.cf_attn_window_fwd(p, 8), lambda: B.cf_attn_window_bwd(b, 8), lambda: B.cf_attn_paged_fwd(paged), lambda: B.cf_kv_append(append)):
        with pytest.raises(ValueError, match="cuda:1, the current device is cuda:0"):
            call()


def test_pairs_are_counted():
    rng = np.random.default_rng(3)
    for _ in range(200):
        lq = rng.integers(1, 40, size=rng.integers(1, 5))
        lk = lq + rng.integers(0, 60, size=len(lq)) * rng.integers(0, 2, size=len(lq))
        window, sinks = int(rng.integers(1, 70)), int(rng.integers(0, 50))
        cu_q, cu_k = np.concatenate([[0], np.cumsum(lq)]), np.concatenate([[0], np.cumsum(lk)])
        want = sum(int(W.visible(int(a), int(b), window, sinks).sum()) for a, b in zip(lq, lk))
        assert B.cf_count_window_pairs(cu_q, cu_k, window, sinks) == want
    cu = [0, 5, 9]
    assert B.cf_count_window_pairs(cu, cu, 2**31 - 1, 2**31 - 1) == B.cf_count_pairs(cu, cu)


MASK_CHECK = r"""
#include <cstdio>
#include "mask.h"
using namespace cf;
static bool sees(const WindowMask &m, int p, int j) { return j <= p && (j > p - m.window || j < m.sinks); }
int main()
{
    long n = 0;
    for (int lq = 1; lq <= 21; lq += 4)
        for (int prefix = 0; prefix <= 33; prefix += 11)
            for (int window = 1; window <= lq + prefix; window += 3)
                for (int sinks = 0; sinks <= lq + prefix; sinks += 5) {
                    const WindowMask m = {window, sinks};
                    const int lk = lq + prefix;
                    for (int i = 0; i < lq; ++i) {                   // the keys of a row
                        const KeysOfRow<WindowMask> keys(m, i + prefix);
                        int x = 0;
                        for (int j = 0; j < lk; ++j)
                            if (sees(m, i + prefix, j)) {
                                if (x >= keys.n || keys.key(x) != j) return printf("key %d %d %d %d: %d\n", i + prefix, window, sinks, x, j), 1;
                                ++x;
                            }
                        if (x != keys.n) return printf("keys %d %d %d\n", i + prefix, window, sinks), 1;
                    }
                    for (int r0 = 0; r0 < lq; r0 += 4) {             // the key tiles of some rows: in order, every visible key in one
                        const int r1 = r0 + 4 < lq ? r0 + 4 : lq;
                        const KeyTiles<8, WindowMask> t(m, r0 + prefix, r1 + prefix);
                        for (int a = 0; a < t.n; ++a) {
                            if (t.start(a) < 0 || t.start(a) >= lk || t.start(a) % 8 || (a && t.start(a) <= t.start(a - 1))) return printf("tile\n"), 1;
                            bool any = false;
                            for (int j = t.start(a); j < t.start(a) + 8; ++j)
                                for (int i = r0; i < r1; ++i) any = any || (j < lk && sees(m, i + prefix, j));
                            if (!any) return printf("tile %d of %d %d %d %d is seen by nobody\n", t.start(a), r0 + prefix, r1, window, sinks), 1;
                        }
                        for (int i = r0; i < r1; ++i)
                            for (int j = 0; j < lk; ++j) {
                                bool in = false;
                                for (int a = 0; a < t.n; ++a) in = in || (j >= t.start(a) && j < t.start(a) + 8);
                                if (sees(m, i + prefix, j) && !in) return printf("missing key\n"), 1;
                            }
                    }
                    for (int k0 = 0; k0 < lk; k0 += 8) {             // the query tiles of some keys
                        const int k1 = k0 + 8 < lk ? k0 + 8 : lk;
                        const QueryTiles<4> q(m, k0, k1, prefix, lq);
                        for (int i = 0; i < lq; ++i)
                            for (int j = k0; j < k1; ++j)
                                if (sees(m, i + prefix, j) && (i / 4 < q.first || i / 4 >= q.end)) return printf("missing row\n"), 1;
                        if (q.end > (lq + 3) / 4 || q.first < 0) return printf("rows\n"), 1;
                    }
                    for (int j = 0; j < lk; ++j)
                        for (int i = 0; i < lq; ++i)
                            if (sees(m, i + prefix, j) != (i >= (j > prefix ? j - prefix : 0) && i < rows_that_see(m, j, prefix, lq)))
                                return printf("rows that see\n"), 1;
                    ++n;
                }
    const WindowMask few = {10, 20};                                 // a row far behind the last key that there is: its sinks
    const KeyTiles<16, WindowMask> left(few, 500, 48);
    if (left.n != 2 || left.start(0) != 0 || left.start(1) != 16) return printf("sinks\n"), 1;
    const int far = 0x7fffffff;                                      // the largest sizes leave no 32 bits
    const WindowMask m = {far, far};
    const KeysOfRow<WindowMask> k(m, far - 1);
    const KeyTiles<64, WindowMask> t(m, far - 200, far - 100);
    if (k.n != far || k.key(far - 1) != far - 1 || t.n != (far - 100 + 63) / 64 || rows_that_see(m, far - 1, 0, far) != far) return printf("far\n"), 1;
    printf("%ld\n", n);
    return 0;
}
"""


def test_tiles_of_the_kernels_hold_every_visible_pair(tmp_path):
    src = tmp_path / "mask.cpp"
    src.write_text(MASK_CHECK)
    exe = str(tmp_path / "mask")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2503_02356_amd", "csrc"), str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and int(r.stdout) > 500, r.stdout + r.stderr


def test_formulas_against_differences_and_differentiation():
    g = torch.Generator().manual_seed(1)
    lq, lk, D, window, sinks = 9, 14, 5, 4, 2
    q, d_o = (torch.randn(lq, D, generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn(lk, D, generator=g, dtype=torch.float64) for _ in range(2))
    seen = W.visible(lq, lk, window, sinks)
    assert [int(x) for x in seen.sum(1)] == [6] * lq
    r = W.attention(q, k, v, 0.3, seen, d_o)
    leaves = [x.clone().requires_grad_(True) for x in (q, k, v)]
    s = (leaves[0] @ leaves[1].T * 0.3).masked_fill(~seen, -float("inf"))
    grads = torch.autograd.grad(torch.softmax(s, 1) @ leaves[2], leaves, d_o)
    for name, want in zip(("dq", "dk", "dv"), grads):
        assert torch.allclose(r[name], want, atol=1e-12)
    loss = lambda *x: float((W.attention(*x, 0.3, seen)["o"] * d_o).sum())
    for n, (x, name) in enumerate(zip((q, k, v), ("dq", "dk", "dv"))):
        for at in itertools.product((0, 3, 8), (0, 4)):
            both = []
            for sign in (1e-5, -1e-5):
                y = x.clone()
                y[at] += sign
                both.append(loss(*[y if i == n else z for i, z in enumerate((q, k, v))]))
            assert abs((both[0] - both[1]) / 2e-5 - float(r[name][at])) < 1e-8


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
def test_nothing_else_touches_an_accumulator_of_the_windowed_kernel(tmp_path):
    """As for the kernels without a window (tests/test_build_checks.py): at head_dim 128 its accumulators are updated in place."""
    out = str(tmp_path / "bwd.s")
    subprocess.run([build.HIPCC] + build.HIP_FLAGS + ["-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "attn_mfma_bwd.hip"), "-o", out], check=True, stderr=subprocess.DEVNULL)
    (name, body), = re.findall(r"^(\S*mfma_window_dkv\S*ILi128E\S*):.*?\n(.*?)^\.Lfunc_end", open(out).read(), re.M | re.S)
    n, regs, faults = accumulator_faults(body)
    assert n > 0 and regs == 128 and faults == [], (name, n, regs, faults[:5])


def test_a_spilled_accumulator_of_the_windowed_kernel_fails_the_build():
    report = REPORT.replace("16mfma_dkv_kernel", "23mfma_window_dkv_kernel")
    assert build.spilled_accumulators(report.format(scratch=0, spill=0)) == []
    assert len(build.spilled_accumulators(report.format(scratch=8, spill=2))) == 2
