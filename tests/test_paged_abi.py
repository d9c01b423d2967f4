"""CPU checks of the paged calls: refusals, and that no key that a table or a length asks for lies outside the pages."""
import os
import subprocess

import pytest

from paper_2503_02356_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def paged(**change):
    p = B.AttnPagedParams()
    p.dtype, p.n_q_heads, p.n_kv_heads, p.head_dim, p.softmax_scale, p.n_tokens, p.n_seqs = B.CF_BF16, 4, 2, 128, 0.1, 10, 3
    p.cu_seqlens_q = p.kv_lens = p.block_table = p.lse = 4096
    p.table_stride, p.pages_per_seq, p.page_size, p.n_pages = 8, 8, 64, 20
    p.q = p.k_pages = p.v_pages = p.o = p.workspace = 1 << 20
    p.q_stride_tok = p.o_stride_tok = 512
    p.q_stride_head = p.o_stride_head = p.kv_stride_head = 128
    p.kv_stride_tok, p.page_stride = 256, 64 * 256
    p.workspace_bytes = 1 << 40
    for name, value in change.items():
        setattr(p, name, value)
    return p


def append(**change):
    p = B.KvAppendParams()
    p.dtype, p.n_kv_heads, p.head_dim, p.n_tokens, p.n_seqs = B.CF_BF16, 2, 128, 10, 3
    p.cu_seqlens_q = p.kv_lens = p.block_table = 4096
    p.table_stride, p.pages_per_seq, p.page_size, p.n_pages = 8, 8, 64, 20
    p.k = p.v = p.k_pages = p.v_pages = 1 << 20
    p.kv_stride_tok, p.kv_stride_head, p.page_stride, p.page_stride_tok, p.page_stride_head = 256, 128, 64 * 256, 256, 128
    for name, value in change.items():
        setattr(p, name, value)
    return p


COMMON = [("dtype", 2, B.CF_EUNSUPPORTED), ("head_dim", 96, B.CF_EUNSUPPORTED), ("n_tokens", 0, B.CF_EINVAL), ("n_seqs", 0, B.CF_EINVAL),
          ("page_size", 8, B.CF_EINVAL), ("page_size", 48, B.CF_EINVAL), ("page_size", 1 << 17, B.CF_EINVAL), ("page_size", -64, B.CF_EINVAL),
          ("n_pages", 0, B.CF_EINVAL), ("pages_per_seq", 0, B.CF_EINVAL), ("pages_per_seq", 9, B.CF_EINVAL), ("table_stride", 7, B.CF_EINVAL),
          ("cu_seqlens_q", None, B.CF_EINVAL), ("kv_lens", None, B.CF_EINVAL), ("block_table", None, B.CF_EINVAL), ("kv_lens", 4098, B.CF_EINVAL),
          ("k_pages", None, B.CF_EINVAL), ("v_pages", 24, B.CF_EINVAL), ("page_stride", 100, B.CF_EINVAL), ("kv_stride_tok", 260, B.CF_EINVAL)]


def refused(code, call, p):
    with pytest.raises(B.CfError) as e:
        call(p, stream=0)
    assert e.value.code == code and call.__name__ in str(e.value), e.value


@pytest.mark.parametrize("name,value,code", COMMON + [
    ("n_q_heads", 5, B.CF_EINVAL), ("n_kv_heads", 0, B.CF_EINVAL), ("n_tokens", 1 << 30, B.CF_EINVAL), ("flags", 2, B.CF_EINVAL),
    ("max_kv_len", -1, B.CF_EINVAL), ("window", -1, B.CF_EINVAL), ("n_sinks", 1, B.CF_EINVAL), ("n_sinks", -1, B.CF_EINVAL),
    ("softmax_scale", float("nan"), B.CF_EINVAL), ("softmax_scale", float("inf"), B.CF_EINVAL), ("q", None, B.CF_EINVAL), ("o", 8, B.CF_EINVAL),
    ("q_stride_head", 64, B.CF_EINVAL), ("o_stride_tok", 516, B.CF_EINVAL), ("lse", 4098, B.CF_EINVAL)])
def test_attention_refuses(name, value, code):
    refused(code, B.cf_attn_paged_fwd, paged(**{name: value}))
    assert B.lib().cf_attn_paged_fwd(None, None) == B.CF_EINVAL and B.lib().cf_attn_paged_workspace_bytes(None) == B.CF_EINVAL


@pytest.mark.parametrize("name,value,code", COMMON + [("n_kv_heads", 0, B.CF_EINVAL), ("k", None, B.CF_EINVAL), ("v", 8, B.CF_EINVAL),
                                                      ("page_stride_head", 4, B.CF_EINVAL), ("page_stride_tok", 12, B.CF_EINVAL)])
def test_append_refuses(name, value, code):
    refused(code, B.cf_kv_append, append(**{name: value}))
    assert B.lib().cf_kv_append(None, None) == B.CF_EINVAL


def test_too_many_columns_are_refused():
    refused(B.CF_EINVAL, B.cf_attn_paged_fwd, paged(pages_per_seq=1 << 26, table_stride=1 << 26))
    refused(B.CF_EINVAL, B.cf_kv_append, append(pages_per_seq=1 << 26, table_stride=1 << 26))


def test_workspace_sizes_need_no_pointers():
    p = paged(cu_seqlens_q=None, kv_lens=None, block_table=None, q=None, k_pages=None, v_pages=None, o=None, workspace=None)
    assert B.cf_attn_paged_workspace_bytes(p) >= 0


PAGES = r"""
#include <climits>
#include <initializer_list>
#include <cstdio>
#include "pages.h"
using namespace cf;
int main()
{
    const int32_t entries[] = {0, 3, -1, 5, INT_MAX, 4, INT_MIN, 1};     // 5 pages: some are none
    const int want[] = {0, 3, -1, -1, -1, 4, -1, 1};
    for (int shift = 4; shift <= 16; shift += 3) {
        const PageTable t{entries, 8, shift, 5};
        const int n = 1 << shift;
        for (int x = 0; x < 8; ++x)
            for (int r : {0, 1, n / 2, n - 1})
                if (t.page_of(x * n + r) != want[x] || t.row_in_page(x * n + r) != r) return std::printf("page %d row %d\n", x, r), 1;
        for (int j : {-1, INT_MIN, 8 * n, 8 * n + 1, INT_MAX})
            if (t.page_of(j) != -1) return std::printf("key %d\n", j), 1;
        if (t.capacity() != 8 * n) return 1;
    }
    for (int lq : {0, 1, 5, INT_MAX})
        for (int kv : {INT_MIN, -1, 0, 3, INT_MAX}) {
            const NewRows r(0, lq, kv);
            const long long first = (kv < 0 ? 0 : (long long)kv) - lq;
            for (int i : {0, lq / 2, lq - 1})
                if (i >= 0 && r.position(i) != (first + i < -1 ? -1 : first + i)) return std::printf("position %d of %d, %d keys\n", i, lq, kv), 1;
        }
    return 0;
}
"""


def test_no_key_lies_outside_the_pages(tmp_path):
    src = tmp_path / "pages.cpp"
    src.write_text(PAGES)
    exe = str(tmp_path / "pages")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2503_02356_amd", "csrc"), str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
