"""The paged key/value cache without a GPU: refusals of the entry points (checked
before any device work), the bounds that the kernels check (the same inline
functions, compiled for the host), and the oracle against hand-made values."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import oracle.paged as op
import paper_2608_03682_amd as px
from oracle.numerics import attention, rope

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                # a pointer that is never followed: 16-byte aligned, not NULL
EINVAL = px.PHYAI_EINVAL


def cache(**kw):
    c = dict(k=P, v=P, k_scale=None, v_scale=None, page_table=P, layer_stride=1 << 20, page_stride=64 * 256,
             token_stride=256, head_stride=128, dtype=1, n_layers=2, n_kv_heads=2, head_dim=128, page_size=64,
             n_pages=10, batch=3, max_pages=4, table_stride=4)
    c.update(kw)
    return px._PagedCache(*[c[f] for f, _ in px._PagedCache._fields_])


def rows(heads, data=P, b=4096, t=1024, h=128):
    return px._HeadRows(data, b, t, h, heads)


def attend(c=None, layer=0, q=None, out=None, kv=P, new=None, max_kv=256, scale=0.1, causal=1, window=0, M=4, dtype=1,
           ws=P, ws_bytes=1 << 40):
    r = ctypes.byref
    return px.lib().phyai_paged_attention(r(c or cache()), layer, r(q or rows(8)), r(out or rows(8)), kv, new, max_kv,
                                          scale, causal, window, M, dtype, ws, ws_bytes, None, None)


def refused(rc, needle):
    assert rc == EINVAL
    assert needle in px.lib().phyai_last_error().decode()


CACHE_FAULTS = [
    (dict(k=None), "NULL"), (dict(page_table=None), "NULL"), (dict(k=P + 8), "aligned"), (dict(page_table=P + 2), "aligned"),
    (dict(dtype=3), "dtype"), (dict(dtype=2), "k_scale"), (dict(head_dim=96), "head_dim"), (dict(page_size=48), "page_size"),
    (dict(page_size=8), "page_size"), (dict(page_size=8192), "page_size"), (dict(n_pages=0), "n_pages"),
    (dict(max_pages=0), "max_pages"), (dict(table_stride=3), "table_stride"), (dict(n_layers=0), "n_layers"),
    (dict(n_kv_heads=0), "n_kv_heads"), (dict(batch=0), "batch"), (dict(batch=4097), "batch"),
    (dict(token_stride=-256), "strides"), (dict(page_stride=64 * 256 + 4), "strides"), (dict(token_stride=64), "overlap"),
    (dict(head_stride=0), "overlap"), (dict(max_pages=1 << 25, table_stride=1 << 25), "2^30 tokens"),
    (dict(token_stride=1 << 24), "2^30 bytes"),
]


@pytest.mark.parametrize("kw,needle", CACHE_FAULTS)
def test_a_bad_cache_is_refused_everywhere(kw, needle):
    L, r, c = px.lib(), ctypes.byref, cache(**kw)
    refused(attend(c), needle)
    refused(L.phyai_paged_append(r(c), 0, r(rows(2)), r(rows(2)), 0.0, P, None, 4, 1, None, None), needle)
    refused(L.phyai_paged_gather(r(c), P, P, 16, None, None), needle)
    assert L.phyai_paged_attention_workspace(r(c), 8, 4, 64) == EINVAL


@pytest.mark.parametrize("kw,needle", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(q=rows(7)), "number of heads"), (dict(q=rows(7), out=rows(7)), "multiple"),
    (dict(q=rows(8, data=None)), "NULL"), (dict(q=rows(8, data=P + 4)), "aligned"), (dict(q=rows(8, t=1022)), "strides"),
    (dict(q=rows(8, h=-128)), "strides"), (dict(out=rows(8, t=0)), "overlap"), (dict(out=rows(8, h=64)), "overlap"), (dict(kv=None), "kv_len"),
    (dict(max_kv=0), "max_kv_len"), (dict(max_kv=257), "max_kv_len"), (dict(scale=0.0), "scale"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"),
    (dict(causal=2), "causal"), (dict(window=-1), "window"), (dict(causal=0, window=4), "window"), (dict(M=0), "rows"),
    (dict(M=(1 << 20) + 1), "rows"), (dict(dtype=0), "F32 rows"), (dict(dtype=2), "F32 or BF16"),
])
def test_attention_refuses(kw, needle):
    refused(attend(**kw), needle)


@pytest.mark.parametrize("kw", [dict(ws=None), dict(ws=P + 4), dict(ws_bytes=16)])
def test_attention_refuses_a_workspace_that_a_split_cannot_use(kw):
    long = cache(batch=1, max_pages=4096, table_stride=4096)
    refused(attend(long, max_kv=4096 * 64, M=1, **kw), "workspace")


def test_append_and_gather_refuse():
    L, r, c = px.lib(), ctypes.byref, cache()

    def app(k=rows(2), v=rows(2), base=0.0, past=P, M=4, dtype=1, layer=0):
        return L.phyai_paged_append(r(c), layer, r(k), r(v), base, past, None, M, dtype, None, None)

    for kw, needle in [(dict(k=rows(3)), "n_kv_heads"), (dict(v=rows(1)), "n_kv_heads"), (dict(base=0.5), "rope_base"),
                       (dict(base=float("nan")), "rope_base"), (dict(past=None), "past_len"), (dict(M=0), "rows"),
                       (dict(dtype=0), "F32 rows"), (dict(layer=2), "layer"), (dict(v=rows(2, data=P + 8)), "aligned")]:
        refused(app(**kw), needle)
    refused(L.phyai_paged_gather(r(c), None, P, 16, None, None), "NULL")
    refused(L.phyai_paged_gather(r(c), P, P + 4, 16, None, None), "aligned")
    refused(L.phyai_paged_gather(r(c), P, P, 0, None, None), "rows")
    refused(L.phyai_paged_gather(r(cache(n_layers=1000, batch=4096)), P, P, 16, None, None), "n_layers * 2 * batch")


def test_norm_rope_refuses():
    L, r = px.lib(), ctypes.byref

    def nr(q=rows(8), k=rows(2), qo=rows(8), ko=rows(2), qg=P, kg=None, eps=1e-6, base=1e4, B=2, M=4, D=128, dtype=1):
        p = lambda x: None if x is None else r(x)  # noqa: E731
        return L.phyai_qk_norm_rope(p(q), p(k), p(qo), p(ko), qg, kg, eps, base, None, None, B, M, D, dtype, None, None)

    for kw, needle in [(dict(q=None, k=None, qg=None), "both NULL"), (dict(qo=None), "q_out"), (dict(ko=rows(3)), "number of heads"),
                       (dict(eps=-1.0), "eps"), (dict(eps=0.0), "gains need"), (dict(eps=0.0, base=0.0, qg=None), "nothing to do"),
                       (dict(eps=float("nan")), "eps"), (dict(base=0.9), "rope_base"), (dict(base=float("inf")), "rope_base"),
                       (dict(qg=P + 4), "gains"), (dict(k=None, kg=P), "without its rows"), (dict(B=0), "batch"), (dict(D=32), "head_dim"),
                       (dict(dtype=2), "F32 or BF16"), (dict(qo=rows(8, t=0)), "overlap"), (dict(ko=rows(2, b=0)), "overlap"),
                       (dict(B=4096, M=1 << 20), "batch * rows")]:
        refused(nr(**kw), needle)


def test_more_tokens_than_a_launch_holds_are_refused():
    """One block of 256 threads for every two tokens at least, and a launch has fewer than 2^32 threads."""
    L, r, wide = px.lib(), ctypes.byref, (1 << 24) // 32 + 1
    many = rows(2, b=1 << 30)
    refused(L.phyai_qk_norm_rope(r(many), None, r(many), None, None, None, 0.0, 1e4, P, None, 32, wide, 128, 1, None, None),
            "batch * rows")
    refused(L.phyai_paged_append(r(cache(batch=32)), 0, r(many), r(many), 0.0, P, None, wide, 1, None, None), "batch * rows")


def test_misaligned_words_are_refused():
    """Lengths, scales and the status word (an atomic on a misaligned word faults)."""
    L, r, odd = px.lib(), ctypes.byref, P + 2
    refused(attend(kv=odd), "4-byte")
    refused(attend(new=odd), "4-byte")
    refused(attend(cache(dtype=2, k_scale=odd, v_scale=P)), "4-byte")
    refused(L.phyai_paged_attention(r(cache()), 0, r(rows(8)), r(rows(8)), P, None, 256, 0.1, 1, 0, 4, 1, P, 1 << 40, odd, None), "4-byte")
    refused(L.phyai_paged_append(r(cache()), 0, r(rows(2)), r(rows(2)), 0.0, odd, None, 4, 1, None, None), "4-byte")
    refused(L.phyai_paged_append(r(cache()), 0, r(rows(2)), r(rows(2)), 0.0, P, None, 4, 1, odd, None), "4-byte")
    refused(L.phyai_paged_gather(r(cache()), P, P, 16, odd, None), "4-byte")
    refused(L.phyai_qk_norm_rope(r(rows(8)), None, r(rows(8)), None, None, None, 1e-6, 1e4, None, None, 2, 4, 128, 1, odd, None), "4-byte")


def test_workspace_depends_on_the_split_alone():
    L, r = px.lib(), ctypes.byref
    # a chip full of rows: no split; one row over many keys: split
    assert L.phyai_paged_attention_workspace(r(cache(batch=512, n_kv_heads=2)), 8, 512, 256) == 0
    one = cache(batch=1, max_pages=4096, table_stride=4096)
    n = L.phyai_paged_attention_workspace(r(one), 8, 1, 4096 * 64)
    assert n > 0 and n % (2 * 4 * 130 * 4) == 0          # K/V heads x rows x (128 values, maximum, sum) x splits
    assert L.phyai_paged_attention_workspace(r(one), 8, 1, 4096 * 64) == n
    assert L.phyai_paged_attention_workspace(None, 8, 1, 64) == EINVAL
    assert L.phyai_paged_attention_workspace(r(one), 7, 1, 64) == EINVAL


HOST = r"""
#include "paged.hpp"
#include <cstdio>
#include <cstdlib>
using namespace phyai;
#define CHECK(x) do { if (!(x)) { std::printf("%d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  for (int n : {1, 7, 1 << 30, INT32_MAX}) {
    for (int64_t p : {int64_t(INT32_MIN), int64_t(-2), int64_t(-1), int64_t(n), int64_t(n) + 1, int64_t(INT32_MAX)})
      CHECK(page_ok((int32_t)p, n) == (p >= 0 && p < n));
    CHECK(page_ok(0, n) && page_ok(n - 1, n));
  }
  // whatever the device holds, what a kernel uses lies inside the host's bounds
  for (int n : {INT32_MIN, -1, 0, 1, 5, 6, INT32_MAX})
    for (int past : {INT32_MIN, -1, 0, 95, 96, 100, INT32_MAX}) {
      const RowSpan s = row_span(n, past, 5, 100);
      CHECK(s.ok == (n >= 0 && n <= 5 && past >= 0 && (int64_t)past + n <= 100));
      CHECK(s.n >= 0 && s.n <= 5 && s.past >= 0);
      if (s.ok) CHECK(s.n == n && s.past == past && s.past + s.n <= 100);
    }
  for (int kv = 0; kv < 9; ++kv)
    for (int n = 1; n < 9; ++n)
      for (int t = 0; t < n; ++t)
        for (int w = 0; w < 5; ++w)
          for (int causal = 0; causal < 2; ++causal) {
            const int lo = seen_begin(t, n, kv, causal ? w : 0), hi = seen_end(t, n, kv, causal);
            CHECK(lo >= 0 && hi >= 0 && hi <= kv);
            for (int j = 0; j < kv; ++j) {
              const int pos = kv - n + t;
              const bool see = !causal || (j <= pos && (!w || j > pos - w));
              CHECK(see == (j >= lo && j < hi));
            }
          }
  CHECK(seen_begin(0, 1, 100, INT32_MAX) == 0);
  PagePool p{};
  p.page_bytes = int64_t(1) << 33; p.token_bytes = 4096; p.head_bytes = 512; p.page_shift = 6;
  CHECK(page_row_offset(p, 5, 64 * 7 + 63, 3) == 5 * (int64_t(1) << 33) + 63 * 4096 + 3 * 512);
  std::puts("ok");
  return 0;
}
"""


def test_the_kernels_bounds_on_the_host(tmp_path):
    src, exe = tmp_path / "b.cpp", tmp_path / "b"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" +
                    os.path.join(ROOT, "paper_2608_03682_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_oracle_attention_is_the_pinned_attention_over_gathered_pages():
    rng = np.random.default_rng(3)
    ps, nkv, D, H = 16, 2, 8, 4
    kp, vp = rng.standard_normal((2, 7, ps, nkv, D))
    table = np.array([[5, 0, 3], [6, 2, -1]])
    kv, new = [37, 20], [5, 3]
    q = rng.standard_normal((2, 5, H, D))
    o, _ = op.paged_attention(q, kp, vp, table, kv, new, np.full(q.shape, 7.0))
    for b in range(2):
        k, v = op.tokens_of(kp, table[b], kv[b]), op.tokens_of(vp, table[b], kv[b])
        assert (k[17] == kp[table[b][1], 1]).all()
        n = new[b]
        want = attention(q[b, :n], k, v, op.visible(n, kv[b]))
        np.testing.assert_allclose(o[b, :n], want, rtol=1e-12, atol=1e-12)
    assert (o[1, 3:] == 7.0).all()
    # the last row of a causal chunk sees all, a window of one sees itself alone
    w, _ = op.paged_attention(q, kp, vp, table, kv, new, np.zeros(q.shape), window=1)
    np.testing.assert_allclose(w[0, 4, 3], op.tokens_of(vp, table[0], 37)[36, 1], rtol=1e-12)
    # more rows than keys: the first of them see none
    z, _ = op.paged_attention(q, kp, vp, table, [2, 2], [5, 3], np.full(q.shape, 7.0))
    assert (z[0, :3] == 0).all() and (z[0, 3:] != 0).all()


def test_oracle_append_then_gather():
    rng = np.random.default_rng(4)
    pool, x = rng.standard_normal((4, 16, 1, 8)), rng.standard_normal((1, 20, 1, 8))
    table = np.array([[2, 0, 1]])
    got = op.paged_append(pool, table, x, [10], [20], 1e4)
    g = op.paged_gather(got, got, table, [30], 33)
    np.testing.assert_allclose(g[0, 0, 10:30], rope(x[0], 10 + np.arange(20), 1e4).reshape(20, 8), rtol=1e-12)
    assert (g[0, 0, :10] == pool[2, :10, 0]).all() and (g[:, :, 30:] == 0).all()
    assert (got[3] == pool[3]).all() and (got[0, 14:] == pool[0, 14:]).all()


def test_oracle_chunks_are_the_prefix_block_and_the_causal_model():
    """One chunk without a causal mask is the pinned prefix LM; causal chunks do not depend
    on where they are cut; a later chunk leaves the earlier ones as they were."""
    import oracle
    import workloads as wl
    cfg = wl.CONFIGS["plm_tiny_fp32"]
    case = wl.make_prefill_case(cfg, seed=3)
    n = 24
    x = np.asarray(case.embeds[0, :n], dtype=np.float64)
    one = op.prefill_chunks(cfg, case.weights, x, [n], [False])
    np.testing.assert_allclose(one, oracle.prefill_request(cfg, case.weights, x), rtol=1e-10, atol=1e-12)
    a = op.prefill_chunks(cfg, case.weights, x, [n], [True])
    b = op.prefill_chunks(cfg, case.weights, x, [9, 1, 14], [True] * 3)
    np.testing.assert_allclose(a, b, rtol=1e-10, atol=1e-12)
    c = op.prefill_chunks(cfg, case.weights, x, [9, 15], [False, True])
    np.testing.assert_allclose(c[:, :, :9], oracle.prefill_request(cfg, case.weights, x[:9]), rtol=1e-10, atol=1e-12)
    assert np.abs(c - a).max() > 1e-4 and np.abs(c - one).max() > 1e-4


def test_prefill_paged_refuses_without_a_handle():
    assert px.lib().phyai_prefill_paged(None, P, ctypes.byref(cache()), None, None, 4, 0, None, 0, None, None) == EINVAL
    assert b"NULL handle" in px.lib().phyai_last_error()
