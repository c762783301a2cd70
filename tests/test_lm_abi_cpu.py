"""include/vla_lm.h: every declared symbol is exported, and argument errors come back before any launch."""
import os
import re

import pytest

from paper_2505_18719_gb300 import build as B
from paper_2505_18719_gb300 import vla as V

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return V.load()


def test_every_declared_symbol_is_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vla_lm.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(vla_[a-z0-9_]+)\s*\(", src)))
    assert names == ["vla_page_plan", "vla_paged_attn", "vla_paged_attn_workspace_bytes", "vla_rope_append", "vla_rope_table",
                     "vla_token_logprobs", "vla_token_logprobs_grad"]
    for n in names:
        assert hasattr(lib, n), n


def refused(rc, code, name):
    assert rc == code and name in V.vla_last_error(), (rc, V.vla_last_error())


def plan(**kw):
    a = dict(ctx_in_ptr=16, new_len_ptr=16, release_ptr=0, n_env=2, page_size=16, table_ptr=16, max_pages=4, pool_ptr=16, n_pages=8,
             n_free_in_ptr=16, ctx_out_ptr=16, n_free_out_ptr=16, row_start_ptr=16, row_env_ptr=16, row_pos_ptr=16, row_slot_ptr=16,
             max_rows=8)
    a.update(kw)
    return V.vla_page_plan(**a)


@pytest.mark.parametrize("name", ["ctx_in_ptr", "new_len_ptr", "table_ptr", "pool_ptr", "n_free_in_ptr", "ctx_out_ptr", "n_free_out_ptr",
                                  "row_start_ptr", "row_env_ptr", "row_pos_ptr", "row_slot_ptr", "n_env", "page_size", "max_pages", "n_pages"])
def test_page_plan_refuses_nothing_where_something_is_due(name):
    refused(plan(**{name: 0}), V.VLA_ERR_ARG, "vla_page_plan")


def test_page_plan_refusals():
    refused(plan(max_rows=-1), V.VLA_ERR_ARG, "vla_page_plan")
    refused(plan(n_env=-3), V.VLA_ERR_ARG, "vla_page_plan")
    refused(plan(n_pages=1 << 20, page_size=1 << 11), V.VLA_ERR_ARG, "2^31")
    refused(plan(n_env=4097), V.VLA_ERR_UNSUPPORTED, "4096")


def test_rope_table_refusals():
    t = lambda *a, **k: V.vla_rope_table(*a, **k)  # noqa: E731
    refused(t(0, 4, 64, 1e4), V.VLA_ERR_ARG, "vla_rope_table")
    refused(t(16, 0, 64, 1e4), V.VLA_ERR_ARG, "vla_rope_table")
    refused(t(16, 4, 63, 1e4), V.VLA_ERR_ARG, "vla_rope_table")
    refused(t(16, 4, 64, 0.0), V.VLA_ERR_ARG, "vla_rope_table")
    refused(t(16, 4, 64, float("nan")), V.VLA_ERR_ARG, "vla_rope_table")
    refused(t(16, 4, 64, 1e4, 4), V.VLA_ERR_UNSUPPORTED, "vla_rope_table")
    refused(t(16, 4, 64, 1e4, V.VLA_ROPE_LINEAR, 0.5), V.VLA_ERR_ARG, "factor")
    refused(t(16, 4, 64, 1e4, V.VLA_ROPE_TURNS, 4.0, 0.0, 1.0, 4.0), V.VLA_ERR_ARG, "original_len")
    refused(t(16, 4, 64, 1e4, V.VLA_ROPE_LOG_TURNS, 4.0, 4096.0, 4.0, 4.0), V.VLA_ERR_ARG, "low < high")
    refused(t(16, 4, 64, 1e4, amplitude=0.0), V.VLA_ERR_ARG, "vla_rope_table")


def cache(**kw):
    a = dict(k=16, v=16, dtype=V.VLA_F16, n_pages=8, page_size=16, n_heads=2, head_dim=64, page_stride=2048, head_stride=1024,
             slot_stride=64)
    a.update(kw)
    return V.VlaPagedKv(*a.values())


BAD_CACHES = [(dict(k=0), V.VLA_ERR_ARG), (dict(v=0), V.VLA_ERR_ARG), (dict(k=24), V.VLA_ERR_ARG), (dict(v=18), V.VLA_ERR_ARG),
              (dict(n_pages=0), V.VLA_ERR_ARG), (dict(page_size=-1), V.VLA_ERR_ARG), (dict(n_heads=0), V.VLA_ERR_ARG),
              (dict(page_stride=2052), V.VLA_ERR_ARG), (dict(slot_stride=-64), V.VLA_ERR_ARG), (dict(head_stride=1), V.VLA_ERR_ARG),
              (dict(n_pages=1 << 28), V.VLA_ERR_ARG), (dict(dtype=V.VLA_F32), V.VLA_ERR_UNSUPPORTED),
              (dict(dtype=7), V.VLA_ERR_UNSUPPORTED), (dict(head_dim=96), V.VLA_ERR_UNSUPPORTED)]


def append(kv=None, **kw):
    a = dict(q_ptr=16, ldq=512, k_ptr=16, ldk=512, v_ptr=16, ldv=512, dtype=V.VLA_F16, rows=4, n_q_heads=4, kv=kv or cache(), q_gain_ptr=0,
             k_gain_ptr=0, eps=1e-6, rope_ptr=16, n_pos=10, rope_dim=64, interleaved=0, row_pos_ptr=16, row_slot_ptr=16, q_out_ptr=16,
             ldqo=512)
    a.update(kw)
    return V.vla_rope_append(**a)


def attend(kv=None, **kw):
    a = dict(q_ptr=16, ldq=256, dtype=V.VLA_F16, rows=4, n_q_heads=4, kv=kv or cache(), table_ptr=16, max_pages=4, n_env=2, row_env_ptr=16,
             row_pos_ptr=16, scale=0.1, out_ptr=16, ldo=256, lse_ptr=0, ws_ptr=16, ws_bytes=1 << 30)
    a.update(kw)
    return V.vla_paged_attn(**a)


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_cache_descriptors_that_are_refused(change, code):
    refused(append(cache(**change)), code, "vla_rope_append")
    refused(attend(cache(**change)), code, "vla_paged_attn")


@pytest.mark.parametrize("change", [dict(q_ptr=0), dict(k_ptr=0), dict(v_ptr=0), dict(q_out_ptr=0), dict(row_pos_ptr=0), dict(row_slot_ptr=0),
                                    dict(q_ptr=8), dict(ldq=248), dict(ldk=120), dict(ldv=130), dict(ldqo=516), dict(rows=-1),
                                    dict(n_q_heads=0), dict(q_gain_ptr=8), dict(k_gain_ptr=2), dict(eps=-1.0), dict(eps=float("nan")),
                                    dict(rope_ptr=8), dict(rope_dim=24), dict(rope_dim=80), dict(rope_dim=0), dict(n_pos=0),
                                    dict(ldqo=256)])
def test_rope_append_refusals(change):
    refused(append(**change), V.VLA_ERR_ARG, "vla_rope_append")


def test_rope_append_types_and_no_rows():
    refused(append(dtype=3), V.VLA_ERR_UNSUPPORTED, "vla_rope_append")
    assert append(rows=0) == V.VLA_OK
    assert V.load().vla_rope_append(None, 0, None, 0, None, 0, 0, 1, 1, None, None, None, 0.0, None, 0, 0, 0, None, None, None, 0,
                                    None) == V.VLA_ERR_ARG


@pytest.mark.parametrize("change", [dict(q_ptr=0), dict(out_ptr=0), dict(table_ptr=0), dict(row_env_ptr=0), dict(row_pos_ptr=0), dict(ws_ptr=0),
                                    dict(ws_ptr=8), dict(ws_bytes=8), dict(rows=-1), dict(n_q_heads=3), dict(n_q_heads=0), dict(ldq=128),
                                    dict(ldo=260), dict(max_pages=0), dict(n_env=0), dict(scale=float("inf")), dict(out_ptr=20)])
def test_paged_attn_refusals(change):
    refused(attend(**change), V.VLA_ERR_ARG, "vla_paged_attn")


def test_paged_attn_types_workspace_and_no_rows():
    refused(attend(dtype=V.VLA_BF16), V.VLA_ERR_UNSUPPORTED, "vla_paged_attn")
    refused(attend(cache(dtype=V.VLA_BF16), dtype=V.VLA_F32), V.VLA_ERR_UNSUPPORTED, "vla_paged_attn")
    assert attend(rows=0) == V.VLA_OK
    assert V.vla_paged_attn_workspace_bytes(64) >= 16 and V.vla_paged_attn_workspace_bytes(128) >= 16
    assert V.vla_paged_attn_workspace_bytes(96) == 0


def logprobs(**kw):
    a = dict(logits_ptr=16, ld=100, dtype=V.VLA_F32, rows=2, vocab=100, tokens_ptr=16, temperature=1.0, top_k=2, logprob_ptr=16, entropy_ptr=16,
             lse_ptr=16, top_ids_ptr=16, top_logprobs_ptr=16)
    a.update(kw)
    return V.vla_token_logprobs(**a)


@pytest.mark.parametrize("change", [dict(logits_ptr=0), dict(logits_ptr=18), dict(ld=99), dict(rows=-1), dict(vocab=0), dict(temperature=-1.0),
                                    dict(temperature=float("nan")), dict(top_k=-1), dict(vocab=1, ld=1), dict(top_ids_ptr=0),
                                    dict(top_logprobs_ptr=0), dict(tokens_ptr=0)])
def test_token_logprobs_refusals(change):
    refused(logprobs(**change), V.VLA_ERR_ARG, "vla_token_logprobs")


def test_token_logprobs_unsupported_and_no_rows():
    refused(logprobs(dtype=3), V.VLA_ERR_UNSUPPORTED, "vla_token_logprobs")
    refused(logprobs(top_k=33), V.VLA_ERR_UNSUPPORTED, "32")
    assert logprobs(rows=0) == V.VLA_OK


def grad(**kw):
    a = dict(logits_ptr=16, ld=100, dtype=V.VLA_BF16, rows=2, vocab=100, tokens_ptr=16, temperature=1.0, lse_ptr=16, entropy_ptr=16,
             g_logprob_ptr=16, g_entropy_ptr=16, d_logits_ptr=32, ldd=100)
    a.update(kw)
    return V.vla_token_logprobs_grad(**a)


@pytest.mark.parametrize("change", [dict(logits_ptr=0), dict(logits_ptr=17), dict(d_logits_ptr=33), dict(ld=99), dict(ldd=99), dict(rows=-1),
                                    dict(vocab=0), dict(temperature=float("inf")), dict(tokens_ptr=0), dict(lse_ptr=0), dict(entropy_ptr=0),
                                    dict(g_logprob_ptr=0), dict(d_logits_ptr=0), dict(d_logits_ptr=16, ldd=104)])
def test_token_logprobs_grad_refusals(change):
    refused(grad(**change), V.VLA_ERR_ARG, "vla_token_logprobs_grad")


def test_token_logprobs_grad_unsupported_and_no_rows():
    refused(grad(dtype=-1), V.VLA_ERR_UNSUPPORTED, "vla_token_logprobs_grad")
    assert grad(rows=0) == V.VLA_OK


def test_counts_whose_arithmetic_would_pass_32_bits():
    many = (1 << 30) + 1
    refused(attend(cache(n_heads=1), n_q_heads=1, ldq=128, ldo=128, rows=many), V.VLA_ERR_UNSUPPORTED, "2^30")
    refused(logprobs(vocab=many, ld=many), V.VLA_ERR_UNSUPPORTED, "2^30")
    refused(grad(vocab=many, ld=many, ldd=many), V.VLA_ERR_UNSUPPORTED, "2^30")
