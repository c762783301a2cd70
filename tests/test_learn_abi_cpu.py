"""include/vla_learn.h: every declared symbol is exported, and argument errors come back before any launch."""
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
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vla_learn.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(vla_[a-z0-9_]+)\s*\(", src)))
    assert names == ["vla_block_norm", "vla_block_norm_grad", "vla_block_norm_grad_workspace_bytes", "vla_prompt_attn", "vla_prompt_attn_grad",
                     "vla_prompt_attn_grad_workspace_bytes"]
    for n in names:
        assert hasattr(lib, n), n


def refused(rc, code, name):
    assert rc == code and name in V.vla_last_error(), (rc, V.vla_last_error())


def attend(**kw):
    a = dict(q_ptr=16, ldq=512, k_ptr=16, ldk=512, v_ptr=16, ldv=512, dtype=V.VLA_F16, rows=4, n_q_heads=4, n_kv_heads=2, head_dim=64,
             seq_start_ptr=16, n_seq=2, scale=0.1, out_ptr=16, ldo=256, lse_ptr=0)
    a.update(kw)
    return V.vla_prompt_attn(**a)


def attend_grad(**kw):
    a = dict(q_ptr=16, ldq=512, k_ptr=16, ldk=512, v_ptr=16, ldv=512, dtype=V.VLA_F16, rows=4, n_q_heads=4, n_kv_heads=2, head_dim=64,
             seq_start_ptr=16, n_seq=2, scale=0.1, out_ptr=16, ldo=256, lse_ptr=16, d_out_ptr=16, lddo=256, d_q_ptr=32, lddq=512, d_k_ptr=32,
             lddk=512, d_v_ptr=32, lddv=512, ws_ptr=16, ws_bytes=1 << 30)
    a.update(kw)
    return V.vla_prompt_attn_grad(**a)


BOTH = [dict(q_ptr=0), dict(k_ptr=0), dict(v_ptr=0), dict(out_ptr=0), dict(seq_start_ptr=0), dict(seq_start_ptr=18), dict(q_ptr=8), dict(k_ptr=24),
        dict(v_ptr=18), dict(out_ptr=20), dict(ldq=248), dict(ldk=120), dict(ldv=130), dict(ldo=250), dict(ldo=260), dict(rows=-1), dict(n_q_heads=0),
        dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=8), dict(n_seq=0), dict(n_seq=-1), dict(scale=0.0), dict(scale=1e-31), dict(scale=-1.0),
        dict(scale=float("nan")), dict(scale=float("inf")), dict(lse_ptr=18)]


@pytest.mark.parametrize("change", BOTH)
def test_prompt_attn_refusals(change):
    refused(attend(**change), V.VLA_ERR_ARG, "vla_prompt_attn")


@pytest.mark.parametrize("change", BOTH + [dict(lse_ptr=0), dict(d_out_ptr=0), dict(d_q_ptr=0), dict(d_k_ptr=0), dict(d_v_ptr=0), dict(d_out_ptr=8),
                                           dict(d_q_ptr=40), dict(lddo=248), dict(lddq=260), dict(lddk=64), dict(lddv=132), dict(ws_ptr=0),
                                           dict(ws_ptr=8), dict(ws_bytes=8)])
def test_prompt_attn_grad_refusals(change):
    refused(attend_grad(**change), V.VLA_ERR_ARG, "vla_prompt_attn_grad")


@pytest.mark.parametrize("call,name", [(attend, "vla_prompt_attn"), (attend_grad, "vla_prompt_attn_grad")])
def test_prompt_attn_what_is_not_supported_and_no_rows(call, name):
    for change in (dict(dtype=V.VLA_F32), dict(dtype=7), dict(head_dim=96), dict(head_dim=256), dict(rows=1 << 29),
                   dict(n_q_heads=1 << 17, n_kv_heads=1, ldq=1 << 24, ldo=1 << 24)):
        refused(call(**change), V.VLA_ERR_UNSUPPORTED, name)
    assert call(rows=0) == V.VLA_OK
    assert call(rows=0, q_ptr=0, seq_start_ptr=0) == V.VLA_OK


def test_prompt_attn_grad_workspace_sizes():
    f = V.vla_prompt_attn_grad_workspace_bytes
    assert f(10, 4, 2, 64) >= 10 * 4 * 4
    for bad in ((-1, 4, 2, 64), (10, 4, 3, 64), (10, 0, 1, 64), (10, 4, 2, 32), (1 << 29, 4, 2, 64)):
        assert f(*bad) == 0


def norm(**kw):
    a = dict(y_ptr=16, ldy=64, dtype=V.VLA_BF16, h_ptr=16, ldh=64, h_dtype=V.VLA_F32, rows=3, dim=64, post_gain_ptr=16, gate_ptr=16, ldg=64,
             residual_scale=1.0, pre_gain_ptr=16, eps=1e-6, h_out_ptr=16, ldho=64, x_ptr=32, ldx=64, rstd_ptr=16)
    a.update(kw)
    return V.vla_block_norm(**a)


def norm_grad(**kw):
    a = dict(y_ptr=16, ldy=64, dtype=V.VLA_BF16, h_out_ptr=16, ldho=64, h_dtype=V.VLA_F32, rows=3, dim=64, post_gain_ptr=16, gate_ptr=16, ldg=64,
             residual_scale=1.0, pre_gain_ptr=16, rstd_ptr=16, d_x_ptr=16, lddx=64, d_h_out_ptr=16, lddho=64, d_h_ptr=32, lddh=64, d_y_ptr=32,
             lddy=64, d_gate_ptr=32, lddg=64, d_post_gain_ptr=16, d_pre_gain_ptr=16, ws_ptr=16, ws_bytes=1 << 30)
    a.update(kw)
    return V.vla_block_norm_grad(**a)


@pytest.mark.parametrize("change", [dict(y_ptr=0), dict(h_ptr=0), dict(h_out_ptr=0), dict(x_ptr=0), dict(pre_gain_ptr=0), dict(y_ptr=17), dict(h_ptr=18),
                                    dict(h_out_ptr=18), dict(x_ptr=17), dict(gate_ptr=17), dict(post_gain_ptr=17), dict(pre_gain_ptr=17),
                                    dict(rstd_ptr=18), dict(ldy=63), dict(ldh=63), dict(ldg=63), dict(ldho=63), dict(ldho=72), dict(ldx=63), dict(rows=-1),
                                    dict(dim=0), dict(eps=-1.0), dict(eps=float("nan")), dict(residual_scale=float("inf")),
                                    dict(y_ptr=0, post_gain_ptr=0, gate_ptr=0)])
def test_block_norm_refusals(change):
    refused(norm(**change), V.VLA_ERR_ARG, "vla_block_norm")


@pytest.mark.parametrize("change", [dict(y_ptr=0), dict(h_out_ptr=0), dict(d_x_ptr=0), dict(d_h_ptr=0), dict(d_y_ptr=0), dict(d_gate_ptr=0),
                                    dict(d_post_gain_ptr=0), dict(d_pre_gain_ptr=0), dict(rstd_ptr=0), dict(ws_ptr=0), dict(ws_ptr=8), dict(ws_bytes=8),
                                    dict(y_ptr=17), dict(h_out_ptr=18), dict(d_x_ptr=17), dict(d_h_ptr=18), dict(d_y_ptr=17), dict(d_gate_ptr=17),
                                    dict(d_gate_ptr=18, ldg=0), dict(d_post_gain_ptr=18), dict(d_pre_gain_ptr=18), dict(lddx=63), dict(lddho=63),
                                    dict(lddh=63), dict(lddy=63), dict(lddg=63), dict(rows=-1), dict(dim=0), dict(residual_scale=float("nan")),
                                    dict(d_h_out_ptr=32, lddho=72)])
def test_block_norm_grad_refusals(change):
    refused(norm_grad(**change), V.VLA_ERR_ARG, "vla_block_norm_grad")


@pytest.mark.parametrize("call,name", [(norm, "vla_block_norm"), (norm_grad, "vla_block_norm_grad")])
def test_block_norm_what_is_not_supported(call, name):
    for change in (dict(dtype=5), dict(h_dtype=V.VLA_F16), dict(dtype=V.VLA_F32, h_dtype=V.VLA_BF16), dict(dim=16385)):
        refused(call(**change), V.VLA_ERR_UNSUPPORTED, name)


def test_block_norm_no_rows_and_workspace_sizes():
    assert norm(rows=0) == V.VLA_OK
    assert norm(rows=0, y_ptr=0, post_gain_ptr=0, gate_ptr=0, h_out_ptr=0, h_ptr=0, x_ptr=0) == V.VLA_OK
    f = V.vla_block_norm_grad_workspace_bytes
    assert f(3, 64) >= 64 * 12 and f(-1, 64) == f(3, 0) == f(3, 16385) == 0
    assert f(1 << 30, 16384) < 1 << 30
