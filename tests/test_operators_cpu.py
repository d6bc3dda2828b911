"""Refusals of the operators around the layer: on the host, before any device work, with a reason."""
import ctypes
import os

import pytest

from paper_2506_02965_gb300 import build as _build

if not os.path.exists(_build.LIB) or _build._stale(_build.LIB, os.path.join(_build.CSRC, "moe_abi.cu")):
    _build.build()
from paper_2506_02965_gb300 import _lib as L  # noqa: E402


def refused(frag, status, fn, *args):
    with pytest.raises(L.MoEError) as e:
        fn(*args, stream=0)
    assert e.value.status == status and frag in str(e.value), str(e.value)


BAD = L.MOE_ERR_INVALID_ARG


@pytest.mark.parametrize("change,frag", [
    (dict(rows=-1), "rows=-1"), (dict(rows=1 << 31), "rows="), (dict(d=0), "width 0"), (dict(dtype=5), "dtype"),
    (dict(x=None), "x is NULL"), (dict(x=17), "x is not aligned"), (dict(gamma=None), "gamma is NULL"), (dict(gamma=18), "gamma"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(residual=16), "h is NULL"), (dict(h=16), "without a residual"),
    (dict(y=None), "y is NULL"), (dict(mean=16), "mean and rstd"), (dict(q=16), "h_q and h_scale")])
def test_norm_forward(change, frag):
    a = dict(rows=4, d=64, dtype=L.MOE_BF16, x=16, residual=None, gamma=16, beta=None, eps=1e-5, h=None, y=16, mean=None, rstd=None,
             q=None, scale=None)
    a.update(change)
    refused(frag, BAD, L.moe_layer_norm_fwd, *a.values())


def test_norm_width_limit():
    refused("16385", L.MOE_ERR_UNSUPPORTED, L.moe_layer_norm_fwd, 4, 16385, L.MOE_F32, 16, None, 16, None, 1e-5, None, 16)
    with pytest.raises(L.MoEError):
        L.moe_layer_norm_workspace_size(4, 16385)
    assert L.moe_layer_norm_workspace_size(4, 16384) >= 2 * 4 * 16384 * 4


@pytest.mark.parametrize("change,frag", [
    (dict(dy=None), "dy is NULL"), (dict(h=None), "one of h and h_q"), (dict(q=16, scale=16), "one of h and h_q"),
    (dict(h=None, q=16), "h_q and h_scale"), (dict(mean=None), "mean is NULL"), (dict(dx=None), "dx is NULL"),
    (dict(dgamma=None), "dgamma is NULL"), (dict(ws=None), "workspace is NULL"), (dict(wsb=8), "workspace of 8 bytes"),
    (dict(rstd=18), "rstd is not aligned"), (dict(rows=-2), "rows=")])
def test_norm_backward(change, frag):
    a = dict(rows=4, d=64, dtype=L.MOE_F32, dy=16, h=16, q=None, scale=None, mean=16, rstd=16, gamma=16, dh=None, dx=16, dgamma=16,
             dbeta=None, ws=16, wsb=1 << 20)
    a.update(change)
    refused(frag, BAD, L.moe_layer_norm_bwd, *a.values())


@pytest.mark.parametrize("kw,frag", [
    (dict(score=2), "score 2"), (dict(n_groups=0), "n_groups=0"), (dict(n_groups=3), "n_groups=3"), (dict(n_groups=64), "n_groups=64"),
    (dict(n_groups=8, top_groups=9), "top_groups=9"), (dict(top_groups=0), "top_groups=0"),
    (dict(n_groups=32, top_groups=1), "fewer than top_k"), (dict(group_top=3), "group_top=3"),
    (dict(n_groups=32, top_groups=32, group_top=0), "group_top=0"), (dict(scale=float("inf")), "scale"),
    (dict(scale=float("nan")), "scale")])
def test_rules(kw, frag):
    cfg = L.make_config(8, 128, 64, 128, 4)
    r = L.make_gate_rule(**kw)
    refused(frag, BAD, L.moe_gate, cfg, r, 16, None, None, None, 16, 16, 16)
    refused(frag, BAD, L.moe_route_gate, cfg, r, 16, 16, None, None, None, 16, 16, 16, 16, 16)
    refused(frag, BAD, L.moe_gate_bwd, cfg, r, 16, 16, 16, None, None, 16)


def test_group_of_one_expert_has_no_second_key():
    cfg = L.make_config(8, 128, 16, 128, 4)
    refused("group_top=2", BAD, L.moe_gate, cfg, L.make_gate_rule(n_groups=16, top_groups=8, group_top=2), 16, None, None, None, 16, 16, 16)


def test_gate_arguments():
    cfg, r = L.make_config(8, 128, 64, 128, 4), L.make_gate_rule()
    refused("logits is NULL", BAD, L.moe_gate, cfg, r, None, None, None, None, 16, 16, 16)
    refused("counts is NULL", BAD, L.moe_gate, cfg, r, 16, None, None, None, 16, 16, None)
    refused("topk_w is not aligned", BAD, L.moe_gate, cfg, r, 16, None, None, None, 16, 18, 16)
    refused("rule is NULL", BAD, L.moe_gate, cfg, None, 16, None, None, None, 16, 16, 16)
    two = L.make_config(8, 128, 64, 128, 4, n_parties=2)
    refused("party_offsets", BAD, L.moe_gate, two, r, 16, None, None, None, 16, 16, 16)
    refused("n_experts=257", L.MOE_ERR_UNSUPPORTED, L.moe_gate, L.make_config(8, 128, 257, 128, 4), r, 16, None, None, None, 16, 16, 16)
    refused("come with dw_router", BAD, L.moe_gate_bwd, cfg, r, 16, 16, 16, None, None, 16, 16, 16, None, 16)
    refused("workspace of 16", BAD, L.moe_gate_bwd, cfg, r, 16, 16, 16, None, None, 16, 16, 16, 16, None, 16, 16, 16)
    refused("x is NULL", BAD, L.moe_gate_bwd, cfg, r, 16, 16, 16, None, None, 16, None, 16, 16, None, 16, 16, 16)
    refused("rate", BAD, L.moe_gate_balance, cfg, 16, float("nan"), 16, 16)
    refused("bias_out is NULL", BAD, L.moe_gate_balance, cfg, 16, 0.1, 16, None)


def test_checkpoint_arguments():
    for fn, n in ((L.moe_ckpt_pack, 3), (L.moe_ckpt_unpack, 3), (L.moe_ckpt_swiglu_bwd, 5)):
        refused("rows=-1", BAD, fn, -1, 8, L.MOE_F32, *[16] * n)
        refused("width 0", BAD, fn, 4, 0, L.MOE_F32, *[16] * n)
        refused("dtype", BAD, fn, 4, 8, 9, *[16] * n)
        refused("NULL", BAD, fn, 4, 8, L.MOE_F32, *[None] * n)
    refused("x is not aligned", BAD, L.moe_ckpt_pack, 4, 8, L.MOE_F32, 18, 16, 16)
    refused("scale is not aligned", BAD, L.moe_ckpt_unpack, 4, 8, L.MOE_F32, 16, 17, 16)
    refused("2^30", BAD, L.moe_ckpt_swiglu_bwd, 1, 1 << 30, L.MOE_F32, *[16] * 5)
    cfg = L.make_config(8, 128, 8, 128, 2)
    refused("gu_q is NULL", BAD, L.moe_expert_ffn_bwd_ckpt, cfg, 16, 16, 16, 16, None, 16, 16, 16, 16, 16, 16, 16, 16)
    refused("dact is not 16-byte", BAD, L.moe_expert_ffn_bwd_ckpt, cfg, 16, 16, 16, 16, 16, 16, 16, 24, 16, 16, 16, 16, 16)


def test_tensors_are_looked_at():
    """A tensor of another type, size, layout or place is refused before its address is taken."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    for bad in (x, x.to(torch.float64), x[:, ::2], x[:2]):
        with pytest.raises(L.MoEError, match="dense GPU tensor"):
            L.moe_ckpt_pack(4, 8, L.MOE_F32, bad, None, None, stream=0)
    with pytest.raises(L.MoEError, match="balance_bias"):
        L.moe_gate(L.make_config(8, 128, 64, 128, 4), L.make_gate_rule(), 16, x, None, None, 16, 16, 16, stream=0)


def test_rule_struct_layout():
    assert ctypes.sizeof(L.moe_gate_rule) == 20
    assert [f[0] for f in L.moe_gate_rule._fields_] == ["score", "n_groups", "top_groups", "group_top", "scale"]


def test_argument_checks_in_both_languages():
    """The C++ form of the checks, where it is built, refuses what the Python form refuses, with its words."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    assert L._arr("f", "x", None, L.MOE_F32, 32) is None and L._arr("f", "x", 48, L.MOE_F32, 32) == 48
    for bad in (x, x.bool(), x.t(), torch.sparse_coo_tensor(size=(4, 8)), torch.empty(4, 8, device="meta")):
        said = []
        for check in (L._arr, L._check_arr):
            with pytest.raises(Exception) as e:
                check("f", "x", bad, L.MOE_F32, 32)
            said.append((type(e.value), str(e.value)))
        assert said[0] == said[1]


def test_expert_backward_and_workspaces_are_looked_at():
    """The tensors of the experts' backward from a checkpoint, and workspaces: refused before their address is taken, with
    what they should have been. What a call does not use is not looked at."""
    torch = pytest.importorskip("torch")
    T, d, E, F, k, S, Fs = 8, 128, 4, 256, 2, 1, 128
    cfg = L.make_config(T, d, E, F, k, n_shared=S, d_ff_shared=Fs)
    TK = T * k
    sizes = {"x_perm": TK * d, "offsets": E + 1, "w1": E * 2 * F * d, "w2": E * d * F, "gu_q": TK * 2 * F, "gu_scale": TK * 4,
             "dy_perm": TK * d, "dact": TK * F, "act": TK * F, "dh": TK * 2 * F, "dx_perm": TK * d, "dw1": E * 2 * F * d,
             "dw2": E * d * F, "x": T * d, "dout": T * d, "ws1": S * 2 * Fs * d, "ws2": S * d * Fs, "h_gu_sh": S * T * 2 * Fs,
             "act_sh": S * T * Fs, "dh_sh": S * T * 2 * Fs, "dx_sh": S * T * d, "dws1": S * 2 * Fs * d, "dws2": S * d * Fs,
             "group_expert": E}
    kinds = {"offsets": "int32", "group_expert": "int32", "gu_q": "int8", "gu_scale": "float32"}
    for name, n in sizes.items():
        say = f"{name}: expected a dense GPU tensor of {n} elements of torch.{kinds.get(name, 'bfloat16')}"
        with pytest.raises(L.MoEError, match=say):
            L.moe_expert_ffn_bwd_ckpt(cfg, **{**dict.fromkeys(sizes, 16), name: torch.zeros(n - 1)}, stream=0)
    small = torch.zeros(4)
    unused = {m: small if m not in ("dw1", "dw2") else None for m in sizes}
    with pytest.raises(L.MoEError, match="dw1 is NULL"):
        L.moe_expert_ffn_bwd_ckpt(L.make_config(0, d, E, F, k), **unused, stream=0)
    with pytest.raises(L.MoEError, match="workspace: expected a dense GPU tensor of 64 bytes"):
        L.moe_layer_norm_bwd(4, 64, L.MOE_F32, 16, 16, None, None, 16, 16, 16, None, 16, 16, None, small, 64, stream=0)
    one, r = L.make_config(8, 128, 64, 128, 4), L.make_gate_rule()
    with pytest.raises(L.MoEError, match="workspace: expected a dense GPU tensor of 64 bytes"):
        L.moe_gate_bwd(one, r, 16, 16, 16, None, None, 16, 16, 16, 16, None, 16, small, 64, stream=0)
    with pytest.raises(L.MoEError, match="come with dw_router"):
        L.moe_gate_bwd(one, r, 16, 16, 16, None, None, 16, 16, 16, None, 16, None, small, 64, stream=0)


@pytest.mark.parametrize("name", ["x", "w_router", "router_bias", "balance_bias", "logits", "scores", "topk_idx", "topk_w", "counts"])
def test_route_gate_refuses_before_it_launches(name):
    """A pointer off its alignment or missing is an invalid argument, not the status of a launch on the way to it."""
    cfg, r = L.make_config(8, 128, 64, 128, 4), L.make_gate_rule()
    a = dict(x=16, w_router=16, router_bias=None, balance_bias=None, party_offsets=None, logits=16, scores=16, topk_idx=16, topk_w=16,
             counts=16)
    refused(f"{name} is not ", BAD, L.moe_route_gate, cfg, r, *{**a, name: 18}.values())
    if a[name] is not None:
        refused(f"{name} is NULL", BAD, L.moe_route_gate, cfg, r, *{**a, name: None}.values())
