"""Embedding lookup and its gradient by sorted tokens against a plain form in 64 bits.

Tolerances, from the arithmetic: the lookup is one fp32 product and one rounding to the storage type; a gradient row of n
tokens is n fp32 additions, one product and one rounding, so it is off by at most (n + 2) 2^-24 of the sum of its
terms' magnitudes and half a step of the storage type.
"""
import pytest
import torch

from paper_2506_02965_gb300 import _lib as L

pytestmark = pytest.mark.gpu
DT = {"f32": (L.MOE_F32, torch.float32), "bf16": (L.MOE_BF16, torch.bfloat16)}


def half(dt):
    return torch.finfo(dt).eps / 2


def make(T, d, V, kind, seed, skew=True, off=0):
    """ids, w, dout; `off` elements off an allocation's start."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[kind][1]

    def rnd(r, c):
        flat = torch.randn(r * c + off, generator=g, device="cuda").to(dt)
        return flat[off:].view(r, c)

    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    ids = (V ** u).long().sub(1) if skew else (u * V).long()
    ids = ids.clamp(0, V - 1).int()
    return ids, rnd(V, d), rnd(T, d)


def check_fwd(ids, w, scale, out):
    live = (ids >= 0) & (ids < w.shape[0])
    ref = torch.where(live[:, None], w.double()[ids.long().clamp(0, w.shape[0] - 1)] * scale, 0.0)
    assert ((out.double() - ref).abs() <= (half(w.dtype) + 2.0 ** -24) * ref.abs()).all()


def grad_ref(ids, dout, V, scale):
    live = (ids >= 0) & (ids < V)
    at = torch.where(live, ids, V).long()
    d64 = dout.double()
    ref = torch.zeros(V + 1, dout.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, d64)[:V] * scale
    mag = torch.zeros(V + 1, dout.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, d64.abs())[:V] * abs(scale)
    n = torch.bincount(at, minlength=V + 1)[:V, None]
    return ref, mag, n


def backward(ids, dout, V, kind, scale, dw, accumulate=False, stream=None):
    T, d = dout.shape
    ws = torch.empty(L.moe_embed_workspace_size(T, d, V), dtype=torch.uint8, device="cuda")
    L.moe_embed_bwd(T, d, V, DT[kind][0], ids, dout, scale, accumulate, dw, ws, ws.numel(), stream=stream)
    return dw


def check_bwd(ids, dout, V, scale, dw, base=None):
    ref, mag, n = grad_ref(ids, dout, V, scale)
    if base is not None:
        ref, mag = ref + base.double(), mag + base.double().abs()
    err = (dw.double() - ref).abs()
    bound = (n + 2) * 2.0 ** -24 * mag + half(dw.dtype) * ref.abs() * (1 + 1e-6)
    assert (err <= bound).all(), (err - bound).max()
    if base is not None:
        still = n[:, 0] == 0
        assert torch.equal(dw[still], base[still])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(1, 8, 1), (1, 4096, 131072), (7, 1, 3), (33, 100, 517), (64, 130, 511), (65, 64, 512), (300, 333, 513),
                                   (2049, 72, 1000), (4097, 1024, 50021), (9000, 40, 262143), (16500, 24, 262144), (1000, 3, 300000)])
def test_step(kind, T, d, V):
    ids, w, dout = make(T, d, V, kind, T + d)
    ids[::5] = torch.where(torch.arange(ids[::5].numel(), device="cuda") % 3 == 0, -1 - ids[::5], ids[::5])
    out = torch.full_like(dout, float("nan"))
    L.moe_embed_fwd(T, d, V, DT[kind][0], ids, w, 1.7, out)
    check_fwd(ids, w, 1.7, out)
    dw = backward(ids, dout, V, kind, 1.7, torch.full_like(w, float("nan")))
    check_bwd(ids, dout, V, 1.7, dw)
    again = backward(ids, dout, V, kind, 1.7, torch.empty_like(w))
    assert torch.equal(dw, again)  # fixed order of additions
    base = w.clone()
    check_bwd(ids, dout, V, 1.7, backward(ids, dout, V, kind, 1.7, w.clone(), accumulate=True), base)
    assert L.moe_device_status() == 0


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 31, 32, 33, 64, 65, 2048, 8192, 8193, 40000])
@pytest.mark.parametrize("pattern", ["one", "two", "distinct", "padding"])
def test_runs(kind, T, pattern):
    """All tokens alike, two ids that meet inside a chunk, no two alike, nothing but padding."""
    V, d = 70000, 24
    _, w, dout = make(T, d, V, kind, T)
    i = torch.arange(T, device="cuda", dtype=torch.int32)
    ids = {"one": i * 0 + V - 1, "two": (i % 7 == 0).int() * 5, "distinct": (i * 7919) % V, "padding": i * 0 - 1}[pattern].int().contiguous()
    check_bwd(ids, dout, V, 0.5, backward(ids, dout, V, kind, 0.5, torch.full_like(w, float("nan"))))
    base = w.clone()
    check_bwd(ids, dout, V, 0.5, backward(ids, dout, V, kind, 0.5, w, accumulate=True), base)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("off", [1, 2, 4])
@pytest.mark.parametrize("d", [64, 250])
def test_alignment(kind, off, d):
    T, V = 500, 300
    ids, w, dout = make(T, d, V, kind, 3, off=off)
    out = torch.empty(T * d + off, dtype=w.dtype, device="cuda")[off:].view(T, d)
    L.moe_embed_fwd(T, d, V, DT[kind][0], ids, w, 3.0, out)
    check_fwd(ids, w, 3.0, out)
    dw = torch.empty(V * d + off, dtype=w.dtype, device="cuda")[off:].view(V, d)
    check_bwd(ids, dout, V, 3.0, backward(ids, dout, V, kind, 3.0, dw))


def test_a_long_run_of_unequal_terms():
    """One id, 2^24 and then ones: a 1 that meets the large sum alone is half a step and lost, those of later chunks are added
    up first. Between the two extremes, the same bits on every call, and whatever other ids are in the batch."""
    T, V, d = 200, 9, 4
    ids = torch.full((T,), 4, dtype=torch.int32, device="cuda")
    dout = torch.ones(T, d, device="cuda")
    dout[0] = 2.0 ** 24
    dw = backward(ids, dout, V, "f32", 1.0, torch.empty(V, d, device="cuda"))
    check_bwd(ids, dout, V, 1.0, dw)
    assert (dw[4] > 2.0 ** 24).all() and (dw[4] <= 2.0 ** 24 + T - 1).all() and (dw[:4] == 0).all() and (dw[5:] == 0).all()
    for _ in range(3):
        assert torch.equal(dw, backward(ids, dout, V, "f32", 1.0, torch.empty(V, d, device="cuda")))
    ids[50::50] = 7
    check_bwd(ids, dout, V, 1.0, backward(ids, dout, V, "f32", 1.0, torch.empty(V, d, device="cuda")))


def test_ids_out_of_range_are_recorded():
    T, V, d = 40, 50, 16
    ids, w, dout = make(T, d, V, "f32", 5)
    ids[3], ids[7] = V, 2 ** 31 - 1
    out = torch.empty_like(dout)
    L.moe_embed_fwd(T, d, V, L.MOE_F32, ids, w, 1.0, out)
    check_fwd(ids, w, 1.0, out)
    assert L.moe_device_status() == L.MOE_ERR_DEVICE_CHECK and L.moe_device_status() == 0
    check_bwd(ids, dout, V, 1.0, backward(ids, dout, V, "f32", 1.0, torch.empty_like(w)))
    assert L.moe_device_status() == L.MOE_ERR_DEVICE_CHECK and L.moe_device_status() == 0


def test_no_tokens():
    w = torch.ones(10, 4, device="cuda")
    L.moe_embed_fwd(0, 4, 10, L.MOE_F32, None, None, 1.0, None)
    L.moe_embed_bwd(0, 4, 10, L.MOE_F32, None, None, 1.0, True, w, None, 0)
    assert (w == 1).all()
    L.moe_embed_bwd(0, 4, 10, L.MOE_F32, None, None, 1.0, False, w, None, 0)
    assert (w == 0).all()


def test_infinities_stay_in_their_rows():
    ids = torch.tensor([3, 1, 3, 2, 0], dtype=torch.int32, device="cuda")
    dout = torch.ones(5, 8, device="cuda")
    dout[1], dout[3, 2] = float("inf"), float("nan")
    dw = backward(ids, dout, 5, "f32", 1.0, torch.empty(5, 8, device="cuda"))
    assert torch.isinf(dw[1]).all() and torch.isnan(dw[2, 2]) and torch.isfinite(dw[[0, 3, 4]]).all() and (dw[3] == 2).all()


@pytest.mark.slow
def test_offsets_past_32_bits():
    T, d, V = 600, 8192, 270000  # 2.2e9 elements of W
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[-1], w[-2] = 2.0, 3.0
    ids = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    ids[::2] = V - 2
    out = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    L.moe_embed_fwd(T, d, V, L.MOE_BF16, ids, w, 2.0, out)
    assert (out[1::2] == 4).all() and (out[::2] == 6).all()
    dw = backward(ids, out, V, "bf16", 1.0, w)
    assert (dw[-1] == 1200).all() and (dw[-2] == 1800).all() and not dw[:-2].any()


def test_other_stream_and_graph():
    T, d, V = 3000, 256, 5000
    ids, w, dout = make(T, d, V, "bf16", 11)
    out, dw = torch.empty_like(dout), torch.empty_like(w)
    ws = torch.empty(L.moe_embed_workspace_size(T, d, V), dtype=torch.uint8, device="cuda")

    def step():
        L.moe_embed_fwd(T, d, V, L.MOE_BF16, ids, w, 16.0, out)
        L.moe_embed_bwd(T, d, V, L.MOE_BF16, ids, dout, 16.0, False, dw, ws, ws.numel())

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    check_fwd(ids, w, 16.0, out)
    check_bwd(ids, dout, V, 16.0, dw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ids.copy_(make(T, d, V, "bf16", 12)[0])
    out.zero_(), dw.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    check_fwd(ids, w, 16.0, out)
    check_bwd(ids, dout, V, 16.0, dw)
