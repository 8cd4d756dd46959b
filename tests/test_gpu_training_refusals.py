"""What the calls around a training step's layers refuse: a status, a message, nothing launched, nothing written."""
import ctypes

import pytest
import torch

from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

CAP, T, D, V = 3, 16, 64, 80
INVALID, TABLE, TENANT, SMALL = (B.MARLAAS_ERR_INVALID_ARG, B.MARLAAS_ERR_BAD_SEGMENT_TABLE, B.MARLAAS_ERR_UNKNOWN_TENANT,
                                 B.MARLAAS_ERR_WORKSPACE_TOO_SMALL)


class Env:
    """One valid set of arguments per call, as ctypes takes them; `call` with some of them replaced."""

    def __init__(self):
        self.lib = B.load_library()
        self.pool = B.AdapterPool(D, V, 8, CAP)
        B.marlaas_adapter_pool_register(self.pool, 5, 0, 0, 1.0, None, None)        # slot 0; slots 1 and 2 hold nobody
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.x, self.dy, self.W = torch.zeros((T, D), **bf), torch.zeros((T, V), **bf), torch.zeros((D, V), **bf)
        self.out = torch.full((T, V), 7.0, **bf)
        self.gain = torch.ones((CAP + 1, D), device="cuda")
        self.f = torch.full((T * 64,), 7.0, device="cuda")
        self.targets = torch.zeros(T, dtype=torch.int32, device="cuda")
        self.rates = torch.zeros(CAP, device="cuda")
        self.ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
        self.seg = B.Segments(torch.tensor([0, T], dtype=torch.int32, device="cuda"), torch.tensor([0], dtype=torch.int32, device="cuda"))
        self.host = B.Segments(torch.tensor([0, T], dtype=torch.int32), torch.tensor([0], dtype=torch.int32))
        self.drop = B.marlaas_dropout_t(self.rates.data_ptr(), 1, 2)
        p = lambda t: t.data_ptr()      # noqa: E731
        h, ws, n = self.pool.handle, p(self.ws), self.ws.numel()
        self.args = dict(
            layer_norm=dict(pool=h, T=T, d=D, x=p(self.x), ldx=D, seg=self.seg.ref, gain=p(self.gain), bias=p(self.gain), eps=1e-5, y=p(self.out), ldy=V,
                            mean=p(self.f), rstd=p(self.f), ws=ws, n=n, flags=0, st=0),
            layer_norm_backward=dict(pool=h, T=T, d=D, x=p(self.x), ldx=D, dy=p(self.x), lddy=D, seg=self.seg.ref, gain=p(self.gain), mean=p(self.f),
                                     rstd=p(self.f), dx=p(self.out), lddx=V, dgain=p(self.f), dbias=p(self.f), ws=ws, n=n, flags=0, st=0),
            head_cross_entropy=dict(pool=h, T=T, d=D, V=V, x=p(self.x), ldx=D, W=p(self.W), ldw=V, targets=p(self.targets), seg=self.seg.ref,
                                    weight=None, k=1.0, scale=1.0, dx=p(self.out), lddx=V, logp=p(self.f), stats=p(self.f), ws=ws, n=n, flags=0, st=0),
            lora_forward_dropout=dict(pool=h, T=T, x=p(self.x), ldx=D, W=p(self.W), ldw=V, y=p(self.out), ldy=V, seg=self.seg.ref,
                                      drop=ctypes.byref(self.drop), h=p(self.f), ws=ws, n=n, flags=0, st=0),
            lora_backward_dropout=dict(pool=h, T=T, x=p(self.x), ldx=D, W=p(self.W), ldw=V, dy=p(self.dy), lddy=V, dx=p(self.out), lddx=V, dA=None, dB=None,
                                       seg=self.seg.ref, drop=ctypes.byref(self.drop), h=None, ws=ws, n=n, flags=0, st=0))

    def call(self, name, **change):
        a = dict(self.args[name], **change)
        return getattr(self.lib, "marlaas_" + name)(*a.values())

    def refused(self, name, status, **change):
        before = B.marlaas_kernel_launch_count()
        assert self.call(name, **change) == status, (name, change, B.marlaas_last_error())
        assert B.marlaas_last_error().startswith(name)
        assert B.marlaas_kernel_launch_count() == before
        torch.cuda.synchronize()
        assert torch.all(self.out == 7) and torch.all(self.f == 7)


@pytest.fixture(scope="module")
def env():
    return Env()


def tables():
    """Host tables that are not as described, and their statuses."""
    def seg(off, slot):
        return B.Segments(torch.tensor(off, dtype=torch.int32), torch.tensor(slot, dtype=torch.int32))
    return [(seg([1, T], [0]), TABLE), (seg([0, T - 1], [0]), TABLE), (seg([0, 9, 5, T], [0, 0, 0]), TABLE), (seg([0, T], [CAP]), TABLE),
            (seg([0, T], [-2]), TABLE), (seg([0, T], [1]), TENANT)]


MATRICES = dict(layer_norm=("x", "y"), layer_norm_backward=("x", "dy", "dx"), head_cross_entropy=("x", "W", "dx"),
                lora_forward_dropout=("x", "W", "y"), lora_backward_dropout=("W", "dy", "dx"))
OPTIONAL = {"dx"}


@pytest.mark.parametrize("name", sorted(MATRICES))
def test_common(env, name):
    bad = lambda **c: env.refused(name, INVALID, **c)       # noqa: E731
    bad(pool=None)
    bad(T=-1)
    bad(T=1 << 31)
    bad(flags=B.MARLAAS_FLAG_REUSE_PLAN)
    bad(flags=B.MARLAAS_FLAG_CUDA_CORE_PATH)
    bad(flags=1 << 31)
    bad(seg=None)
    for m in MATRICES[name]:
        if m not in OPTIONAL:
            bad(**{m: None})
        bad(**{m: env.args[name][m] + 2})
        bad(**{"ld" + m.lower(): 8 * 7})         # below the width
        bad(**{"ld" + m.lower(): V + 4})
    bad(ws=env.args[name]["ws"] + 16) if name != "layer_norm" else None
    if name != "layer_norm":
        bad(ws=None)
        env.refused(name, SMALL, n=64)
    for s, status in tables():
        env.refused(name, status, seg=s.ref, flags=B.MARLAAS_FLAG_HOST_TABLE)
    empty = B.marlaas_segments_t(0, None, None)
    env.refused(name, TABLE, seg=ctypes.byref(empty))
    env.refused(name, INVALID, seg=ctypes.byref(B.marlaas_segments_t(-1, None, None)))


def test_layer_norm(env):
    for name in ("layer_norm", "layer_norm_backward"):
        for d in (0, 4, 12, B.MARLAAS_MAX_NORM_WIDTH + 8):
            env.refused(name, INVALID, d=d)
        env.refused(name, INVALID, gain=None)
        env.refused(name, INVALID, gain=env.args[name]["gain"] + 4)
    bad = lambda **c: env.refused("layer_norm", INVALID, **c)       # noqa: E731
    bad(bias=env.args["layer_norm"]["bias"] + 8)
    for eps in (-1.0, float("nan"), float("inf")):
        bad(eps=eps)
    bad(flags=B.MARLAAS_FLAG_ACCUMULATE)
    bad(mean=env.args["layer_norm"]["mean"] + 2)
    bad(y=env.args["layer_norm"]["x"] + 16, ldy=D)           # overlaps x
    bad(ws=None, flags=B.MARLAAS_FLAG_HOST_TABLE, seg=env.host.ref)
    env.refused("layer_norm", SMALL, n=8, flags=B.MARLAAS_FLAG_HOST_TABLE, seg=env.host.ref)
    bad = lambda **c: env.refused("layer_norm_backward", INVALID, **c)       # noqa: E731
    bad(rstd=None)
    bad(mean=None)
    bad(dx=None, dgain=None, dbias=None)
    bad(dgain=env.args["layer_norm_backward"]["dgain"] + 4)
    bad(dx=env.args["layer_norm_backward"]["x"] + 32, lddx=D)


def test_head(env):
    bad = lambda **c: env.refused("head_cross_entropy", INVALID, **c)       # noqa: E731
    for d in (0, 12, B.MARLAAS_MAX_HEAD_WIDTH + 8):
        bad(d=d)
    for v in (0, B.MARLAAS_MAX_VOCABULARY + 1):
        bad(V=v)
    bad(targets=None)
    bad(targets=env.args["head_cross_entropy"]["targets"] + 1)
    bad(weight=2)
    for k in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        bad(k=k)
    bad(scale=float("nan"))
    bad(dx=None, logp=None, stats=None)
    bad(logp=env.args["head_cross_entropy"]["targets"], weight=env.args["head_cross_entropy"]["targets"])
    bad(dx=env.args["head_cross_entropy"]["x"] + 16, lddx=D)
    bad(flags=B.MARLAAS_FLAG_RMS_NORM)
    assert B.marlaas_head_cross_entropy_workspace_bytes(env.pool, T, 12, V, 1, True) == 0
    assert B.marlaas_head_cross_entropy_workspace_bytes(env.pool, T, D, 0, 1, True) == 0
    # without stats the table is not read
    assert env.call("head_cross_entropy", seg=None, stats=None, dx=None, logp=env.ws.data_ptr() + (1 << 25)) == B.MARLAAS_OK


def test_dropout(env):
    for name in ("lora_forward_dropout", "lora_backward_dropout"):
        env.refused(name, INVALID, drop=None)
        env.refused(name, INVALID, drop=ctypes.byref(B.marlaas_dropout_t(None, 1, 2)))
        env.refused(name, INVALID, drop=ctypes.byref(B.marlaas_dropout_t(env.rates.data_ptr() + 2, 1, 2)))
        env.refused(name, INVALID, h=env.f.data_ptr() + 4)
    tab = (ctypes.c_void_p * CAP)(env.f.data_ptr() + 2, None, None)
    env.refused("lora_backward_dropout", INVALID, dA=tab)
    env.refused("lora_backward_dropout", INVALID, dB=tab)
    ok = (ctypes.c_void_p * CAP)(env.f.data_ptr(), None, None)
    env.refused("lora_backward_dropout", INVALID, dA=ok, x=None)
    env.refused("lora_backward_dropout", INVALID, dB=ok, x=None)         # h is not saved: x is read
    env.refused("lora_forward_dropout", INVALID, flags=B.MARLAAS_FLAG_ACCUMULATE)


def test_captures_refuse_host_tables(env):
    s = env.host
    st = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        env.out.add_(0)         # (a graph of something)
        for name in MATRICES:
            assert env.call(name, seg=s.ref, flags=B.MARLAAS_FLAG_HOST_TABLE, st=st.cuda_stream) == INVALID, name
            assert "captured" in B.marlaas_last_error()


def test_captures_refuse_pointer_tables_of_large_pools():
    pool = B.AdapterPool(D, V, 8, 65)
    x, dy, W = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((T, D), (T, V), (D, V)))
    B.marlaas_adapter_pool_register(pool, 1, 0, 8, 8.0, torch.zeros((D, 8), dtype=torch.bfloat16, device="cuda"),
                                    torch.zeros((8, V), dtype=torch.bfloat16, device="cuda"))
    dA = [torch.full((D, 8), 2.0, device="cuda")]
    seg = B.Segments(torch.tensor([0, T], dtype=torch.int32, device="cuda"), torch.tensor([0], dtype=torch.int32, device="cuda"))
    rates = torch.zeros(65, device="cuda")
    B.marlaas_lora_backward_dropout(pool, x, W, dy, seg, rates, 1, dA=dA)
    assert not dA[0].any()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_lora_backward_dropout(pool, x, W, dy, seg, rates, 1, dA=dA)
        assert e.value.status == INVALID


def test_the_binding_checks_its_tensors(env):
    x, W, seg, rates, gain = env.x, env.W, env.seg, env.rates, env.gain
    with pytest.raises(AssertionError):
        B.marlaas_lora_forward_dropout(env.pool, x.float(), W, seg, rates, 1)
    with pytest.raises(AssertionError):
        B.marlaas_lora_forward_dropout(env.pool, x, W, seg, rates[:2], 1)
    with pytest.raises(AssertionError):
        B.marlaas_lora_forward_dropout(env.pool, x, W, seg, rates, -1)
    with pytest.raises(AssertionError):
        B.marlaas_lora_forward_dropout(env.pool, x, W, seg, rates, 1 << 64)
    with pytest.raises(AssertionError):
        B.marlaas_layer_norm(env.pool, x, seg, gain[:2])
    with pytest.raises(AssertionError):
        B.marlaas_layer_norm(env.pool, x.t(), seg, gain)
    with pytest.raises(AssertionError):
        B.marlaas_head_cross_entropy(env.pool, x, W, env.targets.long(), seg)
    with pytest.raises(AssertionError):
        B.marlaas_head_cross_entropy(env.pool, x, W, env.targets, stats=torch.zeros((CAP + 1, 4), device="cuda"))
    with pytest.raises(B.MarlaasError):
        B.marlaas_layer_norm(env.pool, x[:1].expand(T, D), seg, gain)           # rows on top of one another
