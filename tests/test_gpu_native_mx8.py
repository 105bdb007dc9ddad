"""The native calls of the rotary options and the quantised cache against the Python path: a call with no
`stream` goes to the native module first, one that names the current stream takes the Python path; both enqueue
the same kernels, so everything is equal bit for bit, and what the native module does not take still runs or
raises as the Python path does."""
import pytest
import torch

pytestmark = pytest.mark.gpu

u = pytest.importorskip("paper_2609_32518_amd")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

B, H, GH, GW, C, S, R, W, F0 = 2, 3, 4, 5, 2, 1, 7, 4, 9
N = C * GH * GW


def same(a, b):
    if isinstance(a, (tuple, list)):
        assert len(a) == len(b)
        for x, y in zip(a, b):
            same(x, y)
    elif a is None:
        assert b is None
    else:
        assert a.dtype == b.dtype and a.shape == b.shape
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def data(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = torch.randn(B, N, 3, H, 128, device="cuda", generator=g).bfloat16().unbind(2)
    w = [(1 + 0.1 * torch.randn(H * 128, device="cuda", generator=g)).bfloat16() for _ in range(2)]
    return q, k, v, w


def cache(kind):
    c = u.Cache(B, H, GH, GW, S, R) if kind == "bf16" else u.CacheMX8(B, H, GH, GW, S, R)
    for t in ((c.k, c.v) if kind == "bf16" else (c.k8, c.v8, c.k_scale, c.v_scale)):
        t.view(torch.uint8).fill_(60)
    for f in range(F0):
        c.advance(f, 1)
    return c


def buffers(c):
    return (c.k, c.v) if isinstance(c, u.Cache) else (c.k8, c.v8, c.k_scale, c.v_scale)


@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("given", [True, False])
def test_native_equals_python(with_q, norm, given, monkeypatch):
    taken = []
    for name in ("tables", "append_rotary", "append_mx8", "window_attn_mx8", "step_mx8", "read_mx8", "dequantize"):
        fn = getattr(u._calls_mx8, name)
        monkeypatch.setattr(u._calls_mx8, name, lambda *a, fn=fn, name=name: taken.append((name, r := fn(*a))) or r)
    q, k, v, w = data(1)
    kw = dict(layout="half")
    if norm:
        kw.update(q_norm_weight=w[0] if with_q else None, k_norm_weight=w[1], norm_eps=1e-5)
    res = []
    for stream in (None, torch.cuda.current_stream()):
        out = {}
        new = lambda *s, dt=torch.bfloat16: torch.empty(*s, 1, dtype=torch.uint8, device="cuda").squeeze(-1).view(dt) if dt.itemsize == 1 else torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        cos, sin = u.unstep_rotary_tables(F0, C, GH, GW, dims=(32, 16, 16), scaling="parts", factor=4.0, trained_frames=64.0, stream=stream)
        out["tables"] = (cos, sin)
        b, m = cache("bf16"), cache("mx8")
        g = dict(q_rot=new(B, N, H, 128)) if given and with_q else {}
        out["rotary"] = b.unstep_kv_append_rotary(F0, C, q if with_q else None, k, v, cos, sin, **kw, **g, stream=stream)
        g = dict(q8=new(B, N, H, 128, dt=torch.float8_e4m3fn), q_scale=new(B, N, H, 4, dt=torch.uint8)) if given and with_q else {}
        out["append"] = m.unstep_kv_append_mx8(F0, C, q if with_q else None, k, v, cos, sin, softmax_scale=0.07, **kw, **g, stream=stream)
        if given and with_q:
            assert out["append"][0] is g["q8"] and out["append"][1] is g["q_scale"]
        out["buffers"] = [t.clone() for t in buffers(b) + buffers(m)]
        g = dict(k_out=new(B, N, H, 128), v_out=new(B, N, H, 128)) if given else {}
        out["read"] = m.unstep_kv_read_mx8(F0, C, **g, stream=stream)
        if with_q:
            out["deq"] = u.unstep_mx8_dequantize(*out["append"], out=new(B, N, H, 128) if given else None, stream=stream)
            lse = [torch.empty(B, H, N, device="cuda") for _ in range(2)]
            g = dict(out=new(B, N, H, 128)) if given else {}
            for f in range(W + 1):                             # real rows in the window
                m.advance(F0 + C + f, 1)
            m = cache("mx8")
            for t in buffers(m):
                t.view(torch.uint8).fill_(56 if t.dtype != torch.uint8 else 127)
            step_kw = dict(kw)
            out["step"] = m.unstep_step_mx8(F0, C, W, q, k, v, cos, sin, lse=lse[0], **step_kw, **g, stream=stream)
            out["attn"] = m.unstep_window_attn_mx8(F0, C, W, *out["append"], lse=lse[1], stream=stream)
            out["lse"] = lse
        torch.cuda.synchronize()
        res.append(out)
    same([res[0][n] for n in res[0]], [res[1][n] for n in res[1]])
    want = {"tables", "append_rotary", "append_mx8", "read_mx8"} | ({"window_attn_mx8", "step_mx8", "dequantize"} if with_q else set())
    assert {n for n, r in taken if r is not None} == want and len(taken) == len(want)


def test_what_the_native_module_leaves_to_python():
    q, k, v, _ = data(2)
    cos, sin = u.unstep_rotary_tables(F0, C, GH, GW)
    m = cache("mx8")
    with pytest.raises(ValueError):
        m.unstep_kv_append_mx8(F0, C, q.float(), k, v, cos, sin)
    with pytest.raises(ValueError):
        m.unstep_kv_append_mx8(F0, C, q, k, v, cos, sin, layout="other")
    with pytest.raises(u.UnstepError) as e:
        m.unstep_kv_append_mx8(F0 + 3, C, q, k, v, cos, sin)
    assert e.value.code == u.E_STATE and m.frame_map()[1] == F0 - 1
    with pytest.raises(u.UnstepError) as e:
        m.unstep_step_mx8(F0, C, 50, q, k, v, cos, sin)
    assert e.value.code == u.E_RANGE and m.frame_map()[1] == F0 - 1
    with pytest.raises(u.UnstepError) as e:
        u.unstep_rotary_tables(0, 1, 2, 2, dims=(44, 42, 40))
    assert e.value.code == u.E_SHAPE
    # integers given for floats, and parameters as tensors, run
    a = m.unstep_step_mx8(F0, C, W, torch.nn.Parameter(q, requires_grad=False), k, v, cos, sin, softmax_scale=0)
    b = m.unstep_step_mx8(F0, C, W, q, k, v, cos, sin)
    same(a, b)

    class Mine(u.CacheMX8):
        def workspace(self, *a):
            asked.append(a)
            return None
    asked = []
    c = Mine(B, H, GH, GW, S, R)
    for f in range(F0):
        c.advance(f, 1)
    c.unstep_step_mx8(F0, C, W, q, k, v, cos, sin)
    assert asked
