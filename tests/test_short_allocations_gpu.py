"""New outputs of the native short forms are torch's: its dispatcher sees them made, and they hold what it
fills new memory with where deterministic algorithms are asked for."""
import pytest

from test_short_forms_gpu import ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from torch.utils._python_dispatch import TorchDispatchMode

import fp4_ref as ref


class Made(TorchDispatchMode):
    """Bytes of the tensors made under it."""

    def __init__(self):
        super().__init__()
        self.bytes = 0

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        r = func(*args, **(kwargs or {}))
        if func.overloadpacket in (torch.ops.aten.empty, torch.ops.aten.empty_strided):
            self.bytes += r.untyped_storage().nbytes()
        return r


def calls(ip, rows):  # noqa: F811
    x = torch.randn(rows, 100, device="cuda").bfloat16()
    g, ws = torch.ones(100, device="cuda").bfloat16(), torch.zeros(256, dtype=torch.uint8, device="cuda")
    w8, w4 = ip.quantize_rows_i8(torch.randn(64, 100, device="cuda")), ip.quantize_fp4(torch.randn(64, 100, device="cuda"))
    x8, x4 = ip.quantize_rows_i8(x), ip.quantize_fp4(x)
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    return {"quantize_rows_i8": lambda: ip.quantize_rows_i8(x), "linear_scaled_i8": lambda: ip.linear_scaled_i8(*x8, *w8, workspace=ws),
            "quantize_fp4": lambda: ip.quantize_fp4(x), "linear_fp4": lambda: ip.linear_fp4(*x4, *w4, workspace=ws),
            "rmsnorm_i8": lambda: ip.rmsnorm_i8(x, g, x), "rmsnorm_fp4": lambda: ip.rmsnorm_fp4(x, g, x),
            "dequantize_i8": lambda: ip.dequantize_i8(*x8), "dequantize_fp4": lambda: ip.dequantize_fp4(*x4),
            "token_logprobs": lambda: ip.token_logprobs(x, tok, top=3, workspace=ws)}


@pytest.mark.parametrize("rows", [5, 5000])
def test_the_dispatcher_sees_new_outputs(ip, rows):  # noqa: F811
    for name, call in calls(ip, rows).items():
        with Made() as made:
            out = call()
        out = [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]
        assert made.bytes >= sum(t.numel() * t.element_size() for t in out), name


def test_the_cache_s_calls(ip):  # noqa: F811
    page, L, H = 64, 128, 2
    cache = ip.kv4_cache(4, H, page)
    table = torch.tensor([[0, 1]], device="cuda", dtype=torch.int32)
    lengths = torch.tensor([L], device="cuda", dtype=torch.int32)
    k = torch.randn(1, L, H, 128, device="cuda").bfloat16()
    ip.kv4_append(k, k, lengths - L, table, cache)
    ws = torch.zeros(ip.kv4_attention_workspace_bytes(1, 1, H, H, L), dtype=torch.uint8, device="cuda")
    q = torch.randn(1, 1, H, 128, device="cuda").bfloat16()
    with Made() as made:
        y = ip.kv4_attention(q, lengths, table, cache, max_len=L, workspace=ws)
        a, b = ip.kv4_read(cache, lengths - L, table, L)
    assert made.bytes >= sum(t.numel() * t.element_size() for t in (y, a, b))


def test_memory_is_filled_where_asked_for(ip):  # noqa: F811
    fill = torch.utils.deterministic.fill_uninitialized_memory
    for rows in (5, 3000):
        x = torch.randn(rows, 1000, device="cuda")
        junk = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
        del junk                     # what a new allocation would find
        try:
            torch.use_deterministic_algorithms(True)
            torch.utils.deterministic.fill_uninitialized_memory = True
            blocks = ip.quantize_fp4(x)[1]
        finally:
            torch.use_deterministic_algorithms(False)
            torch.utils.deterministic.fill_uninitialized_memory = fill
        assert (blocks[ref.untouched(blocks, rows)] == 255).all()


def test_a_profiler_sees_new_outputs(ip):  # noqa: F811
    for name, call in calls(ip, 5).items():
        call()
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as prof:
            call()
        assert any(e.name in ("aten::empty", "aten::empty_strided") for e in prof.events()), name


def test_no_memory_no_call(ip):  # noqa: F811
    # tensors made under this mode have none: a call with them fails on the host
    from torch._subclasses.fake_tensor import FakeTensorMode
    for name, call in calls(ip, 5).items():
        with pytest.raises(Exception):
            with FakeTensorMode(allow_non_fake_inputs=True):
                call()
    torch.cuda.synchronize()


def test_what_a_new_output_is(ip):  # noqa: F811
    # in its own right: an ordinary tensor, whichever way it was made
    for name, call in calls(ip, 5).items():
        for mode in (torch.inference_mode(), torch.no_grad(), torch.autocast("cuda", torch.bfloat16)):
            plain = call()
            with mode:
                under = call()
            for a, b in zip(*((r if isinstance(r, tuple) else (r,)) for r in (plain, under))):
                if a is not None:
                    assert type(a) is type(b) is torch.Tensor and not a.requires_grad and a.shape == b.shape and a.stride() == b.stride()
                    assert a.is_inference() is False and b.is_inference() is isinstance(mode, torch.inference_mode)
                    a.add_(1)        # in place, with the version counter that this takes
                    assert a._version == 1
