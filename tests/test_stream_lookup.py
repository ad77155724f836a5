"""The current stream's handle without torch's raw lookups (underscore names that
a torch may lack) and without an initialised device: the public way."""
import pytest
import torch

from paper_2606_20537_amd import _native as N


class Stream:
    cuda_stream = 77


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_torch_without_raw_lookups(monkeypatch, missing):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    monkeypatch.delattr(torch._C, missing, raising=False)
    monkeypatch.setattr(N, "_raw", None)
    assert N._stream(None) == 77 and N._stream(None) == 77


@pytest.mark.parametrize("initialised", [False, True])
def test_raw_lookups_only_when_initialised(monkeypatch, initialised):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: initialised)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(N, "_raw", None)
    assert N._stream(None) == (1003 if initialised else 77)
    assert N._stream(5) == 5 and N._stream(Stream) == 77


@pytest.mark.parametrize("handle, stream", [(77, None), (5, "external 5"), (2, "external 2"), (0, "default"), (1, "default")])
def test_scratch_belongs_to_the_stream_of_the_call(monkeypatch, handle, stream):
    """A workspace allocated for one call is of the pool of the stream that the call launches on: torch hands memory of
    the current stream's pool to the next allocation there, while the call's kernels still use it."""
    under, made = [], []

    class Under:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            under.append(self.s)

        def __exit__(self, *_):
            under.pop()

    monkeypatch.setattr(N, "_raw", ())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: "default")
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: "external %d" % handle)
    monkeypatch.setattr(torch.cuda, "stream", Under)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: made.append((a, kw, list(under))))
    N._scratch(100, "cuda:0", handle)
    assert made == [((100,), dict(dtype=torch.uint8, device="cuda:0"), [stream] if stream else [])]


@pytest.mark.parametrize("name", ["kvb_attend", "kvb_select"])
def test_calls_take_their_scratch_on_their_stream(monkeypatch, name):
    """The two calls that allocate a workspace hand their own stream on, another than the current one too."""
    import ctypes as ct

    class Lib:
        def kvb_attend_workspace_bytes(self, a):
            return 640
        kvb_select_workspace_bytes = kvb_attend_workspace_bytes

        def kvb_attend(self, a, handle):
            args = ct.cast(a, ct.POINTER(getattr(N, name + "_args"))).contents
            called.append((args.workspace, args.workspace_bytes, handle))
            return 0
        kvb_select = kvb_attend

    called, asked = [], []
    scratch = torch.zeros(640, dtype=torch.uint8)
    monkeypatch.setattr(N, "load", lambda: Lib())
    monkeypatch.setattr(N, "_kvb_device", lambda *a: None)
    monkeypatch.setattr(N, "_scratch", lambda need, device, handle: asked.append((need, handle)) or scratch, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    t = N.kvb_seqs([[0, 0, 0, 0, 0, 64, 3, 3]])
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    if name == "kvb_attend":
        N.kvb_attend(t, q, torch.empty_like(q), kv_heads=2, scale=1.0, stream=5)
    else:
        N.kvb_select(t, q, torch.zeros((3, 2, 4), dtype=torch.int32), kv_heads=2, stream=5)
    assert asked == [(640, 5)] and called == [(scratch.data_ptr(), 640, 5)]


def test_delta_rule_prefill_takes_its_scratch_on_its_stream(monkeypatch):
    """The delta-rule prefill likewise."""
    import ctypes as ct

    class Lib:
        def gdn_workspace_bytes(self, T, H, chunk):
            return 640

        def gdn_chunked_prefill(self, a, handle):
            args = ct.cast(a, ct.POINTER(N.gdn_args)).contents
            called.append((args.workspace, args.workspace_bytes, handle))
            return 0

    called, asked = [], []
    scratch = torch.zeros(640, dtype=torch.uint8)
    monkeypatch.setattr(N, "load", lambda: Lib())
    monkeypatch.setattr(N, "_scratch", lambda need, device, handle: asked.append((need, handle)) or scratch)
    q, g = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 4))
    N.gdn_chunked_prefill(q, q, q, g, g, torch.zeros((3, 4, 64)), stream=5)
    assert asked == [(640, 5)] and called == [(scratch.data_ptr(), 640, 5)]
