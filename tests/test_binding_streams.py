"""What the binding allocates for a call on a given stream belongs to that stream.
The library's launches are replaced by functions that do nothing, so this runs
without a GPU."""
import contextlib

import pytest
import torch

dar = pytest.importorskip("paper_2606_18587_amd", reason="libdar.so not built")

BF = torch.bfloat16
B, HQ, HKV, D, DD, W, T = 2, 4, 2, 64, 16, 8, 40


class FakeStream:
    cuda_stream = 0x1234
    device = torch.device("cpu")


class Launches:
    """The library with every entry point that would launch replaced."""

    def __init__(self, real):
        self.real, self.streams = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)

        def call(*args):
            self.streams.append(args[-1])
            return dar.DAR_OK
        return call


def zeros(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def dense(shared=False):
    c = dar.DarCache(B, HKV, D, DD, W, 100, BF, device="cpu", shared=shared)
    c.struct.len = 60
    return c


def paged():
    return dar.DarPagedCache(B, HKV, D, DD, W, 32, 4, 8, BF, device="cpu")


def rope():
    return dar.Rope(16, n_pos=512, table=zeros(512, 16, dtype=torch.float32))


Q, K, WD, WU = zeros(B, HQ, T, D), zeros(B, HKV, T, D), zeros(HKV, D, DD), zeros(HKV, DD, D)
Q1, C, LSE = zeros(B, HQ, D), zeros(B, HKV, T, DD), zeros(B, HQ, T, dtype=torch.float32)
SC, SCP = zeros(B, HKV, 100, dtype=torch.float32), zeros(B, HKV, 128, dtype=torch.float32)
BLOCKS = torch.zeros(2, dtype=torch.int32)

CALLS = {
    "prefill": lambda s: dar.dar_attn_prefill(Q, K, K, WD, None, W, stream=s, return_lse=True),
    "prefill_rope": lambda s: dar.dar_attn_prefill_rope(Q, K, K, WD, None, W, rope(), stream=s, return_lse=True),
    "prefill_shared": lambda s: dar.dar_attn_prefill_shared(Q, K, K, C, WU, WU, W, stream=s, return_lse=True),
    "backward": lambda s: dar.dar_attn_prefill_backward(Q, K, K, WD, WU, W, Q, LSE, Q, stream=s),
    "rope_backward": lambda s: dar.dar_attn_prefill_rope_backward(Q, K, K, WD, WU, W, rope(), Q, LSE, Q, stream=s),
    "chunk": lambda s: dar.dar_attn_prefill_chunk(dense(), Q, K, K, WD, stream=s, return_lse=True),
    "chunk_rope": lambda s: dar.dar_attn_prefill_chunk_rope(dense(), Q, K, K, WD, rope(), stream=s, return_lse=True),
    "chunk_paged": lambda s: dar.dar_attn_prefill_chunk_paged(paged(), Q, K, K, WD, stream=s, return_lse=True),
    "decode": lambda s: dar.dar_attn_decode(dense(), Q1, WD, stream=s),
    "decode_noalloc": lambda s: dar.dar_attn_decode_noalloc(dense(), Q1, WD, stream=s),
    "decode_rope": lambda s: dar.dar_attn_decode_rope(dense(), Q1, WD, rope(), stream=s),
    "decode_shared": lambda s: dar.dar_attn_decode_shared(dense(True), Q1, WU, WU, stream=s),
    "decode_paged": lambda s: dar.dar_attn_decode_paged(paged(), Q1, WD, stream=s),
    "decode_paged_rope": lambda s: dar.dar_attn_decode_paged_rope(paged(), Q1, WD, rope(), stream=s),
    "rope_table": lambda s: dar.dar_rope_table(16, 10000.0, 512, device="cpu", stream=s),
    "scored": lambda s: dar.dar_attn_decode_scored(dense(), Q1, WD, SC, stream=s),
    "paged_scored": lambda s: dar.dar_attn_decode_paged_scored(paged(), Q1, WD, SCP, stream=s),
    "paged_prefix": lambda s: dar.dar_attn_decode_paged_prefix(paged(), Q1, WD, BLOCKS, stream=s),
    "evict": lambda s: dar.dar_cache_evict(dense(), SC, 8, stream=s),
    "evict_paged": lambda s: dar.dar_cache_evict_paged(paged(), SCP, 8, stream=s),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations_belong_to_the_stream(monkeypatch, name):
    current, taken = [], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def watched(real):
        def make(*args, **kw):
            taken.append(current[-1] if current else None)
            return real(*args, **kw)
        return make

    launches, stream = Launches(dar.lib), FakeStream()
    monkeypatch.setattr(dar, "lib", launches)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", watched(torch.empty))
    monkeypatch.setattr(torch, "empty_like", watched(torch.empty_like))
    CALLS[name](stream)
    assert launches.streams == [stream.cuda_stream]
    assert taken and all(s is stream for s in taken)


def test_a_stream_of_another_device_is_refused():
    """Checked before anything else by the serving operators."""
    other = FakeStream()
    other.device = torch.device("cuda", 1)
    for name in ("scored", "paged_scored", "paged_prefix", "evict", "evict_paged"):
        with pytest.raises(ValueError, match="stream"):
            CALLS[name](other)
