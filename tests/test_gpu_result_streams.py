"""Results that a call allocates come from the pool of the stream that it works
on: a block of another stream could still be in use there, and would go back there
while the call writes it."""
import numpy as np
import pytest

from test_gpu_kv4 import BS, case, dev, kv4, torch  # noqa: F401  (two are fixtures)

pytestmark = pytest.mark.gpu


def check_pool(torch, call):  # noqa: F811
    """call(stream) returns results of 16 MiB or more, each a segment of its own.
    With nothing else cached, a block that the current stream frees is the first
    choice for a result of its size there."""
    s = torch.cuda.Stream()
    want = [x.clone() for x in call(None)]
    torch.cuda.synchronize()
    n = [x.numel() for x in want]
    assert all(x.dtype is torch.float16 and x.numel() >= 1 << 23 for x in want)

    def blocks():
        return [torch.empty(k, dtype=torch.float16, device="cuda") for k in n]

    torch.cuda.empty_cache()
    held = blocks()
    own = {x.data_ptr() for x in held}
    del held
    got = call(s)
    assert not own & {x.data_ptr() for x in got}
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # dropped, they go back to the call's stream
    theirs = {x.data_ptr() for x in got}
    del got
    assert not theirs & {x.data_ptr() for x in blocks() + blocks()}
    with torch.cuda.stream(s):
        assert theirs & {x.data_ptr() for x in blocks()}


def test_kv4_gather(torch, kv4):  # noqa: F811
    _, cache, table, lens = case([300], 8, 8, seed=1)
    dc, = dev(torch, cache)
    slots = torch.from_numpy(np.resize(table[0, :1].astype(np.int64) * BS + np.arange(BS), 10000)).cuda()
    check_pool(torch, lambda s: kv4.gather(dc, slots, stream=s))


def test_kv4_attention(torch, kv4):  # noqa: F811
    q, cache, table, lens = case([20], 8, 1, seed=2)
    B = 9000
    dq, dc, dt, dl = dev(torch, np.repeat(q, B, 0), cache, np.repeat(table, B, 0), np.repeat(lens, B))
    ws = torch.zeros(kv4.attention_workspace_bytes(B, 8, 1), dtype=torch.uint8, device="cuda")
    check_pool(torch, lambda s: [kv4.attention(dq, dc, dt, dl, 0.1, workspace=ws, stream=s)])


@pytest.fixture(scope="module")
def apex():
    import paper_2506_03296_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("name", ["decode_attention", "decode_attention_ex"])
def test_decode_attention(torch, apex, name):  # noqa: F811
    B = 9000
    q = torch.randn((1, 8, 128), device="cuda").half().repeat(B, 1, 1)
    k, v = (torch.randn((2, 1, BS, 128), device="cuda").half() for _ in range(2))
    bt = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda").repeat(B, 1)
    lens = torch.full((B,), 20, dtype=torch.int32, device="cuda")
    check_pool(torch, lambda s: [getattr(apex, name)(q, k, v, bt, lens, 0.1, stream=s)])
