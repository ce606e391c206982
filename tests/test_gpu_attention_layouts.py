"""Gradients into interleaved layouts: the bits of gradients into tensors of their own."""
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [32, 128])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("S,Sk", [(1, 1), (1, 70), (150, 150)])
def test_interleaved_gradients(S, Sk, bf16, hd):
    import torch
    from paper_2606_30634_amd import attention as T
    log(f"S {S} Sk {Sk} bf16 {bf16} hd {hd}")
    B, H, KV = 3, 4, 2
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator(device="cuda:0").manual_seed(S + hd)
    q, k, v, do = (torch.randn(B, s, h, hd, generator=g, device="cuda:0").to(dt) for s, h in ((S, H), (Sk, KV), (Sk, KV), (S, H)))
    f = T.attention(q, k, v, keep_f32=bf16)
    want = T.attention_backward(q, k, v, f, do)

    def buf(*shape):
        return torch.full(shape, float("nan"), dtype=dt, device="cuda:0")

    layouts = []
    if S == Sk:
        p = buf(B, S, H + 2 * KV, hd)
        layouts.append((p[:, :, :H], p[:, :, H:H + KV], p[:, :, H + KV:]))
        p = buf(S, B, H + 2 * KV, hd).transpose(0, 1)
        layouts.append((p[:, :, :H], p[:, :, H:H + KV], p[:, :, H + KV:]))
        p = buf(B, H + 2 * KV, S, hd).transpose(1, 2)
        layouts.append((p[:, :, :H], p[:, :, H:H + KV], p[:, :, H + KV:]))
    p = buf(B, Sk, KV, 2, hd)
    layouts.append((buf(B, S, H, hd), p[..., 0, :], p[..., 1, :]))
    p = buf(B, Sk, 2 * KV, hd)
    layouts.append((buf(B, S, H, hd), p[:, :, :KV], p[:, :, KV:]))
    for out in layouts:
        got = T.attention_backward(q, k, v, f, do, out=out)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
