"""Calls on rows of logits from several threads at once, each on its own stream: what the library keeps per thread does not mix.  And rows far apart."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def work(seed):
    """Calls of several sizes, so of several launch shapes; returns all outputs."""
    from paper_2505_19201_b200 import api
    out = []
    for i, (R, V) in enumerate([(1, 32000), (5, 262144), (40, 9001), (300, 777), (12, 131072), (700, 4000)]):
        dtype = torch.bfloat16 if (seed + i) % 2 else torch.float32
        g = torch.Generator(device="cuda").manual_seed(100 * seed + i)
        x = (torch.randn(R, V, device="cuda", generator=g) * 2).to(dtype)
        u = torch.rand(R, device="cuda", generator=g)
        tok, kept = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
        api.dream_sample(x, u, tok, top_p=torch.full((R,), 0.9, device="cuda"), kept=kept)
        cut = torch.zeros_like(x)
        api.dream_truncate_logits(x, cut, top_k=torch.full((R,), 30, dtype=torch.int32, device="cuda"))
        top, ids = torch.topk(x.float(), 16, dim=1)
        loss, lse, grad, back = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda"), torch.zeros_like(x), torch.zeros_like(x)
        api.dream_distill_loss(x, ids.int(), top, loss, lse, grad=grad)
        api.dream_distill_grad(x, ids.int(), top, lse, back)
        out += [tok, kept, cut, loss, lse, grad, back]
    torch.cuda.current_stream().synchronize()
    return [t.cpu() for t in out]


def test_threads():
    want = [work(s) for s in range(4)]
    got, failed = [None] * 4, []

    def run(s):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(3):
                    got[s] = work(s)
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=run, args=(s,)) for s in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_beyond_32_bits(dtype):
    """Three rows 2^30 elements and a little apart: offsets pass 2^31 elements.  The same as of three rows side by side, bit by bit."""
    from paper_2505_19201_b200 import api
    R, V, ld = 3, 20008, 2 ** 30 + 64
    if torch.cuda.mem_get_info()[0] < 26 << 30:
        pytest.skip("less than 26 GB free on the device")
    far = [torch.empty(2 * ld + V, dtype=dtype, device="cuda").as_strided((R, V), (ld, 1)) for _ in range(2)]
    near = [torch.empty(R, V, dtype=dtype, device="cuda") for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(R, V, device="cuda", generator=g) * 2
    u, tk = torch.rand(R, device="cuda", generator=g), torch.full((R,), 40, dtype=torch.int32, device="cuda")
    top, ids = torch.topk(x, 9, dim=1)
    res = []
    for src, dst in (far, near):
        src.copy_(x)
        tok, lp = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")
        loss, lse = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
        api.dream_sample(src, u, tok, logprob=lp)
        out = [tok, lp, loss, lse]
        for call in (lambda: api.dream_truncate_logits(src, dst, top_k=tk), lambda: api.dream_distill_loss(src, ids.int(), top, loss, lse, grad=dst),
                     lambda: api.dream_distill_grad(src, ids.int(), top, lse, dst)):
            dst.fill_(7.0)
            call()
            out.append(dst.clone().contiguous())
        res.append([t.cpu() for t in out])
    assert all(torch.equal(a, b) for a, b in zip(*res))
