"""Calls on rows of logits from several threads at once, each on its own stream: what the library keeps per thread does not mix."""
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
