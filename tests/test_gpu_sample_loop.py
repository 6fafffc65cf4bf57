"""Truncated sampling in the decode loop: the first token is drawn, the verification's logits are cut, and the acceptance follows what
is left of the target's distribution."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _start(preset="toy", **over):
    from paper_2505_19201_b200 import api, configs, synth
    dev = "cuda:0"
    p = configs.scaled(preset, **over)
    ctx = api.Context(api.make_config(p), synth.target_weights(p, 0, dev), synth.draft_weights(p, 0, dev), dev)
    vis, ids = synth.request_inputs(p, 0, dev)
    return p, ctx, vis, ids


def test_first_token_is_drawn_from_the_prompts_logits():
    """Against the oracle's logits.  The two sides' logits differ by up to 1e-3 (Tol of the fp32 parity), which moves the running sum of a
    nearly uniform row of 1024 by up to 1e-3 / temperature, some three tokens."""
    from tests.parity import Pair
    from tests.test_gpu_sample import kept_ids
    pr = Pair("toy")
    try:
        p, ctx = pr.p, pr.ctx
        from paper_2505_19201_b200 import synth
        vis, ids = synth.request_inputs(p, 0, "cuda:0")
        _, otok, _ = pr.orc.prefill(vis.cpu().to(pr.odt), 0, ids.cpu().tolist())
        lg = pr.orc._logits(pr.orc._last_hidden[-1:])[0].double()
        tok, lp = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
        ctx.dream_prefill(0, vis, 0, ids)
        for u in (0.01, 0.2, 0.43, 0.61, 0.87, 0.99):
            for s in (dict(temperature=1.0), dict(temperature=0.3, top_k=20), dict(temperature=0.7, top_p=0.8), dict(temperature=0.5, top_k=30, min_p=0.3)):
                ctx.dream_sample_first(0, torch.tensor([u], device="cuda"), first_token=tok, logprob=lp, **s)
                ctx.dream_poll()
                assert ctx.dream_seq_state(0)[1] == int(tok)            # the pending token is the one drawn
                keep, w = kept_ids(lg, s["temperature"], s.get("top_k", 0), s.get("top_p", 1.0), s.get("min_p", 0.0))
                srt = torch.sort(keep).values
                run = torch.cumsum(w[srt], 0) / w[srt].sum()
                if len(s) > 1:
                    assert int(tok) in set(torch.sort(lg, descending=True).indices[:keep.numel() + 8].tolist())
                    continue                                             # the cut itself may differ by a token at its edge
                i = int((run <= u).sum())
                assert int(tok) in srt[max(0, i - 3):i + 4].tolist()
        ctx.dream_sample_first(0, torch.tensor([0.7], device="cuda"), temperature=1.0, top_k=1, first_token=tok, logprob=lp)
        ctx.dream_poll()
        assert int(tok) == otok and float(lp) == 0.0
    finally:
        pr.close()


def test_drawn_first_token_reaches_the_draft():
    p, ctx, vis, ids = _start()
    try:
        tok = torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.dream_prefill(0, vis, 0, ids)
        ctx.dream_sample_first(0, torch.tensor([0.9], device="cuda"), temperature=2.0, first_token=tok)
        ctx.dream_compress_visual(0, p["k_visual"])
        tree = ctx.new_tree()
        ctx.dream_draft_tree([0], [tree])
        ctx.dream_poll()
        assert int(tree.tokens[0]) == int(tok)
    finally:
        ctx.close()


def test_first_token_refusals():
    from paper_2505_19201_b200 import api
    p, ctx, vis, ids = _start(batch=2)
    try:
        u = torch.tensor([0.5], device="cuda")
        code = lambda *a, **k: _code(api, ctx.dream_sample_first, *a, **k)  # noqa: E731
        assert code(0, u) == -2                                          # nothing prefilled
        ctx.dream_prefill(0, vis, 0, ids)
        assert code(0, None) == -1 and code(0, u, temperature=0.0) == -1 and code(0, u, temperature=float("nan")) == -1
        assert code(5, u) == -1
        ctx.dream_prefill(1, vis, 0, ids)
        assert code(0, u) == -2                                          # another prompt has been read since
        assert code(1, u) == 0
        ctx.dream_compress_visual(1, p["k_visual"])
        assert code(1, u) == -2
        ctx.dream_poll()
    finally:
        ctx.close()


def _code(api, fn, *a, **k):
    try:
        fn(*a, **k)
    except api.DreamError as e:
        return e.code
    return 0


@pytest.mark.parametrize("preset,over", [("toy", {}), ("smolvlm2b", dict(n_layers=2, n_visual=96, k_visual=24, n_prompt=40, decode_steps=4))])
def test_rounds_on_a_truncated_target(preset, over):
    """Verify, cut in place, accept: every emitted token is one that its node's row kept, draft tokens among them only where kept, and with one
    token kept per row the walk is the greedy one."""
    from paper_2505_19201_b200 import api
    p, ctx, vis, ids = _start(preset, **over)
    try:
        dev, T, D, V = "cuda:0", ctx.T, p["tree_depth"], p["vocab"]
        full = lambda v, kind=torch.float32: torch.full((T,), v, dtype=kind, device=dev)  # noqa: E731
        am, alen = torch.zeros(T, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
        out, src = torch.zeros(D + 1, dtype=torch.int32, device=dev), torch.zeros(D + 1, dtype=torch.int32, device=dev)
        lg, kept = torch.zeros(T, V, device=dev), torch.zeros(T, dtype=torch.int32, device=dev)
        ctx.dream_prefill(0, vis, 0, ids)
        ctx.dream_sample_first(0, torch.tensor([0.3], device=dev), temperature=0.8, top_k=40, top_p=0.95)
        ctx.dream_compress_visual(0, p["k_visual"])
        g = torch.Generator(device=dev).manual_seed(5)
        for rnd in range(3):
            tree = ctx.new_tree()
            ctx.dream_draft_tree([0], [tree])
            ctx.dream_verify_tree([0], [tree], am, None, lg)
            whole = lg.clone()
            if rnd < 2:
                api.dream_truncate_logits(lg, lg, temperature=full(0.8), top_k=full(40, torch.int32), top_p=full(0.95), kept=kept)
            else:
                api.dream_truncate_logits(lg, lg, top_k=full(1, torch.int32), kept=kept)
            ctx.dream_accept_sample([0], [tree], lg, 0.8, torch.rand(D + 1, T, device=dev, generator=g), alen, out, src)
            ctx.dream_poll()
            A, toks, path = int(alen), out.tolist(), src.tolist()
            assert bool((kept >= 1).all()) and bool((kept <= (40 if rnd < 2 else 1)).all())
            assert torch.equal((lg > float("-inf")).sum(1).int(), kept)
            assert bool(((lg == whole) | (lg == float("-inf"))).all())
            for j in range(A + 1):
                assert float(lg[path[j], toks[j]]) > float("-inf")
            if rnd == 2:
                assert toks[A] == int(am[path[A]])
    finally:
        ctx.close()
