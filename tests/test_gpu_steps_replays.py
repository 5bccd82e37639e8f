"""Steps of several tokens a request in graphs that are replayed with other inputs, in
two calls at once, on the library's own workspace as it grows, and the shared-key
prompt kernel with more requests than a wave sorts."""
import numpy as np
import pytest

from oracle import steps as O
from test_gpu_steps import SCALE, check, dev, device, oracle, prompts, run_prompts, steps, torch, trees  # noqa: F401
from test_gpu_steps_blocks import pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes,Hq,Hkv", [([8, 4, 3], 4, 1), ([16, 5, 9], 8, 2), ([32, 30, 1], 4, 1), ([64, 20, 40], 8, 2)])
def test_tree_replayed_with_other_lengths(torch, steps, nodes, Hq, Hkv):  # noqa: F811
    """Each replay against the oracle on what the buffers hold then."""
    c = trees([700, 20, 300], nodes, Hq, Hkv, 71, pad=2)
    args = device(torch, c)
    out = torch.empty_like(args[0])
    lse = torch.empty(c["q"].shape[:2], dtype=torch.float32, device="cuda")
    workspace = torch.empty(steps.tree_workspace_bytes(c["max_nodes"], Hq, Hkv), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps.tree_attention(*args, SCALE, out=out, lse_out=lse, workspace=workspace)
    for lens, counts in (([700, 20, 300], nodes), ([0, 20, 1], nodes), ([655, 17, 0], nodes[::-1]), ([3, 20, 290], [nodes[0], 0, 1]),
                         ([0, 0, 0], [1, 1, 1]), ([700, 20, 300], nodes)):
        now = dict(c, lens=np.array(lens, np.int32), offsets=np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
        rng = np.random.default_rng(sum(lens))
        for name in ("q", "k", "v"):
            now[name] = rng.standard_normal(c[name].shape).astype(np.float16)
        fresh = device(torch, now)
        for i in (0, 1, 2, 3, 8):
            assert args[i].shape == fresh[i].shape
            args[i].copy_(fresh[i])
        out.fill_(7)
        lse.fill_(7)
        workspace.fill_(255)
        eager = steps.tree_attention(*fresh, SCALE)
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        rows = check(oracle(now), got, lse.cpu().numpy(), SCALE)
        end = sum(counts)
        assert rows[:end].all() and (got[end:] == 7).all()
        assert torch.equal(out[:end], eager[:end])


def test_extend_and_release_replayed_with_other_lengths(torch, steps):  # noqa: F811
    """New tokens get their blocks, then what is not kept goes back: one graph."""
    bs, width, rng = 16, 40, np.random.default_rng(72)
    B, T = 70, 1400
    lens = rng.integers(0, 200, B).astype(np.int32)
    table, free, height, nb = pool(rng, lens, width, bs, 300)
    d_lens, d_news, d_keeps, d_table, d_free, d_state = dev(torch, lens, np.zeros(B, np.int32), np.zeros(B, np.int32), table, free,
                                                            np.array([height, 0], np.int32))
    plan = steps.empty_plan(B, T, "cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        steps.extend(d_lens, d_news, d_table, d_free, d_state, T, plan=plan)
        steps.release(plan.total_lens, d_keeps, d_table, d_free, d_state)
    for i in range(6):
        news = rng.integers(0, [1, 20, 40, 2, 0, 20][i] + 1, B).astype(np.int32)
        keeps = np.maximum(lens + news - rng.integers(0, 100, B), 0).astype(np.int32)
        if i == 3:
            keeps[:] = 0
        for t, x in ((d_lens, lens), (d_news, news), (d_keeps, keeps)):
            t.copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        s.synchronize()
        table, height, offsets, totals, slots, positions = O.extend(lens, news, table, free, height, T, nb, bs)
        for got, want in zip(plan, (offsets, totals, slots, positions)):
            assert np.array_equal(got.cpu().numpy(), want)
        table, free, height = O.release(totals, keeps, table, free, height, nb, bs)
        assert np.array_equal(d_table.cpu().numpy(), table) and d_state.tolist() == [height, 0]
        assert np.array_equal(d_free.cpu().numpy()[:height], free[:height])
        lens = np.minimum(totals, keeps).astype(np.int32)


def test_two_calls_at_once(torch, steps):  # noqa: F811
    """Prompts, and blocks of two pools, on two streams."""
    cases = [prompts([500, 70], 8, 2, 73), prompts([30, 600, 9], 8, 2, 74)]
    args = [dev(torch, *c) for c in cases]
    alone = [steps.prompt_attention(*a, SCALE) for a in args]
    outs = [torch.empty_like(a[0]) for a in args]
    rng = np.random.default_rng(75)
    pools, wants = [], []
    for i in range(2):
        lens, news = rng.integers(0, 90, 50 + i).astype(np.int32), rng.integers(0, 90, 50 + i).astype(np.int32)
        table, free, height, nb = pool(rng, lens, 12, 16, 400)
        pools.append(dev(torch, lens, news, table, free, np.array([height, 0], np.int32)))
        e = O.extend(lens, news, table, free, height, 5000, nb, 16)
        wants.append((e, O.release(e[3], np.zeros_like(lens), e[0], free, e[1], nb, 16)))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    plans = []
    for a, o, p, s in zip(args, outs, pools, streams):
        for _ in range(5):
            steps.prompt_attention(*a, SCALE, out=o, stream=s)
        with torch.cuda.stream(s):
            plans.append(steps.extend(*p, 5000))
            steps.release(plans[-1].total_lens, torch.zeros_like(p[0]), *p[2:])
    torch.cuda.synchronize()
    for o, ref, p, plan, (e, r) in zip(outs, alone, pools, plans, wants):
        assert torch.equal(o, ref)
        assert np.array_equal(plan.slot_mapping.cpu().numpy(), e[4])
        assert np.array_equal(p[2].cpu().numpy(), r[0]) and np.array_equal(p[3].cpu().numpy(), r[1]) and p[4].tolist() == [r[2], 0]


def test_the_librarys_workspace_grows_and_goes(torch, steps):  # noqa: F811
    """Calls without a workspace, of pairs that need more each time, and after a release."""
    cases = [trees([300, 9], nodes, 8, 2, 76) for nodes in ([3, 2], [16, 5], [32, 9], [64, 60])]
    steps.release_workspace()
    for c in cases + cases[::-1]:
        out = steps.tree_attention(*device(torch, c), SCALE)
        check(oracle(c), out.cpu().numpy(), None, SCALE)
    steps.release_workspace()
    out = steps.tree_attention(*device(torch, cases[0]), SCALE)
    check(oracle(cases[0]), out.cpu().numpy(), None, SCALE)


@pytest.mark.parametrize("B,low,high", [(65, 200, 320), (70, 1, 540), (90, 0, 560)])
def test_many_prompts_whose_keys_two_waves_share(torch, steps, B, low, high):  # noqa: F811
    """More than 64 requests of 256 tokens and more on the average, one head."""
    rng = np.random.default_rng(B)
    lens = rng.integers(low, high + 1, B)
    lens[-1] += max(0, 257 * B - lens.sum())
    assert 256 * B <= lens.sum() and lens.sum() // 128 + B <= 320      # the rule of that kernel on 256 compute units
    q, k, v, offsets = prompts(lens.tolist(), 1, 1, B)
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    assert check(O.prompt(q, k, v, offsets, SCALE), got, lse, SCALE).all()
