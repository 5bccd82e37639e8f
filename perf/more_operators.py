"""Timed cases of the calls for steps with several new tokens a request: what they
are, how their inputs are made, one pass of each (in plain torch operations, or
through the library), and the same result in 64 bits.

  extend   cache blocks for the new tokens of a batch, taken from the free ones,
           and the tokens' slots, positions and offsets
  release  blocks of tokens that are dropped, given back
  prompt   causal attention of packed prompts over themselves
  tree     attention of drafted tokens over a paged cache and, by a mask, over
           each other

Request lengths and counts of drafted tokens belong to the case (drawn from its
`lens_seed`); block placement, the shapes of trees and all values come from the
seed that `prepare` is given.
"""
import math

import numpy as np
import torch

own = False

D = 128
BS = 16
SCALE = float(np.float32(1.0 / math.sqrt(D)))


def _case(name, kind, B, lens, lo, hi, lens_seed, **more):
    return dict(name=name, kind=kind, B=B, lens=lens, lo=lo, hi=hi, lens_seed=lens_seed, **more)


def listed():
    return [
        # One decode step's slots: one token a request, a block now and then.
        _case("extend_decode", "extend", 32, "uniform", 1024, 4096, 1, new_lo=1, new_hi=1),
        # Prompts about to be written: about 55 000 tokens of 24 requests, in a
        # batch that is padded to whole buckets.
        _case("extend_prompts", "extend", 24, "uniform", 0, 0, 2, new_lo=512, new_hi=4096, bucket=8192),
        # What a speculative step leaves over: a few tokens of many requests.
        _case("release_trim", "release", 128, "uniform", 1024, 4096, 3, drop=0.01),
        # A long-output batch that ends as a whole.
        _case("release_batch", "release", 32, "lognormal", 4096, 32768, 4, drop=1.0),
        # One short question on Llama-3.1-8B heads: launch and latency.
        _case("prompt_one_short", "prompt", 1, "uniform", 61, 61, 5, Hq=32, Hkv=8),
        # Chat prompts of different lengths in one call, read out of a fused
        # projection buffer, with their log-sum-exp.
        _case("prompt_chat", "prompt", 16, "uniform", 64, 1024, 6, Hq=32, Hkv=8, lse=True, fused=True),
        # Llama-2-7B heads (every q-head has its own kv-head), ragged.
        _case("prompt_mha_ragged", "prompt", 8, "spread", 33, 4095, 7, Hq=32, Hkv=32),
        # One long document.
        _case("prompt_long", "prompt", 1, "uniform", 32768, 32768, 8, Hq=32, Hkv=8),
        # Eight drafted tokens of a single short request: launch and latency.
        _case("tree_one_short", "tree", 1, "uniform", 511, 511, 9, Hq=32, Hkv=8, new_lo=8, new_hi=8),
        # A chat batch with trees of up to 32 nodes, with their log-sum-exp.
        _case("tree_chat", "tree", 16, "uniform", 256, 4096, 10, Hq=32, Hkv=8, new_lo=5, new_hi=32, lse=True),
        # Full trees of 64 nodes on Llama-2-7B heads.
        _case("tree_mha_full", "tree", 16, "uniform", 512, 2048, 11, Hq=32, Hkv=32, new_lo=64, new_hi=64),
        # The long-output batch of Llama-3.1-8B heads, eight nodes a request.
        _case("tree_long_output", "tree", 32, "lognormal", 4096, 32768, 12, Hq=32, Hkv=8, new_lo=8, new_hi=8),
    ]


# q-heads and kv-heads: the models the repository names, one rank's share of
# them, and groups that are no power of two
_HEADS = [(32, 32), (32, 8), (32, 8), (64, 8), (32, 16), (16, 4), (8, 2), (4, 1), (16, 16), (8, 1), (12, 4), (14, 2)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["extend", "release"] + ["prompt"] * 4 + ["tree"] * 4)
        lens = rng.choice(["uniform", "uniform", "lognormal", "bimodal", "spread"])
        B = _log(rng, 1, 512 if kind in ("extend", "release") else 128)
        hi = _log(rng, 16, 32768 if B <= 64 else 8192)
        lo = hi if rng.random() < 0.15 else max(1, int(hi * rng.uniform(0.02, 0.6)))
        c = dict(kind=kind, B=B, lens=lens, lo=lo, hi=hi, lens_seed=rng.randrange(1, 1 << 20))
        if kind == "extend":
            c["new_hi"] = _log(rng, 1, 4096)
            c["new_lo"] = rng.choice([c["new_hi"], 0, 1])
            c["bucket"] = rng.choice([1, 256, 4096])
            if B * (hi + c["new_hi"]) <= 1 << 21:
                return c
            continue
        if kind == "release":
            c["drop"] = rng.choice([1.0, rng.uniform(0.005, 0.9)])
            if B * hi <= 1 << 20:
                return c
            continue
        c["Hq"], c["Hkv"] = rng.choice(_HEADS)
        c["lse"] = rng.random() < 0.4
        if kind == "prompt":
            c["fused"] = rng.random() < 0.4
            if B * hi * hi * c["Hq"] <= 32768 * 32768 * 32 // 2 and B * hi <= 1 << 18:
                return c
        else:
            c["new_hi"] = rng.randint(1, 64)
            c["new_lo"] = rng.choice([c["new_hi"], 1, 0])
            if B * hi * c["Hkv"] <= 32 * 16384 * 8 and B * hi * c["Hq"] * c["new_hi"] <= 1 << 30:
                return c


def _lens(how, lo, hi, B, rng):
    """int64 [B], both bounds inclusive."""
    if how == "uniform":
        return rng.integers(lo, hi, size=B, endpoint=True)
    if how == "spread":      # evenly over the logarithm, both ends among them
        return np.rint(np.exp(np.linspace(math.log(lo), math.log(hi), B))).astype(np.int64)
    if how == "lognormal":   # around a third of the way to the longest
        x = np.exp(rng.normal(math.log(max(lo, 0.37 * hi)), 0.5, size=B))
        return np.clip(np.rint(x), lo, hi).astype(np.int64)
    # bimodal: half up to 4 lo, half from hi / 4
    a = rng.integers(lo, max(lo, min(4 * lo, hi)), size=B // 2, endpoint=True)
    b = rng.integers(max(lo, hi // 4), hi, size=B - B // 2, endpoint=True)
    x = np.concatenate([a, b])
    rng.shuffle(x)
    return x


def lengths(case):
    """Lengths of the requests and, where a case has them, their new tokens."""
    rng = np.random.default_rng(case["lens_seed"])
    lens = _lens(case["lens"], case["lo"], case["hi"], case["B"], rng)
    if "new_hi" not in case:
        return lens, None
    new = _lens("uniform", case["new_lo"], case["new_hi"], case["B"], rng)
    new[0] = case["new_hi"]
    return lens, new


def _kept(case, lens):
    """Lengths after a release."""
    rng = np.random.default_rng(case["lens_seed"] + 1)
    if case["drop"] == 1.0:
        return np.zeros_like(lens)
    return lens - np.minimum(lens, rng.integers(0, 2 * case["drop"] * lens, endpoint=True).astype(np.int64))


# --- inputs -------------------------------------------------------------------

def _offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def _tree(rng, n):
    """Masks of a tree of n drafted tokens, uint64 [n]: each node sees itself and
    its ancestors; a node's parent is one of the few before it, or the context."""
    m = np.zeros(n, dtype=np.uint64)
    for i in range(n):
        p = int(rng.integers(max(0, i - 8), i + 1)) - 1
        m[i] = (m[p] if p >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(i))
    return m


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed * 1000003 + 31)
    host = np.random.default_rng(seed * 7919 + 5)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float16)

    def ints(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)

    kind, B = case["kind"], case["B"]
    lens, new = lengths(case)
    s = {"case": dict(case), "host_lens": lens.tolist(), "lens": ints(lens)}
    if kind == "prompt":
        Hq, Hkv, T = case["Hq"], case["Hkv"], int(lens.sum())
        shift = normal(1, Hkv, D) * 0.5
        if case.get("fused"):       # q, k and v rows of a token side by side
            x = normal(T, Hq + 2 * Hkv, D)
            s["q"], s["k"], s["v"] = x.split([Hq, Hkv, Hkv], dim=1)
            s["k"] += shift
        else:
            s["q"], s["k"], s["v"] = normal(T, Hq, D), normal(T, Hkv, D) + shift, normal(T, Hkv, D)
        s["offsets"] = ints(_offsets(lens))
        return s
    end = lens + new if kind == "extend" else lens
    nblk = -(-lens // BS)
    used, most = int(nblk.sum()), int((-(-end // BS)).sum())
    pool = most + most // 8 + 1       # an engine's pool is never quite full
    width = int((-(-end // BS)).max())
    n = torch.from_numpy(nblk).to(dev)
    ids = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    table[torch.arange(width, device=dev)[None, :] < n[:, None]] = ids[:used]
    s["table"] = table
    if kind in ("extend", "release"):
        s["free0"] = torch.full((pool,), -1, dtype=torch.int32, device=dev)
        s["free0"][:pool - used] = ids[used:]
        s["state0"] = torch.tensor([pool - used, 0], dtype=torch.int32, device=dev)
        s["free"], s["state"] = s["free0"].clone(), s["state0"].clone()
        if kind == "extend":
            s["new"] = ints(new)
            bucket = case.get("bucket", 1)
            s["T"] = max(1, -(-int(new.sum()) // bucket)) * bucket
        else:
            s["table0"] = table.clone()
            s["keep"] = ints(_kept(case, lens))
        return s
    Hq, Hkv, T = case["Hq"], case["Hkv"], int(new.sum())
    s["host_new"] = new.tolist()
    shift = normal(1, Hkv, 1, D) * 0.5
    s["k_cache"], s["v_cache"] = normal(pool, Hkv, BS, D), normal(pool, Hkv, BS, D)
    s["k_cache"] += shift
    s["q"], s["k"], s["v"] = normal(T, Hq, D), normal(T, Hkv, D) + shift[:, :, 0], normal(T, Hkv, D)
    s["offsets"] = ints(_offsets(new))
    mask = np.concatenate([_tree(host, int(m)) for m in new] + [np.zeros(0, np.uint64)])
    s["mask"] = torch.from_numpy(mask.view(np.int64)).to(dev)
    return s


# --- one pass -----------------------------------------------------------------

def _softmax_rows(score, v):
    """Weighted rows and log-sum-exp of scores [..., m, n] (-inf: masked) and rows
    [..., n, D], in 32 bits; a row with no score gives zeros and -inf."""
    m = score.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(score - m)
    total = p.sum(-1, keepdim=True)
    out = torch.where(total > 0, (p @ v) / total, torch.zeros((), device=p.device))
    return out, (m + torch.log(total)).squeeze(-1)


def _plain_attention(s):
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    G = Hq // Hkv
    T, dev = s["q"].shape[0], s["q"].device
    out = torch.empty((T, Hq, D), dtype=torch.float16, device=dev)
    lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    at = 0
    for b, L in enumerate(s["host_lens"]):
        n = L if c["kind"] == "prompt" else s["host_new"][b]
        if n == 0:
            continue
        k, v = (x[at:at + n].float().transpose(0, 1) for x in (s["k"], s["v"]))       # [Hkv][n][D]
        if c["kind"] == "tree":
            seen = ((s["mask"][at:at + n, None] >> torch.arange(n, device=dev)) & 1).bool()
            ids = s["table"][b, :-(-L // BS)].long()
            ck, cv = (x[ids].float().transpose(0, 1).flatten(1, 2)[:, :L] for x in (s["k_cache"], s["v_cache"]))
            k, v = torch.cat([ck, k], 1), torch.cat([cv, v], 1)
        q = s["q"][at:at + n].float().view(n, Hkv, G, D).permute(1, 2, 0, 3)           # [Hkv][G][n][D]
        # so many rows at once that the scores stay below 2^28 numbers
        step = n if c["kind"] == "tree" else max(1, min(n, (1 << 28) // (Hq * L)))
        for i in range(0, n, step):
            j = min(n, i + step)
            # a chunk of a prompt sees nothing behind its last row
            kk, vv = (k[:, :j], v[:, :j]) if c["kind"] == "prompt" else (k, v)
            score = (q[:, :, i:j].reshape(Hkv, -1, D) @ kk.transpose(1, 2)).view(Hkv, G, j - i, -1) * SCALE
            if c["kind"] == "prompt":
                r = torch.arange(i, j, device=dev)
                score.masked_fill_(torch.arange(j, device=dev)[None, :] > r[:, None], -math.inf)
            else:
                score[..., L:].masked_fill_(~seen[i:j], -math.inf)
            o, e = _softmax_rows(score.view(Hkv, G * (j - i), -1), vv)
            out[at + i:at + j] = o.view(Hkv, G, j - i, D).permute(2, 0, 1, 3).reshape(j - i, Hq, D)
            lse[at + i:at + j] = e.view(Hkv, G, j - i).permute(2, 0, 1).reshape(j - i, Hq)
        at += n
    return [out, lse] if c.get("lse") else out


def _restore(s):
    """Every pass starts from the same free blocks (and, where blocks are given
    back, the same table)."""
    s["state"].copy_(s["state0"])
    if "table0" in s:
        s["table"].copy_(s["table0"])


def _run_plain(s):
    c = s["case"]
    if c["kind"] in ("prompt", "tree"):
        return _plain_attention(s)
    _restore(s)
    table, free, state, L = s["table"], s["free"], s["state"], s["lens"].long()
    dev, B, width = table.device, c["B"], table.shape[1]
    col = torch.arange(width, device=dev)[None, :]
    have = (L + BS - 1) // BS
    if c["kind"] == "release":
        first = ((s["keep"].long() + BS - 1) // BS)[:, None]
        gone = (col >= first) & (col < have[:, None])
        ids = table[gone]
        free[state[0] + torch.arange(ids.numel(), device=dev)] = ids
        table.masked_fill_(gone, -1)
        state[0] += ids.numel()
        return [table, free, state]
    n, T = s["new"].long(), s["T"]
    need = (L + n + BS - 1) // BS - have
    taken = torch.cumsum(need, 0)
    first = (state[0] - 1 - (taken - need))[:, None]
    fresh = (col >= have[:, None]) & (col < (have + need)[:, None])
    table.copy_(torch.where(fresh, free[(first - (col - have[:, None])).clamp(min=0)], table))
    state[0] -= taken[-1].int()
    offsets = torch.zeros(B + 1, dtype=torch.int32, device=dev)
    offsets[1:] = torch.cumsum(n, 0)
    t = torch.arange(T, device=dev)
    b = torch.searchsorted(offsets[1:].long(), t, right=True)
    live = b < B
    b = b.clamp(max=B - 1)
    pos = L[b] + t - offsets[b]
    slot = table[b, (pos // BS).clamp(max=width - 1)].long() * BS + pos % BS
    slots = torch.where(live, slot, torch.full_like(slot, -1))
    positions = torch.where(live, pos, torch.zeros_like(pos)).int()
    return [table, state, offsets, (L + n).int(), slots, positions]


def run(s):
    if not own:
        return _run_plain(s)
    from paper_2506_03296_amd import steps
    c = s["case"]
    kind = c["kind"]
    if kind == "extend":
        _restore(s)
        plan = steps.extend(s["lens"], s["new"], s["table"], s["free"], s["state"], s["T"])
        return [s["table"], s["state"], plan.token_offsets, plan.total_lens, plan.slot_mapping, plan.token_positions]
    if kind == "release":
        _restore(s)
        steps.release(s["lens"], s["keep"], s["table"], s["free"], s["state"])
        return [s["table"], s["free"], s["state"]]
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=s["q"].device) if c.get("lse") else None
    if kind == "prompt":
        out = steps.prompt_attention(s["q"], s["k"], s["v"], s["offsets"], SCALE, lse_out=lse)
    else:
        out = steps.tree_attention(s["q"], s["k"], s["v"], s["offsets"], s["mask"], s["k_cache"], s["v_cache"],
                                   s["table"], s["lens"], c["new_hi"], SCALE, lse_out=lse)
    return [out, lse] if c.get("lse") else out


def work(case):
    """Every input read once and every result written once; the products of the
    scores and of the weights with V that the masks leave (a tree: all of its
    nodes with each other)."""
    lens, new = lengths(case)
    B, kind = case["B"], case["kind"]
    if kind == "extend":
        blocks = int((-(-(lens + new) // BS) - -(-lens // BS)).sum())
        return {"bytes": B * 16 + 8 + blocks * 8 + 12 * int(new.sum()), "flops": 0}
    if kind == "release":
        blocks = int((-(-lens // BS) - -(-_kept(case, lens) // BS)).sum())
        return {"bytes": B * 8 + 8 + blocks * 12, "flops": 0}
    Hq, Hkv = case["Hq"], case["Hkv"]
    lse = 4 * Hq if case.get("lse") else 0
    if kind == "prompt":
        T = int(lens.sum())
        return {"bytes": T * (4 * D * (Hq + Hkv) + lse) + 4 * (B + 1), "flops": 2 * D * Hq * int((lens * (lens + 1)).sum())}
    T = int(new.sum())
    tokens = int(lens[new > 0].sum())
    table = 4 * int((-(-lens // BS)).sum())
    return {"bytes": (tokens + T) * 4 * D * Hkv + T * (4 * D * Hq + 8 + lse) + table + 8 * B,
            "flops": 4 * D * Hq * int((new * (lens + new)).sum())}


# --- the same in 64 bits --------------------------------------------------------

def exact(case, seed):
    kind = case["kind"]
    if kind in ("extend", "release"):
        return None
    lens, new = lengths(case)
    if work(case)["flops"] > 1e13:
        return None
    s = prepare(case, seed)
    Hq, Hkv, dev = case["Hq"], case["Hkv"], s["q"].device
    G, T = Hq // Hkv, s["q"].shape[0]
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=dev)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=dev)
    first = s["offsets"].tolist()
    for b in range(case["B"]):
        lo, hi, L = first[b], first[b + 1], int(lens[b])
        n = hi - lo
        if n == 0:
            continue
        if kind == "tree":
            bits = s["mask"][lo:hi].cpu().numpy().view(np.uint64)
            see = torch.tensor([[True] * L + [bool((int(w) >> j) & 1) for j in range(n)] for w in bits], device=dev)
            slot = torch.arange(L, device=dev)
            slot = s["table"][b].long()[slot // BS], slot % BS
        for h in range(Hkv):
            k, v = s["k"][lo:hi, h].double(), s["v"][lo:hi, h].double()
            if kind == "tree":
                k = torch.cat([s["k_cache"][slot[0], h, slot[1]].double(), k])
                v = torch.cat([s["v_cache"][slot[0], h, slot[1]].double(), v])
            kt = k.t().contiguous()
            for j in range(h * G, h * G + G):
                for i in range(0, n, 4096):
                    e = min(n, i + 4096)
                    x = torch.mm(s["q"][lo + i:lo + e, j].double(), kt) * SCALE
                    if kind == "tree":
                        x = x.masked_fill(~see[i:e], -math.inf)
                    else:
                        x = x.masked_fill(torch.ones(e - i, n, dtype=torch.bool, device=dev).triu(i + 1), -math.inf)
                    lse[lo + i:lo + e, j] = torch.logsumexp(x, -1)
                    out[lo + i:lo + e, j] = torch.mm(torch.softmax(x, -1), v)
    return [out, lse] if case.get("lse") else out
