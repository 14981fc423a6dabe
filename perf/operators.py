"""Sampled decoding of several continuations of one prompt: the operators such a program calls beside the steps.

Kinds of cases:

* ``sample``  tokens drawn from logits with temperature, top-k, top-p and min-p, and their probabilities
  (``Engine.sf_op_sample``);
* ``accept``  lossless acceptance of a drafted block at temperature > 0 and its commit (``Engine.sf_op_accept_sampled``);
* ``prefix``  attention of a batch whose sequences continue one shared prompt (``Engine.sf_op_prefix_attention``).

A row's distribution.  Tokens are ranked by falling logit, equal ones by index; the weight of a token is
exp((logit - largest) / temperature).  Kept are the top_k first of the ranking (0: all), of those the ones whose better
ranked tokens weigh less than top_p of them together, of those the ones of at least min_p; the first always.
Temperature 0 keeps the first alone.  A token is drawn as the first, in the order of the vocabulary, whose running kept
weight exceeds u times the kept weight.  Acceptance: slot i's token d stays while u_i * q_i(d) < p_i(d); behind the last
accepted one a token is drawn from max(p - q, 0), or from p behind a block that stays whole.  Weights and their sums are
kept in 64 bits: a token next to a border must not depend on the order of a sum.
"""
import math
import random

import torch

own = False

# query heads, kv heads, head dim, type, vocabulary of the repository's model shapes
MODELS = {"tiny": (4, 4, 64, "f32", 1024), "1b": (32, 8, 64, "bf16", 32000), "8b": (32, 8, 128, "bf16", 128256),
          "14b": (40, 8, 128, "bf16", 152064)}


def listed():
    return [
        # one user at a terminal: one row, latency counts
        {"name": "sample_1b_one", "kind": "sample", "rows": 1, "group": 1, "vocab": 32000, "filters": "common"},
        # a ragged handful of requests, each with settings of its own, over a vocabulary of odd size with masked tokens
        {"name": "sample_odd_vocab", "kind": "sample", "rows": 19, "group": 1, "vocab": 50257, "filters": "mixed"},
        # the draft's slots of a batch: 64 sequences of 4 slots that share their sequence's settings
        {"name": "sample_8b_slots", "kind": "sample", "rows": 256, "group": 4, "vocab": 128256, "filters": "mixed"},
        # the largest: every row of a verified block of 128 sequences, nucleus sampling
        {"name": "sample_14b_rows", "kind": "sample", "rows": 640, "group": 5, "vocab": 152064, "filters": "nucleus"},
        # one user, sampled drafts
        {"name": "accept_1b_one", "kind": "accept", "batch": 1, "k": 4, "vocab": 32000, "draft": "sampled", "filters": "common"},
        # a batch with settings of its own per sequence, sampled drafts
        {"name": "accept_8b_sampled", "kind": "accept", "batch": 64, "k": 4, "vocab": 128256, "draft": "sampled", "filters": "mixed"},
        # the draft step's own greedy tokens, accepted at temperature 1 without filters
        {"name": "accept_14b_greedy", "kind": "accept", "batch": 128, "k": 4, "vocab": 152064, "draft": "greedy", "filters": "plain"},
        # the fp32 mode of small models
        {"name": "prefix_tiny_f32", "kind": "prefix", "model": "tiny", "batch": 4, "rows": 5, "prefix": 64, "lo": 0, "hi": 64, "mask": "causal"},
        # eight continuations of a short prompt, plain decoding: latency counts
        {"name": "prefix_1b_plain", "kind": "prefix", "model": "1b", "batch": 8, "rows": 1, "prefix": 701, "lo": 0, "hi": 60, "mask": "causal"},
        # the small model's batch, verified blocks of five
        {"name": "prefix_1b_b32", "kind": "prefix", "model": "1b", "batch": 32, "rows": 5, "prefix": 2048, "lo": 1, "hi": 300, "mask": "causal"},
        # draft slots that see each other, odd batch, a prompt that ends inside a tile
        {"name": "prefix_8b_slots", "kind": "prefix", "model": "8b", "batch": 37, "rows": 4, "prefix": 1500, "lo": 16, "hi": 512, "mask": "bidir"},
        # the largest: 128 continuations of a long document, verified blocks of five
        {"name": "prefix_14b_b128", "kind": "prefix", "model": "14b", "batch": 128, "rows": 5, "prefix": 8192, "lo": 32, "hi": 512, "mask": "causal"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges; its work stays below that of the kind's largest listed one."""
    kind = rng.choice(["sample", "accept", "prefix"])
    if kind == "prefix":
        model = rng.choice(["tiny", "1b", "8b", "14b"])
        hq, hkv, hd, dtype, _ = MODELS[model]
        batch = _log_int(rng, 1, 16 if dtype == "f32" else 128)
        rows = rng.randint(1, 9)
        room = 640 * 40 * 128 * 8192 // (batch * rows * hq * hd)
        hi = _log_int(rng, 1, 600)
        return {"kind": kind, "model": model, "batch": batch, "rows": rows, "lo": rng.randint(0, hi), "hi": hi,
                "prefix": min(_log_int(rng, 16, 600 if dtype == "f32" else 8192), max(16, room - hi - rows)),
                "mask": rng.choice(["causal", "bidir"])}
    vocab = rng.choice([1024, 32000, 128256, 152064, _log_int(rng, 1000, 152064), _log_int(rng, 1000, 152064)])
    filters = rng.choice(["common", "mixed", "mixed", "nucleus", "plain"])
    room = 640 * 152064 // vocab
    if kind == "sample":
        group = rng.choice([1, 1, 2, 4, 5])
        return {"kind": kind, "rows": min(_log_int(rng, 1, 640), room), "group": group, "vocab": vocab, "filters": filters}
    k = rng.randint(1, 8)
    return {"kind": kind, "batch": max(1, min(_log_int(rng, 1, 128), room // (k + 2))), "k": k, "vocab": vocab,
            "draft": rng.choice(["sampled", "sampled", "greedy"]), "filters": filters}


def _settings(filters, n, g):
    """Per-request temperature, top_k, top_p, min_p as tensors [n], of what requests commonly ask for."""
    def pick(values, dtype):
        at = torch.randint(0, len(values), (n,), generator=g, device="cuda")
        return torch.tensor(values, dtype=dtype, device="cuda")[at]
    f, i = torch.float32, torch.int32
    if filters == "plain":
        return pick([1.0], f), pick([0], i), pick([1.0], f), pick([0.0], f)
    if filters == "nucleus":
        return pick([0.7, 1.0], f), pick([0], i), pick([0.9, 0.95], f), pick([0.0], f)
    if filters == "common":
        return pick([0.6, 0.8], f), pick([20, 50], i), pick([0.9, 0.95], f), pick([0.0, 0.05], f)
    return (pick([0.0, 0.6, 0.8, 1.0, 1.3], f), pick([0, 0, 1, 20, 50, 200, 1000], i), pick([1.0, 0.98, 0.95, 0.9, 0.5], f),
            pick([0.0, 0.0, 0.02, 0.1], f))


def _logits(rows, vocab, g, masked):
    """Rows as a language model's head gives them: a broad bulk and some forty tokens that fit, by a lead that goes from
    none to speak of (an open choice of thousands of tokens) to certainty.  Every fifth row sits on the grid of bf16, as a
    head of that type leaves it; where masked, every seventh has nine tenths forbidden."""
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 1.8
    lead = 8.0 + 10.0 * torch.rand(rows, 1, generator=g, device="cuda")
    x += lead * (torch.rand(rows, vocab, generator=g, device="cuda") < 40.0 / vocab)
    row = torch.arange(rows, device="cuda")
    x = torch.where((row % 5 == 1)[:, None], x.to(torch.bfloat16).float(), x)
    if masked:
        x.masked_fill_((row % 7 == 3)[:, None] & (torch.rand(rows, vocab, generator=g, device="cuda") < 0.9), -math.inf)
    return x


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 6007 + 11)
    uniform = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    if case["kind"] == "prefix":
        return _prepare_prefix(s, case, seed, g)
    V, masked = case["vocab"], case["filters"] == "mixed"
    if case["kind"] == "sample":
        n = -(-case["rows"] // case["group"])
        s.settings = _settings(case["filters"], n, g)
        s.logits = _logits(case["rows"], V, g, masked)
        s.u = uniform(case["rows"])
        if own:
            s.eng = _small_engine(V, 1, 1)
        return s
    B, k = case["batch"], case["k"]
    s.settings = _settings(case["filters"], B, g)
    s.target = _logits(B * (k + 1), V, g, masked).view(B, k + 1, V)
    # the draft's logits are the target's with an error of its own
    draft = s.target[:, :k] + torch.randn(B, k, V, generator=g, device="cuda")
    s.u_accept, s.u_sample, u_draft = uniform(B, k), uniform(B), uniform(B, k)
    s.kv_len = torch.randint(0, 1000, (B,), generator=g, device="cuda", dtype=torch.int32)
    s.draft_logits = s.draft_dist = None
    if case["draft"] == "sampled":
        s.draft_logits = draft.contiguous()
        s.draft = _pick(_weights(s.draft_logits, *(t[:, None] for t in s.settings)), u_draft).to(torch.int32)
    else:
        s.draft = draft.argmax(-1).to(torch.int32)
    if own:
        s.eng = _small_engine(V, B, k)
        if s.draft_logits is not None:
            # what the draft's own sampling left behind for the acceptance
            _, s.draft_dist = s.eng.sf_op_sample(s.draft_logits.view(B * k, V), u_draft.view(-1), *s.settings, group=k, want_dist=True)
    return s


def _small_engine(vocab, batch, k):
    from paper_2511_20340_amd.engine import Engine
    return Engine({"n_layers": 1, "d_model": 64, "n_q_heads": 1, "n_kv_heads": 1, "head_dim": 64, "d_ffn": 64, "vocab": vocab, "dtype": "bf16"}, batch, 32, k)


def _up32(n):
    return -(-n // 32) * 32


def _prepare_prefix(s, case, seed, g):
    hq, hkv, hd, dtype, vocab = MODELS[case["model"]]
    B, n, P = case["batch"], case["rows"], case["prefix"]
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    cap = _up32(case["hi"] + n)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(t)  # noqa: E731
    r = random.Random(seed * 7919 + 17)
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(B)]
    s.upper = max(lens)
    s.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # rows of order one, as the models' own projections give; some prompt positions draw most of the attention
    s.q = normal(B, n, hq, hd)
    s.pk, s.pv = normal(1, hkv, P, hd), normal(1, hkv, P, hd)
    s.pk[:, :, ::97] *= 2
    s.k, s.v = normal(B, hkv, cap, hd), normal(B, hkv, cap, hd)
    if own:
        from paper_2511_20340_amd import binding
        from paper_2511_20340_amd.engine import Engine
        cfg = {"n_layers": 1, "d_model": 64, "n_q_heads": hq, "n_kv_heads": hkv, "head_dim": hd, "d_ffn": 64, "vocab": vocab, "dtype": dtype}
        s.eng, s.shared = Engine(cfg, B, cap, n - 1), Engine(cfg, 1, _up32(P), 0)
        pad = torch.zeros(1, hkv, _up32(P) - P, hd, dtype=t, device="cuda")
        s.shared.sf_kv_import(torch.cat([s.pk, pad], 2), "tk")
        s.shared.sf_kv_import(torch.cat([s.pv, pad], 2), "tv")
        s.eng.sf_kv_import(s.k, "tk")
        s.eng.sf_kv_import(s.v, "tv")
        s.mask = binding.SF_MASK_BIDIR if case["mask"] == "bidir" else binding.SF_MASK_CAUSAL
    return s


def run(state):
    s, kind = state, state.case["kind"]
    if own:
        if kind == "sample":
            return s.eng.sf_op_sample(s.logits, s.u, *s.settings, group=s.case["group"], want_prob=True)
        if kind == "prefix":
            return s.eng.sf_op_prefix_attention(s.q, s.shared.layer_cache("tk"), s.shared.layer_cache("tv"), s.case["prefix"],
                                                s.eng.layer_cache("tk"), s.eng.layer_cache("tv"), s.kv_len, s.case["rows"], s.mask, len_upper=s.upper)
        s.eng.kv_len.copy_(s.kv_len)
        accept_len, tokens = s.eng.sf_op_accept_sampled(s.case["k"], s.draft, s.target, s.u_accept, s.u_sample, *s.settings,
                                                        draft_logits=s.draft_logits, draft_dist=s.draft_dist)
        return accept_len, tokens, s.eng.kv_len, s.eng.pending, s.eng.n_new, s.eng.cu_new
    if kind == "sample":
        settings = [t.repeat_interleave(s.case["group"])[:s.case["rows"]] for t in s.settings]
        w = _weights(s.logits, *settings)
        ids = _pick(w, s.u)
        return ids.to(torch.int32), (w.gather(-1, ids[:, None])[:, 0] / w.sum(-1)).float()
    if kind == "prefix":
        return _prefix_attention(s)
    return _accept(s)


def _weights(logits, temperature, top_k, top_p, min_p):
    """The kept weights of every row, in the order of the vocabulary, in 64 bits; settings have the shape of the rows."""
    V = logits.shape[-1]
    ranked, index = torch.sort(logits, dim=-1, descending=True, stable=True)
    greedy = temperature <= 0
    t = torch.where(greedy, 1.0, temperature).double()[..., None]
    count = torch.where(greedy, 1, torch.where(top_k > 0, top_k, V))[..., None]
    p, m = top_p.double()[..., None], min_p.double()[..., None]
    w = torch.exp((ranked.double() - ranked[..., :1].double()) / t)
    rank = torch.arange(V, device=logits.device)
    w = w * (rank < count)
    total = torch.cumsum(w, -1)
    better = torch.cat([torch.zeros_like(total[..., :1]), total[..., :-1]], -1)
    keep = (rank < count) & ((better < p * total[..., -1:]) | (p >= 1)) & (w >= m) | (rank == 0)
    return torch.zeros_like(w).scatter_(-1, index, w * keep)


def _pick(w, u):
    """The first index whose running weight exceeds u times the whole."""
    c = torch.cumsum(w, -1)
    return (c <= u.double()[..., None] * c[..., -1:]).sum(-1)


def _accept(s):
    B, k, V = s.case["batch"], s.case["k"], s.case["vocab"]
    settings = [t[:, None] for t in s.settings]
    p = _weights(s.target, *(t.expand(B, k + 1) for t in settings))
    p = p / p.sum(-1, keepdim=True)
    d = s.draft.long()[..., None]
    if s.draft_logits is None:
        q = torch.zeros(B, k + 1, V, dtype=torch.float64, device="cuda")
        q[:, :k].scatter_(-1, d, 1.0)
    else:
        q = _weights(s.draft_logits, *(t.expand(B, k) for t in settings))
        q = torch.cat([q / q.sum(-1, keepdim=True), torch.zeros(B, 1, V, dtype=torch.float64, device="cuda")], 1)
    stays = s.u_accept.double() * q[:, :k].gather(-1, d)[..., 0] < p[:, :k].gather(-1, d)[..., 0]
    n = torch.cumprod(stays.int(), 1).sum(1)
    at = n[:, None, None].expand(B, 1, V)
    rest = (p.gather(1, at) - q.gather(1, at)).clamp(min=0)[:, 0]
    last = _pick(rest, s.u_sample)
    slot = torch.arange(k + 1, device="cuda")
    tokens = torch.cat([s.draft.long(), torch.zeros(B, 1, dtype=torch.int64, device="cuda")], 1)
    tokens = torch.where(slot < n[:, None], tokens, torch.where(slot == n[:, None], last[:, None], -1))
    a = (n + 1).to(torch.int32)
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cumsum(a, 0).to(torch.int32)])
    return a, tokens.to(torch.int32), s.kv_len + a, last.to(torch.int32), a, cu


def _prefix_attention(s):
    hq, hkv, hd, _, _ = MODELS[s.case["model"]]
    B, n, P, cap = s.case["batch"], s.case["rows"], s.case["prefix"], s.k.shape[2]
    G = hq // hkv
    q = s.q.float().view(B, n, hkv, G, hd).permute(2, 0, 1, 3, 4).contiguous()              # [hkv, B, n, G, hd]
    shared = torch.bmm(q.view(hkv, B * n * G, hd), s.pk[0].float().transpose(1, 2).contiguous()).view(hkv, B, n, G, P)
    mine = torch.bmm(q.view(hkv * B, n * G, hd), s.k.float().permute(1, 0, 3, 2).reshape(hkv * B, hd, cap)).view(hkv, B, n, G, cap)
    key = torch.arange(cap, device="cuda") - s.kv_len[:, None, None]                         # [B, 1, cap]: place in the block
    row = torch.arange(n, device="cuda")[None, :, None]
    seen = (key <= row) if s.case["mask"] == "causal" else (key < n).expand(B, n, cap)
    mine = torch.where(seen[None, :, :, None], mine, -math.inf)
    score = torch.cat([shared, mine], -1) / math.sqrt(hd)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    out = torch.bmm(w[..., :P].reshape(hkv, B * n * G, P), s.pv[0].float()).view(hkv, B, n, G, hd)
    out = out + torch.bmm(w[..., P:].reshape(hkv * B, n * G, cap), s.v.float().transpose(0, 1).reshape(hkv * B, cap, hd)).view(hkv, B, n, G, hd)
    return out.permute(1, 2, 0, 3, 4).reshape(B, n, hq, hd).to(s.q.dtype)


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": 4 * (n + 3 * case["rows"]), "flops": 3 * n}
    if case["kind"] == "accept":
        # every row of the block, and one draft row per sequence for what is left of it
        rows = case["batch"] * (case["k"] + 1 + (case["draft"] == "sampled"))
        return {"bytes": 4 * rows * case["vocab"], "flops": 3 * rows * case["vocab"]}
    hq, hkv, hd, dtype, _ = MODELS[case["model"]]
    es = 4 if dtype == "f32" else 2
    B, n, P = case["batch"], case["rows"], case["prefix"]
    mine = B * ((case["lo"] + case["hi"]) / 2 + n)
    return {"bytes": int(es * (2 * hkv * hd * (P + mine) + 2 * B * n * hq * hd)),
            "flops": int(4 * n * hq * hd * (B * P + mine))}


def exact(case, seed):
    """Row by row from the definition, in 64 bits."""
    s = prepare(case, seed)
    if case["kind"] == "prefix":
        return _exact_attention(s)
    B, k, V = case.get("batch", 0), case.get("k", 0), case["vocab"]
    if (case["rows"] if case["kind"] == "sample" else B * (2 * k + 1)) * V > 60e6:
        return None
    import numpy as np
    T, K, P, m = (t.cpu().numpy() for t in s.settings)

    def shares(row, j):
        """Probability of every token under the settings of request j, by walking down the ranking."""
        l = row.astype(np.float64)
        order = np.lexsort((np.arange(V), -l))
        if T[j] <= 0:
            kept, w = order[:1], np.ones(1)
        else:
            kept = order[:K[j]] if K[j] > 0 else order
            w = np.exp((l[kept] - l[kept[0]]) / np.float64(T[j]))
            if P[j] < 1:
                end = max(1, int(np.searchsorted(np.concatenate([[0.0], np.cumsum(w)[:-1]]), np.float64(P[j]) * w.sum(), side="left")))
                kept, w = kept[:end], w[:end]
            end = max(1, int((w >= np.float64(m[j])).sum()))
            kept, w = kept[:end], w[:end]
        p = np.zeros(V)
        p[kept] = w / w.sum()
        return p

    def drawn(p, u):
        c = np.cumsum(p)
        return int(np.searchsorted(c, np.float64(u) * c[-1], side="right"))

    if case["kind"] == "sample":
        logits, u = s.logits.cpu().numpy(), s.u.cpu().numpy()
        found = []
        for r in range(case["rows"]):
            p = shares(logits[r], r // case["group"])
            i = drawn(p, u[r])
            found.append((i, p[i]))
        return torch.tensor([i for i, _ in found], dtype=torch.int32), torch.tensor([p for _, p in found], dtype=torch.float64)
    target, draft = s.target.cpu().numpy(), s.draft.cpu().numpy()
    u, u_last = s.u_accept.cpu().numpy().astype(np.float64), s.u_sample.cpu().numpy()
    dl = None if s.draft_logits is None else s.draft_logits.cpu().numpy()
    n_new, last, tokens = np.zeros(B, np.int32), np.zeros(B, np.int32), np.full((B, k + 1), -1, np.int32)
    for b in range(B):
        for i in range(k + 1):
            rest = shares(target[b, i], b)
            if i < k:
                q = np.eye(1, V, draft[b, i])[0] if dl is None else shares(dl[b, i], b)
                d = draft[b, i]
                if u[b, i] * q[d] < rest[d]:
                    tokens[b, i] = d
                    continue
                rest = np.maximum(rest - q, 0)
            last[b] = tokens[b, i] = drawn(rest, u_last[b])
            n_new[b] = i + 1
            break
    a = torch.from_numpy(n_new)
    cu = torch.cat([torch.zeros(1, dtype=torch.int32), torch.cumsum(a, 0).to(torch.int32)])
    return a, torch.from_numpy(tokens), s.kv_len.cpu() + a, torch.from_numpy(last), a, cu


def _exact_attention(s):
    case = s.case
    hq, hkv, hd, _, _ = MODELS[case["model"]]
    n, P = case["rows"], case["prefix"]
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(s.kv_len.tolist()):
        for h in range(hkv):
            keys = torch.cat([s.pk[0, h], s.k[b, h, :length + n]]).double()
            values = torch.cat([s.pv[0, h], s.v[b, h, :length + n]]).double()
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            for i in range(n):
                end = P + length + (i + 1 if case["mask"] == "causal" else n)
                out[b, i, heads] = torch.softmax(s.q[b, i, heads].double() @ keys[:end].t() * hd ** -0.5, -1) @ values[:end]
    return out
