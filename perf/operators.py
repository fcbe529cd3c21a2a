"""Performance cases of a 4-bit LM head, of token log-probabilities and of the distillation loss's gradient.

Every case is a dict of plain values.  `call` says which operator a pass goes through:

  head       logits of a few hidden rows through a target head of 4-bit weights with group scales
  logprobs   log-probabilities of given tokens, entropy and the most likely alternatives of rows of logits
  learn      the same log-probabilities and entropies, then their gradient with respect to the logits
  loss_grad  the hybrid distillation loss of a batch that a step has verified, then its gradient with respect to the
             drafter's logits

A pass returns float32 logits, log-probabilities and entropies; gradients come in the type of their logits.  Where `own`
is false a pass computes the same from elementary torch operations in float32.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
LAMBDA = 0.2


# ------------------------------------------------------------------------------------------------ the cases
def _head(name, M, d, V, group, scales, zeros):
    c = {"call": "head", "M": M, "d": d, "V": V, "group": group, "scales": scales, "zeros": zeros}
    return dict(c, name=name) if name else c


def _rows(name, call, M, V, dtype, n_tok, n_top, masked, temperature):
    c = {"call": call, "M": M, "V": V, "dtype": dtype, "n_tok": n_tok, "n_top": n_top, "masked": masked, "temperature": temperature}
    return dict(c, name=name) if name else c


def _loss(name, B, k_min, k_max, V_t, V_d, dtype, entries, max_len, approx_kl, greedy):
    c = {"call": "loss_grad", "B": B, "k_min": k_min, "k_max": k_max, "V_t": V_t, "V_d": V_d, "dtype": dtype, "entries": entries,
         "max_len": max_len, "approx_kl": approx_kl, "greedy": greedy}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence on a small target: latency
        _head("head_m1_v32k", 1, 1024, 32000, 128, "bf16", False),
        # one interactive sequence of five drafted tokens on a 152064-id target, zero points and float16 scales
        _head("head_m6_v152k", 6, 3584, 152064, 128, "f16", True),
        # a lightly loaded server; a vocabulary of odd size, a hidden size that ends inside a group
        _head("head_m24_v32003", 24, 2056, 32003, 64, "bf16", True),
        # 16 sequences of 8 drafted tokens on a 128256-id target: the headline batch
        _head("head_m144_v128k", 144, 4096, 128256, 128, "bf16", True),
        # one emitted token with five alternatives
        _rows("logprobs_m1_v32k", "logprobs", 1, 32000, "f32", 1, 5, 0.0, 0.7),
        # the verified rows of the headline batch, twenty alternatives each, half of the rows under a sparse token mask
        _rows("logprobs_m144_v128k", "logprobs", 144, 128256, "f32", 1, 20, 0.5, 0.7),
        # scoring of a long prompt from 16-bit logits, a vocabulary of odd size, two candidate tokens per position
        _rows("logprobs_m2000_v32003", "logprobs", 2000, 32003, "bf16", 2, 0, 0.0, 1.0),
        # the drafter's own rows of the headline batch in a training step
        _rows("learn_m128_v32k", "learn", 128, 32000, "bf16", 1, 0, 0.0, 1.0),
        # a training step on 512 positions of the large vocabulary, some under a mask
        _rows("learn_m512_v128k", "learn", 512, 128256, "f32", 1, 0, 0.25, 1.0),
        # one interactive sequence, drafter and target of one vocabulary
        _loss("loss_grad_b1_v32k", 1, 5, 5, 32000, 32000, "f32", 0, 2, False, 0.0),
        # the headline batch
        _loss("loss_grad_b16_v128k", 16, 8, 8, 128256, 32000, "bf16", 50000, 5, False, 0.0),
        # a busy server's ragged windows, some sequences greedy, the n-gram terms as approximate KL
        _loss("loss_grad_b64_v152k", 64, 1, 10, 152064, 32000, "bf16", 50000, 6, True, 0.25),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    call = rng.choice(["head", "head", "logprobs", "learn", "loss_grad"])
    if call == "head":
        V = _log_int(rng, 4096, 152064)
        d = 8 * _log_int(rng, 32, 512)
        M = max(1, min(_log_int(rng, 1, 160), 144 * 4096 * 128256 // (d * V)))
        return _head(None, M, d, V, rng.choice([32, 64, 128]), rng.choice(["bf16", "f16"]), rng.random() < 0.6)
    if call == "loss_grad":
        V_t = _log_int(rng, 4096, 152064)
        V_d = min(V_t, _log_int(rng, 2000, 32000))
        k_max = rng.randint(1, 10)
        return _loss(None, _log_int(rng, 1, 64), rng.choice([k_max, rng.randint(1, k_max)]), k_max, V_t, V_d, rng.choice(["bf16", "f32"]),
                     min(_log_int(rng, 100, 50000), V_t // 8), rng.randint(2, 6), rng.random() < 0.4, rng.choice([0.0, 0.0, 0.25]))
    V = _log_int(rng, 1000, 152064)
    M = max(1, min(_log_int(rng, 1, 2000), 512 * 128256 // V // (1 if call == "learn" else 2)))
    return _rows(None, call, M, V, rng.choice(["bf16", "f32"]), rng.randint(1, 3), rng.choice([0, 1, 5, 20, 50]) if call == "logprobs" else 0,
                 rng.choice([0.0, 0.0, 0.5]), rng.choice([1.0, 1.0, 0.7, 0.3]))


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _head_inputs(case, seed):
    """Hidden rows N(0, 1), codes around their zero point as rounding of normal weights leaves them, scales that vary by group."""
    gen, d, V, G = _generator(seed), case["d"], case["V"], -(-case["d"] // case["group"])
    zeros = torch.randint(4, 12, (G, V), generator=gen, device=DEVICE, dtype=torch.uint8) if case["zeros"] else None
    codes = torch.empty(d // 2, V, dtype=torch.uint8, device=DEVICE)
    for r in range(0, d // 2, 256):
        n = min(256, d // 2 - r)
        two = (8.0 + 2.6 * torch.randn(2, n, V, generator=gen, device=DEVICE)).round_().clamp_(0, 15).to(torch.uint8)
        codes[r:r + n] = two[0] | (two[1] << 4)
    scales = (0.02 / 2.6) * (0.5 + torch.rand(G, V, generator=gen, device=DEVICE))
    hidden = torch.randn(case["M"], d, generator=gen, device=DEVICE).bfloat16()
    return {"hidden": hidden, "codes": codes, "scales": scales.to(torch.bfloat16 if case["scales"] == "bf16" else torch.float16), "zeros": zeros}


def _row_inputs(case, seed):
    """Rows of logits N(0, 2^2) with one token in front; `masked`: the share of rows whose mask leaves a tenth of the ids."""
    gen, M, V = _generator(seed), case["M"], case["V"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    z = 2.0 * torch.randn(M, V, generator=gen, device=DEVICE)
    tokens = torch.randint(0, V, (M, case["n_tok"]), generator=gen, device=DEVICE, dtype=torch.int32)
    z.scatter_(1, tokens[:, :1].long(), 8.0)
    n = int(round(case["masked"] * M))
    if n:
        out = torch.rand(n, V, generator=gen, device=DEVICE) >= 0.1
        out.scatter_(1, tokens[:n].long(), False)
        z[:n].masked_fill_(out, -math.inf)
    x = {"logits": z.to(dtype), "tokens": tokens, "temperature": torch.full((M,), case["temperature"], device=DEVICE)}
    if case["call"] == "learn":
        x["grad_logprob"] = torch.randn(M, case["n_tok"], generator=gen, device=DEVICE) / M
        x["grad_entropy"] = torch.full((M,), -0.01 / M, device=DEVICE)
    return x


def _translate(ids, dmap, table, max_len):
    """The window's target tokens, left to right, longest n-gram first: (target id, first draft position, draft tokens covered)."""
    got, s = [], 0
    while s < len(ids):
        L = next((n for n in range(min(max_len, len(ids) - s), 1, -1) if ids[s:s + n] in table), 1)
        t = table[ids[s:s + L]] if L > 1 else int(dmap[ids[s]])
        if t < 0:
            break
        got.append((t, s, L))
        s += L
    return got


def _loss_inputs(case, seed):
    """A verified batch: drafter's logits N(0, 2^2) and ids drawn from them, n-gram keys planted over a third of the windows, target
    logits N(0, 1.3^2) that favour the proposed tokens, and the translation of every window."""
    rng, gen = np.random.default_rng([seed, 5]), _generator(seed)
    B, V_t, V_d = case["B"], case["V_t"], case["V_d"]
    k = np.random.default_rng([B, case["k_min"], case["k_max"]]).integers(case["k_min"], case["k_max"] + 1, size=B)
    row_off = np.zeros(B + 1, np.int32)
    row_off[1:] = np.cumsum(k + 1)
    M, K = int(row_off[-1]), int(k.sum())
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    T = rng.choice(np.array([1.0, 0.7], np.float32), size=B)
    T[rng.permutation(B)[:int(round(case["greedy"] * B))]] = 0.0
    if V_d == V_t:
        dmap = np.arange(V_d, dtype=np.int32)
    else:
        dmap = np.full(V_d, -1, np.int32)
        n = min(int(0.93 * V_d), int(0.8 * V_t))
        dmap[rng.choice(V_d, size=n, replace=False)] = rng.choice(V_t, size=n, replace=False)
    n = case["entries"]
    key_off = np.zeros(n + 1, np.int32)
    key_off[1:] = np.cumsum(rng.integers(2, case["max_len"] + 1, size=n))
    key_ids = rng.integers(0, V_d, size=int(key_off[-1])).astype(np.int32)
    targets = rng.integers(0, V_t, size=n).astype(np.int32)
    flat = key_ids.tolist()
    keys = [tuple(flat[key_off[e]:key_off[e + 1]]) for e in range(n)]
    table = dict(zip(keys, targets.tolist()))
    zq = (2.0 * torch.randn(K, V_d, generator=gen, device=DEVICE)).to(dtype)
    z = 1.3 * torch.randn(M, V_t, generator=gen, device=DEVICE)
    ids = rng.integers(0, V_d, size=K).astype(np.int32)
    ids[:] = torch.argmax(zq.float() - torch.log(torch.empty(K, V_d, device=DEVICE).exponential_(generator=gen)), 1).cpu().numpy()
    tokens, favoured = [], []
    for b in range(B):
        q0, s = int(row_off[b]) - b, 0
        while s < k[b]:
            key = keys[rng.integers(n)] if n and rng.random() < 0.15 else ()
            if key and s + len(key) <= k[b]:
                ids[q0 + s:q0 + s + len(key)] = key
                s += len(key)
            s += 1
        got = _translate(tuple(ids[q0:q0 + k[b]].tolist()), dmap, table, case["max_len"])
        tokens.append(got)
        favoured += [(int(row_off[b]) + j, t) for j, (t, _, _) in enumerate(got)]
    if favoured:
        rows, toks = (torch.tensor(v, device=DEVICE) for v in zip(*favoured))
        z[rows, toks] += 4.0
    zq[torch.arange(K, device=DEVICE), torch.from_numpy(ids).to(DEVICE).long()] += 3.0
    return {"k": k, "row_off": row_off, "M": M, "K": K, "T": T, "dmap": dmap, "ngrams": (key_off, key_ids, targets), "logits": z,
            "draft_logits": zq, "draft_ids": ids, "tokens": tokens}


def _terms(case, x):
    """The loss's terms as index tensors: direct tokens, and n-gram tokens with their sub-tokens padded to the longest key."""
    L_max = case["max_len"]
    one, many, inverse = [], [], np.full(case["V_t"], -1, np.int32)
    mapped = np.flatnonzero(x["dmap"] >= 0)
    inverse[x["dmap"][mapped]] = mapped
    for b, got in enumerate(x["tokens"]):
        r0, q0, T = int(x["row_off"][b]), int(x["row_off"][b]) - b, float(x["T"][b])
        for j, (t, s, L) in enumerate(got if T > 0 else []):
            if L == 1:
                one.append((r0 + j, q0 + s, T))
            else:
                at = [q0 + s + min(i, L - 1) for i in range(L_max)]
                many.append((r0 + j, T, t, int(x["dmap"][x["draft_ids"][q0 + s]]), int(inverse[t]), L, at))
    put = lambda v, t=torch.int64: torch.tensor(v, dtype=t, device=DEVICE)  # noqa: E731
    terms = {"one": None, "many": None, "n": max(1, len(one) + sum(m[5] for m in many))}
    kind = np.zeros(x["M"], np.int32)
    if one:
        kind[[o[0] for o in one]] = 1
        rows, drows, T = zip(*one)
        terms["one"] = {"row": put(rows), "drow": put(drows), "T": put(T, torch.float32)[:, None]}
    if many:
        kind[[m[0] for m in many]] = 2
        rows, T, t, pre, inv, L, at = zip(*many)
        terms["many"] = {"row": put(rows), "T": put(T, torch.float32)[:, None], "t": put(t), "pre": put(pre), "inverse": put(inv), "at": put(at),
                         "has": torch.arange(L_max, device=DEVICE)[None, :] < put(L)[:, None]}
    terms["kind"] = torch.from_numpy(kind).to(DEVICE)
    return terms


def prepare(case, seed):
    put = lambda a: torch.from_numpy(a).to(DEVICE)  # noqa: E731
    call = case["call"]
    state = {"call": call, "case": case}
    if call == "head":
        state.update(_head_inputs(case, seed))
        if own:
            from paper_2507_02659_amd.runner import QuantWeights, Verifier
            w = QuantWeights(state["codes"], state["scales"], state["zeros"], case["group"])
            state["v"] = Verifier.quantized(w, V_d=1, direct_map=np.zeros(1, np.int32), max_batch=case["M"], max_k=0)
        return state
    if call != "loss_grad":
        state.update(_row_inputs(case, seed))
        if own:
            from paper_2507_02659_amd.runner import Verifier
            state["v"] = Verifier(d=8, V_t=case["V"], V_d=1, dtype="bf16", W=torch.zeros(8, case["V"], dtype=torch.bfloat16, device=DEVICE),
                                  direct_map=np.zeros(1, np.int32), max_batch=1, max_k=0)
        return state
    x = _loss_inputs(case, seed)
    state.update(x, grad_loss=torch.full((1,), 1.0, device=DEVICE), terms=_terms(case, x), dmap_dev=put(x["dmap"]).long(), ids_dev=put(x["draft_ids"]).long())
    if own:
        # the verification that comes before the loss in a program: it leaves the translation and the rows' statistics
        from paper_2507_02659_amd import binding as ot
        from paper_2507_02659_amd.runner import Verifier
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        v = Verifier(d=8, V_t=case["V_t"], V_d=case["V_d"], dtype=case["dtype"], W=torch.zeros(8, case["V_t"], dtype=dtype, device=DEVICE),
                     direct_map=x["dmap"], max_batch=case["B"], max_k=case["k_max"], max_ngram_len=case["max_len"])
        v.set_cache(*x["ngrams"])
        inp = {"B": case["B"], "M": x["M"], "K": x["K"], "step": 1, "seed": seed, "row_off_host": x["row_off"], "row_off": put(x["row_off"]),
               "hidden": None, "target_logits": x["logits"], "draft_logits": x["draft_logits"], "draft_ids": put(x["draft_ids"]),
               "temperature": put(x["T"]), "draft_temperature": None, "seq_id": torch.arange(case["B"], dtype=torch.int64, device=DEVICE)}
        inp["out"] = v.alloc_outputs(case["B"], x["M"])
        v.step(inp, from_logits=True)
        state.update(v=v, inp=inp, how={"lam": LAMBDA, "lambda_mode": ot.OT_LAMBDA_TARGET_PROB if case["approx_kl"] else ot.OT_LAMBDA_FIXED,
                                        "ngram_term": ot.OT_NGRAM_TERM_APPROX_KL if case["approx_kl"] else ot.OT_NGRAM_TERM_NLL})
    return state


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    call, case = state["call"], state["case"]
    if own:
        v = state["v"]
        if call == "head":
            return {"logits": v.lm_head(state["hidden"])}
        if call == "loss_grad":
            got = v.distill_loss_grad(state["inp"], from_logits=True, grad_loss=state["grad_loss"], **state["how"])
            return {"grad": got["grad"], "kind": got["kind"]}
        got = v.token_logprobs(state["logits"], state["tokens"], temperature=state["temperature"], n_top=case["n_top"])
        if call == "learn":
            got["grad"] = v.token_logprobs_grad(state["logits"], state["tokens"], got, temperature=state["temperature"],
                                                grad_logprob=state["grad_logprob"], grad_entropy=state["grad_entropy"])
        return got
    if call == "head":
        return {"logits": _plain_head(state, case["group"])}
    if call == "loss_grad":
        return _plain_loss_grad(state, case["approx_kl"])
    return _plain_logprobs(state, case["n_top"])


def _plain_head(x, group):
    codes = torch.stack((x["codes"] & 15, x["codes"] >> 4), 1).reshape(-1, x["codes"].shape[1]).float()
    each = torch.arange(codes.shape[0], device=codes.device) // group
    codes -= 8.0 if x["zeros"] is None else x["zeros"].float()[each]
    codes *= x["scales"].float()[each]
    return x["hidden"].float() @ codes


def _plain_logprobs(x, n_top):
    z, T = x["logits"].float(), x["temperature"][:, None]
    mx = z.max(1, keepdim=True).values
    e = torch.exp((z - mx) / T)
    S = e.sum(1, keepdim=True)
    lp = (z - mx) / T - torch.log(S)
    p = e / S
    H = -torch.where(p > 0, p * lp, 0.0).sum(1, keepdim=True)
    given = x["tokens"].long()
    got = {"logprob": lp.gather(1, given), "entropy": H[:, 0], "row_max": mx[:, 0], "row_sumexp": S[:, 0]}
    if n_top:
        # unique whole numbers that order ids by logit, of equal ones the lowest id first; ids that the mask leaves out have none
        bits = (z + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF) - 1, bits)
        key = (order << 32) - torch.arange(z.shape[1], device=z.device)
        top = torch.topk(key, n_top, dim=1).indices
        value = lp.gather(1, top)
        got["top_ids"] = torch.where(value > -math.inf, top, -1).int()
        got["top_logprobs"] = value
    if "grad_logprob" in x:
        g, gH = x["grad_logprob"], x["grad_entropy"][:, None]
        grad = -p * g.sum(1, keepdim=True) - torch.where(p > 0, gH * p * (lp + H), 0.0)
        got["grad"] = (grad.scatter_add(1, given, g) / T).to(x["logits"].dtype)
    return got


def _pull(zq, z, T, dmap):
    """q, ln q of draft rows, ln p of target rows, and ln q - ln p + 1 of the mapped draft ids."""
    lq, lp = torch.log_softmax(zq.float() / T, 1), torch.log_softmax(z / T, 1)
    return torch.exp(lq), lq, lp, torch.where(dmap >= 0, lq - lp[:, dmap.clamp(min=0)] + 1.0, 0.0)


def _plain_loss_grad(x, approx_kl):
    terms, zq, dmap = x["terms"], x["draft_logits"], x["dmap_dev"]
    scale = x["grad_loss"] / terms["n"]
    grad = torch.zeros(zq.shape, dtype=torch.float32, device=zq.device)
    if terms["one"] is not None:
        o = terms["one"]
        q, _, _, a = _pull(zq[o["drow"]], x["logits"][o["row"]], o["T"], dmap)
        grad[o["drow"]] = scale / o["T"] * q * (a - (q * a).sum(1, keepdim=True))
    if terms["many"] is not None:
        m = terms["many"]
        at, has, T = m["at"], m["has"], m["T"]
        ids = x["ids_dev"][at]
        lq = torch.log_softmax(zq[at].float() / T[:, :, None], 2)
        lq_at = lq.gather(2, ids[:, :, None])[:, :, 0]
        if approx_kl:
            q, _, lp, a = _pull(zq[at[:, 0]], x["logits"][m["row"]], T, dmap)
            weight = torch.exp(lp.gather(1, m["t"][:, None]))
            ln_pi = torch.where(has, lq_at, 0.0).sum(1, keepdim=True)
            pi, q_first = torch.exp(ln_pi), torch.exp(lq_at[:, :1])
            q_pre = q_first - pi
            pre = (m["pre"][:, None] >= 0) & (m["pre"] != m["t"])[:, None] & (q_pre > 0)
            r_ng = ln_pi - lp.gather(1, m["t"][:, None]) + 1.0
            r_pre = torch.where(pre, torch.log(q_pre.clamp(min=1e-38)) - lp.gather(1, m["pre"].clamp(min=0)[:, None]) + 1.0, 0.0)
            out = m["inverse"][:, None]
            a = torch.where((out >= 0) & (torch.arange(q.shape[1], device=q.device)[None, :] == out), 0.0, a)
            a = a.scatter(1, ids[:, :1], r_pre)
            first = q * (a - (q * a).sum(1, keepdim=True))
            pull = ((r_ng - r_pre) * pi)[:, :, None]
        else:
            weight = torch.full_like(T, LAMBDA)
            first, pull = 0.0, torch.full_like(T, -1.0)[:, :, None]
        each = -pull * torch.exp(lq)
        each = each.scatter_add(2, ids[:, :, None], pull.expand(-1, at.shape[1], 1))
        each[:, 0] += first
        grad[at[has]] = ((scale * weight / T)[:, :, None] * each)[has]
    return {"grad": grad.to(zq.dtype), "kind": terms["kind"]}


# ------------------------------------------------------------------------------------------------ what a pass costs
def work(case):
    """Inputs read once, outputs written once; operations of the product, or a few per logit where there is none."""
    if case["call"] == "head":
        M, d, V = case["M"], case["d"], case["V"]
        groups = -(-d // case["group"])
        return {"bytes": d * V / 2 + groups * V * (2.5 if case["zeros"] else 2.0) + 2.0 * M * d + 4.0 * M * V, "flops": 2.0 * M * d * V}
    if case["call"] != "loss_grad":
        size = case["M"] * case["V"] * (2.0 if case["dtype"] == "bf16" else 4.0)
        if case["call"] == "learn":
            return {"bytes": 2.0 * size, "flops": 14.0 * case["M"] * case["V"]}
        return {"bytes": size + 4.0 * case["M"] * (2 * case["n_tok"] + 1 + 2 * case["n_top"]), "flops": 8.0 * case["M"] * case["V"]}
    k = np.random.default_rng([case["B"], case["k_min"], case["k_max"]]).integers(case["k_min"], case["k_max"] + 1, size=case["B"])
    K, esz = float(k.sum()), 2.0 if case["dtype"] == "bf16" else 4.0
    mapped = float(case["V_d"] if case["V_d"] == case["V_t"] else min(int(0.93 * case["V_d"]), int(0.8 * case["V_t"])))
    rows = K * (1.0 - case["greedy"]) * (0.7 if case["entries"] and not case["approx_kl"] else 0.9 if case["entries"] else 1.0)
    return {"bytes": rows * 4.0 * mapped + 2.0 * K * case["V_d"] * esz, "flops": 20.0 * rows * case["V_d"]}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_head(case, seed):
    x = _head_inputs(case, seed)
    d, V, G = case["d"], case["V"], case["group"]
    h = x["hidden"].double()
    out = torch.zeros(case["M"], V, dtype=torch.float64, device=DEVICE)
    for g in range(-(-d // G)):                    # group by group: the scale times the whole product of the group
        lo, hi = g * G // 2, min((g + 1) * G, d) // 2
        c = x["codes"][lo:hi]
        zero = 8.0 if x["zeros"] is None else x["zeros"][g].double()
        even, odd = (c & 15).double() - zero, (c >> 4).double() - zero
        out += x["scales"][g].double() * (h[:, 2 * lo:2 * hi:2] @ even + h[:, 2 * lo + 1:2 * hi:2] @ odd)
    return {"logits": out}


def _exact_logprobs(case, seed):
    x = _row_inputs(case, seed)
    raw = x["logits"].double()
    kept = raw > -math.inf
    z = torch.where(kept, raw, 0.0).requires_grad_(case["call"] == "learn")
    scaled = z / x["temperature"].double()[:, None]
    lp = scaled - torch.logsumexp(torch.where(kept, scaled, -math.inf), 1, keepdim=True)
    H = -torch.where(kept, torch.exp(lp) * lp, 0.0).sum(1)
    logprob = lp.gather(1, x["tokens"].long())
    mx = raw.max(1).values
    out = {"logprob": logprob.detach(), "entropy": H.detach(), "row_max": None,
           "row_sumexp": torch.exp((raw - mx[:, None]) / x["temperature"].double()[:, None]).sum(1)}
    if case["n_top"]:
        out["top_ids"] = None
        out["top_logprobs"] = torch.where(kept, lp, -math.inf).sort(1, descending=True).values[:, :case["n_top"]]
    if case["call"] == "learn":
        total = (logprob * x["grad_logprob"].double()).sum() + (H * x["grad_entropy"].double()).sum()
        out["grad"] = torch.autograd.grad(total, z)[0]
    return out


def _exact_loss_grad(case, seed):
    """The loss's definition token by token, differentiated by torch."""
    x = _loss_inputs(case, seed)
    zq = x["draft_logits"].double().requires_grad_(True)
    dmap = torch.from_numpy(x["dmap"]).to(DEVICE).long()
    mapped = torch.nonzero(dmap >= 0)[:, 0]
    total, n, grads = 0.0, 0, torch.zeros_like(zq)
    for b, got in enumerate(x["tokens"]):
        r0, q0, T = int(x["row_off"][b]), int(x["row_off"][b]) - b, float(x["T"][b])
        if T <= 0:
            continue
        total = 0.0
        for j, (t, s, L) in enumerate(got):
            n += L
            lp = torch.log_softmax(x["logits"][r0 + j].double() / T, 0)
            lq = torch.log_softmax(zq[q0 + s:q0 + s + L] / T, 1)
            ids = [int(i) for i in x["draft_ids"][q0 + s:q0 + s + L]]
            if L > 1 and not case["approx_kl"]:
                total = total - float(np.float32(LAMBDA)) * sum(lq[i, c] for i, c in enumerate(ids))
                continue
            q = torch.zeros(case["V_t"], dtype=torch.float64, device=DEVICE).index_put((dmap[mapped],), torch.exp(lq[0])[mapped])
            if L > 1:
                pi = torch.exp(sum(lq[i, c] for i, c in enumerate(ids)))
                pre = int(x["dmap"][ids[0]])
                if pre >= 0:
                    q = q.index_put((torch.tensor([pre], device=DEVICE),), (torch.exp(lq[0, ids[0]]) - pi)[None])
                q = q.index_put((torch.tensor([t], device=DEVICE),), pi[None])
            some = q > 0
            kl = (q[some] * (torch.log(q[some]) - lp[some])).sum()
            total = total + (kl * torch.exp(lp[t]) if L > 1 else kl)
        if isinstance(total, torch.Tensor):
            grads += torch.autograd.grad(total, zq)[0]
    return {"grad": grads / max(1, n), "kind": None}


def exact(case, seed):
    if case["call"] == "head":
        return _exact_head(case, seed)
    if case["call"] == "loss_grad":
        return _exact_loss_grad(case, seed)
    return _exact_logprobs(case, seed)
