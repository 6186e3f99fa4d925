"""The operators of drafted decoding as cases that can be timed and compared: a pass checks several drafted tokens of every
query of a batch.

  draft    attention of up to `rows` drafted tokens per query over the cached prompt of the query's cluster, the query's own
           keys and the drafted tokens in front of it
  project  a layer's product with 8-bit weights, a power-of-two scale for each block of 128
  probs    probabilities of rows of logits
  verify   which drafted tokens stand, and the token behind them

A case is a dict of plain values; lengths and labels follow from its `shape`, values from the seed.  `run` computes the plain form
(elementary torch operations in 32 or 64 bits), or, where `own` is set, makes the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def _draft(hq, hkv, clusters, prefix, queries, suffix, done, rows, **more):
    c = {"op": "draft", "hq": hq, "hkv": hkv, "clusters": clusters, "prefix_lo": prefix[0], "prefix_hi": prefix[1], "queries": queries,
         "suffix_lo": suffix[0], "suffix_hi": suffix[1], "done": done, "rows": rows, "ragged": True, "kv": "bf16", "rope": 500000.0, "shape": 1}
    c.update(more)
    return c


def _project(m, n, k, **more):
    c = {"op": "project", "m": m, "n": n, "k": k, "x": "bf16", "y": "bf16"}
    c.update(more)
    return c


def listed():
    return [
        # one question over one retrieved subgraph, four drafted tokens: the smallest pass, latency
        _draft(32, 8, 1, (411, 411), 1, (23, 23), 6, 5, ragged=False, name="draft_one"),
        # a handful of questions over one longer prompt, as many drafts as each has
        _draft(32, 8, 1, (3001, 3001), 5, (11, 47), 16, 6, name="draft_few"),
        # the benchmark's batch: ten prompts, 32 questions each, three drafted tokens
        _draft(32, 8, 10, (1024, 1024), 320, (16, 64), 24, 4, name="draft_batch"),
        # a layer of 64 query heads over long fp8 prompts, the largest pass of attention
        _draft(64, 8, 8, (12000, 16384), 64, (32, 256), 32, 8, kv="fp8_e4m3", name="draft_long_fp8"),
        # the QKV projection of a handful of questions' drafts: the weights' bytes
        _project(20, 6144, 4096, name="project_few"),
        # the output projection of the benchmark's batch of drafts
        _project(1280, 4096, 4096, name="project_batch"),
        # logits of a vocabulary of odd size, kept in 32 bits
        _project(64, 50021, 4096, y="f32", name="project_logits"),
        # the QKV projection of ten prompts of 1024: matrix rate
        _project(10240, 6144, 4096, name="project_prompts"),
        # probabilities of a handful of rows over a large vocabulary
        {"op": "probs", "rows": 5, "vocab": 131072, "x": "bf16", "temperature": 0.8, "name": "probs_few"},
        # ... of the benchmark's batch of drafts, rows of odd length
        {"op": "probs", "rows": 1280, "vocab": 50021, "x": "f32", "temperature": 1.0, "name": "probs_batch"},
        # drafts copied from the prompt (no draft probabilities) for a handful of questions
        {"op": "verify", "queries": 5, "rows": 6, "vocab": 131072, "draft_probs": False, "name": "verify_few"},
        # drafts of a smaller model with its probabilities, the benchmark's batch
        {"op": "verify", "queries": 320, "rows": 4, "vocab": 50021, "draft_probs": True, "name": "verify_batch"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["draft", "draft", "project", "project", "probs", "verify"])
    if op == "draft":
        hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (32, 32), (8, 2), (12, 4)])
        clusters, prefix, suffix, rows = _log(rng, 1, 16), _log(rng, 20, 12000), _log(rng, 2, 256), rng.randint(1, 16)
        c = _draft(hq, hkv, clusters, (max(1, prefix * rng.randint(40, 100) // 100), prefix), clusters * _log(rng, 1, 32),
                   (max(1, suffix * rng.randint(20, 100) // 100), suffix), rng.randint(0, 40), rows, ragged=rng.random() < 0.75,
                   kv=rng.choice(["bf16", "bf16", "fp8_e4m3"]), rope=rng.choice([10000.0, 500000.0]), shape=rng.randint(1, 1 << 20))
        cap = max(work(x)["flops"] for x in listed() if x["op"] == "draft")
        while c["queries"] > 1 and work(c)["flops"] > cap:
            c["queries"] = max(1, c["queries"] * 2 // 3)
            c["clusters"] = max(1, min(c["clusters"], c["queries"]) * 4 // 5)
        return c
    if op == "project":
        m, n, k = _log(rng, 1, 10240), _log(rng, 40, 60000), 16 * _log(rng, 8, 512)
        while m * n * k > 10240 * 6144 * 4096:
            m = max(1, m // 2)
        return _project(m, n, k, x=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["bf16", "bf16", "f32"]))
    if op == "probs":
        rows, vocab = _log(rng, 1, 1280), _log(rng, 100, 131072)
        while rows * vocab > 1280 * 50021:
            rows = max(1, rows // 2)
        return {"op": "probs", "rows": rows, "vocab": vocab, "x": rng.choice(["bf16", "f32"]), "temperature": rng.choice([0.0, 0.6, 1.0, 1.3])}
    queries, rows, vocab = _log(rng, 1, 320), rng.randint(1, 16), _log(rng, 100, 131072)
    while queries * rows * vocab > 320 * 4 * 50021:
        queries = max(1, queries // 2)
    return {"op": "verify", "queries": queries, "rows": rows, "vocab": vocab, "draft_probs": rng.random() < 0.5}


# ---- draft: lengths, inputs ------------------------------------------------------------------------------------------------
D = 128


def _structure(case):
    rng = np.random.default_rng(case["shape"])
    nc, nq, R = case["clusters"], case["queries"], case["rows"]
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, size=nc)
    labels = rng.permutation(np.arange(nq) % nc)
    suffix = rng.integers(case["suffix_lo"], case["suffix_hi"] + 1, size=nq)
    done = rng.integers(0, case["done"] + 1, size=nq) if case["ragged"] else np.full(nq, case["done"])
    rows = rng.integers(1, R + 1, size=nq) if case["ragged"] else np.full(nq, R)
    return prefix, labels, suffix, done, rows


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _device(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)


def _angles(pos, base):
    """cos and sin [..., d / 2] of integer positions, formed in 64 bits."""
    inv = base ** (-torch.arange(0, D, 2, device=pos.device, dtype=torch.float64) / D)
    a = pos.double().unsqueeze(-1) * inv
    return torch.cos(a), torch.sin(a)


def _rotate(x, pos, base):
    """Rotate-half pairing of x [..., heads, d] at pos [...], in x's own type."""
    c, s = (t.to(x.dtype).unsqueeze(-2) for t in _angles(pos, base))
    a, b = x[..., : D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


class State:
    """A program's tensors and, where the library is used, its context, cache and plan."""
    ctx = cache = plan = None

    def __del__(self):
        if self.ctx is not None:
            from paper_2505_10951_amd import sgc
            if self.plan is not None:
                sgc.sgc_plan_destroy(self.plan)
            if self.cache is not None:
                sgc.sgc_cache_destroy(self.cache)
            sgc.sgc_ctx_destroy(self.ctx)


def _draft_inputs(case, seed):
    """The resident cache (keys rotated; binary16 keys and bf16 values, or e4m3 codes with a scale per cluster and head), the queries' own
    keys as far as they are generated, and the rows of the pass, before rotation."""
    g, s = _generator(seed), State()
    s.case = case
    prefix, labels, suffix, done, rows = _structure(case)
    hq, hkv, R, nq, nc = case["hq"], case["hkv"], case["rows"], case["queries"], case["clusters"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.bfloat16)

    pm, lm = int(prefix.max()), int((suffix + done).max())
    pk, pv = normal(nc, pm, hkv, D), normal(nc, pm, hkv, D)
    pos = torch.arange(pm, device=DEVICE).expand(nc, pm)
    rot = _rotate(pk.float(), pos, case["rope"])
    seen = pos < _device(prefix)[:, None]
    if case["kv"] == "fp8_e4m3":
        s.k_cache, s.k_scale = _e4m3(rot, seen)
        s.v_cache, s.v_scale = _e4m3(pv.float(), seen)
    else:
        s.k_cache, s.v_cache = rot.half(), pv
    s.k_own, s.v_own = normal(nq, lm, hkv, D), normal(nq, lm, hkv, D)
    own_pos = _device(prefix[labels])[:, None] + torch.arange(lm, device=DEVICE)
    s.k_own_rot = _rotate(s.k_own.float(), own_pos, case["rope"]).half()
    s.q, s.k, s.v = normal(nq, R, hq, D), normal(nq, R, hkv, D), normal(nq, R, hkv, D)
    s.prefix, s.labels, s.suffix, s.n_done, s.n_rows = (a.astype(np.int32) for a in (prefix, labels, suffix, done, rows))
    s.done, s.rows = _device(s.n_done), _device(s.n_rows)
    s.d_prefix, s.d_labels, s.d_suffix = (_device(a.astype(np.int64)) for a in (prefix, labels, suffix))
    s.o = torch.zeros_like(s.q)
    return s


def _e4m3(x, seen):
    """Codes and the scale amax / 448 of each (cluster, head) over the tokens that exist."""
    amax = (x.abs() * seen[:, :, None, None]).amax(dim=(1, 3))
    scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return (x / scale[:, None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _draft_prepare(case, seed):
    s = _draft_inputs(case, seed)
    hq, hkv, R, nq, nc = case["hq"], case["hkv"], case["rows"], case["queries"], case["clusters"]
    # queries of a cluster side by side: slot [cluster][i] is a query, or nobody's
    most = int(np.bincount(s.labels, minlength=nc).max())
    slot = np.full((nc, most), -1, dtype=np.int64)
    for c in range(nc):
        mine = np.flatnonzero(s.labels == c)
        slot[c, : len(mine)] = mine
    s.slot = _device(slot)
    if own:
        from paper_2505_10951_amd import sgc
        fp8 = case["kv"] == "fp8_e4m3"
        cap = case["done"] + R
        params = sgc.make_params(n_q_heads=hq, n_kv_heads=hkv, head_dim=D, io_dtype="bf16", kv_dtype=case["kv"], rope_base=case["rope"],
                                 max_position=int(s.prefix.max() + s.suffix.max()) + cap)
        s.ctx = sgc.sgc_ctx_create(params)
        nbytes = sgc.sgc_cache_pool_bytes(params, int(sum(-(-int(p) // 16) for p in s.prefix)))
        s.pool = torch.empty(nbytes, dtype=torch.uint8, device=DEVICE)
        s.cache = sgc.sgc_cache_create(s.ctx, s.pool.data_ptr(), nbytes, nc)
        for c in range(nc):
            sgc.sgc_cache_alloc_cluster(s.ctx, s.cache, c, int(s.prefix[c]))
            scales = (s.k_scale[c].cpu().numpy(), s.v_scale[c].cpu().numpy()) if fp8 else (None, None)
            sgc.sgc_cache_import(s.ctx, s.cache, c, 0, s.k_cache[c].data_ptr(), s.v_cache[c].data_ptr(), *scales, _stream())
        s.plan = sgc.sgc_assign_clusters(s.ctx, s.cache, s.labels, s.suffix, nc)[3]
        sgc.sgc_plan_enable_drafts(s.ctx, s.plan, cap, R)
        # the questions' prefill, then passes that bring the tokens generated so far
        at = np.concatenate([n * s.k_own.shape[1] + np.arange(int(s.suffix[n])) for n in range(nq)])
        k, v = (t.reshape(-1, hkv, D)[_device(at)].contiguous() for t in (s.k_own, s.v_own))
        q = torch.zeros((len(at), hq, D), dtype=torch.bfloat16, device=DEVICE)
        sgc.sgc_suffix_prefill_batched(s.ctx, s.cache, s.plan, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), torch.empty_like(q).data_ptr(), None, _stream())
        for t0 in range(0, int(s.n_done.max()), R):
            idx = (s.d_suffix[:, None] + t0 + torch.arange(R, device=DEVICE)).clamp(max=s.k_own.shape[1] - 1)[:, :, None, None].expand(nq, R, hkv, D)
            k, v = s.k_own.gather(1, idx), s.v_own.gather(1, idx)
            rows, done = (s.done - t0).clamp(0, R).int(), torch.full_like(s.done, t0)
            sgc.sgc_draft_step_batched(s.ctx, s.cache, s.plan, 0, done.data_ptr(), rows.data_ptr(), s.q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                       torch.empty_like(s.q).data_ptr(), None, _stream())
        torch.cuda.synchronize()
    return s


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _draft_run(s):
    if own:
        from paper_2505_10951_amd import sgc
        sgc.sgc_draft_step_batched(s.ctx, s.cache, s.plan, 0, s.done.data_ptr(), s.rows.data_ptr(), s.q.data_ptr(), s.k.data_ptr(), s.v.data_ptr(),
                                   s.o.data_ptr(), None, _stream())
        return s.o
    case, lm = s.case, s.k_own.shape[1]
    hq, hkv, R, nq = case["hq"], case["hkv"], case["rows"], case["queries"]
    nc, pm, grp = s.k_cache.shape[0], s.k_cache.shape[1], hq // hkv
    j = torch.arange(R, device=DEVICE)
    base = s.d_prefix[s.d_labels] + s.d_suffix + s.done
    q = _rotate(s.q.float(), base[:, None] + j, case["rope"]) * (1.0 / math.sqrt(D))
    k_new = _rotate(s.k.float(), base[:, None] + j, case["rope"])
    if case["kv"] == "fp8_e4m3":
        kc = s.k_cache.view(torch.float8_e4m3fn).float() * s.k_scale[:, None, :, None]
        vc = s.v_cache.view(torch.float8_e4m3fn).float() * s.v_scale[:, None, :, None]
    else:
        kc, vc = s.k_cache.float(), s.v_cache.float()
    # scores against the cached prompt, all queries of a cluster at once: [cluster][kv head][slot x row x head of the group][key]
    qh = q.view(nq, R, hkv, grp, D).permute(0, 2, 1, 3, 4)                        # [query][kv head][row][head]
    qc = qh[s.slot.clamp(min=0)].permute(0, 2, 1, 3, 4, 5).reshape(nc, hkv, -1, D)
    sc = qc @ kc.permute(0, 2, 3, 1)
    sc.masked_fill_((torch.arange(pm, device=DEVICE) >= s.d_prefix[:, None])[:, None, None, :], float("-inf"))
    # ... and against the query's own keys: question, generated, and the rows up to its own
    ko = torch.cat([s.k_own_rot.float(), k_new], dim=1)
    vo = torch.cat([s.v_own.float(), s.v.float()], dim=1)
    so = qh.reshape(nq, hkv, R * grp, D) @ ko.permute(0, 2, 3, 1)
    old = (torch.arange(lm, device=DEVICE) < (s.d_suffix + s.done)[:, None])[:, None, :].expand(nq, R, lm)
    see = torch.cat([old, (j[None, :] <= j[:, None]).expand(nq, R, R)], dim=2)
    so.masked_fill_(~see[:, None, :, None, :].expand(nq, hkv, R, grp, lm + R).reshape(nq, hkv, R * grp, lm + R), float("-inf"))
    # one softmax over both
    mc = sc.amax(dim=-1, keepdim=True)
    place = torch.empty(nq, dtype=torch.int64, device=DEVICE)
    real = s.slot.reshape(-1) >= 0
    place[s.slot.reshape(-1)[real]] = torch.arange(s.slot.numel(), device=DEVICE)[real]

    def of_query(t):                         # [cluster][kv head][slot x row x head][c] -> [query][kv head][row x head][c]
        w = t.shape[-1]
        return t.reshape(nc, hkv, -1, R * grp, w).permute(0, 2, 1, 3, 4).reshape(-1, hkv, R * grp, w)[place]

    pc = torch.exp(sc.sub_(mc))
    lc, oc, mc = of_query(pc.sum(dim=-1, keepdim=True)), of_query(pc @ vc.permute(0, 2, 1, 3)), of_query(mc)
    mo = so.amax(dim=-1, keepdim=True)
    po = torch.exp(so.sub_(mo))
    m = torch.maximum(mc, mo)
    wc, wo = torch.exp(mc - m), torch.exp(mo - m)
    o = (oc * wc + (po @ vo.permute(0, 2, 1, 3)) * wo) / (lc * wc + po.sum(dim=-1, keepdim=True) * wo)
    o = o.view(nq, hkv, R, grp, D).permute(0, 2, 1, 3, 4).reshape(nq, R, hq, D)
    return torch.where((j < s.rows[:, None])[:, :, None, None], o, s.o.float()).to(s.o.dtype)


def _draft_exact(case, seed):
    s = _draft_inputs(case, seed)
    hq, hkv, R = case["hq"], case["hkv"], case["rows"]
    out = torch.zeros((case["queries"], R, hq, D), dtype=torch.float64, device=DEVICE)
    for c in range(case["clusters"]):
        P = int(s.prefix[c])
        kc, vc = s.k_cache[c, :P], s.v_cache[c, :P]
        if case["kv"] == "fp8_e4m3":
            kc = kc.view(torch.float8_e4m3fn).double() * s.k_scale[c].double()[:, None]
            vc = vc.view(torch.float8_e4m3fn).double() * s.v_scale[c].double()[:, None]
        kc, vc = kc.double().transpose(0, 1), vc.double().transpose(0, 1)                     # [kv head][key][d]
        for n in np.flatnonzero(s.labels == c):
            L, r = int(s.suffix[n] + s.n_done[n]), int(s.n_rows[n])
            pos = P + L + torch.arange(r, device=DEVICE)
            q = _rotate(s.q[n, :r].double(), pos, case["rope"]).view(r, hkv, hq // hkv, D).permute(1, 0, 2, 3).reshape(hkv, -1, D)
            k = torch.cat([kc, s.k_own_rot[n, :L].double().transpose(0, 1), _rotate(s.k[n, :r].double(), pos, case["rope"]).transpose(0, 1)], dim=1)
            v = torch.cat([vc, s.v_own[n, :L].double().transpose(0, 1), s.v[n, :r].double().transpose(0, 1)], dim=1)
            a = (q @ k.transpose(1, 2)) / math.sqrt(D)
            last = (P + L + torch.arange(r, device=DEVICE)).repeat_interleave(hq // hkv)
            a = torch.softmax(a.masked_fill(torch.arange(P + L + r, device=DEVICE) > last[:, None], float("-inf")), dim=-1)
            out[n, :r] = (a @ v).view(hkv, r, hq // hkv, D).permute(1, 0, 2, 3).reshape(r, hq, D)
    return out


def _draft_work(case):
    prefix, labels, suffix, done, rows = _structure(case)
    hq, hkv, kv = case["hq"], case["hkv"], 1 if case["kv"] == "fp8_e4m3" else 2
    cached = 2.0 * hkv * D * kv * prefix[np.unique(labels)].sum()
    held = 4.0 * hkv * D * (suffix + done).sum()
    seen = rows * (prefix[labels] + suffix + done) + rows * (rows + 1) / 2.0
    return {"bytes": float(cached + held + rows.sum() * (4.0 * hq * D + 8.0 * hkv * D)), "flops": float(4.0 * hq * D * seen.sum())}


# ---- project: x W^T in e4m3, a power-of-two scale (as its biased exponent) for each 128 of a row of x and each 128 x 128 of W -----
def _exponent(amax):
    """Smallest e with amax <= 448 * 2^e, at least -127; 0 where there is nothing."""
    m, e = torch.frexp(amax / 448.0)
    return torch.where(amax > 0, torch.where(m == 0.5, e - 1, e).clamp(-127, 127), torch.zeros_like(e))


def _blocks(x):
    """[rows][k] -> [rows][blocks][128], filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % 128)).unflatten(1, (-1, 128))


def _project_inputs(case, seed):
    g, s = _generator(seed), State()
    s.case = case
    m, n, k = case["m"], case["n"], case["k"]
    s.x = torch.randn((m, k), generator=g, device=DEVICE, dtype=TORCH[case["x"]])
    w = torch.randn((n, k), generator=g, device=DEVICE, dtype=torch.bfloat16) * (1.0 / math.sqrt(k))
    w = _blocks(torch.nn.functional.pad(w, (0, 0, 0, -n % 128)).float())                      # [n'][kb][128]
    e = _exponent(w.abs().unflatten(0, (-1, 128)).amax(dim=(1, 3)))                           # [n' / 128][kb]
    w = torch.ldexp(w, -e.repeat_interleave(128, 0)[:, :, None])
    s.w_codes = w.to(torch.float8_e4m3fn).view(torch.uint8).flatten(1)[:n].contiguous()
    s.w_exponents = (e + 127).to(torch.uint8).contiguous()
    return s


def _project_prepare(case, seed):
    s = _project_inputs(case, seed)
    if own:
        from paper_2505_10951_amd import sgc
        s.ctx = sgc.sgc_ctx_create(sgc.make_params(n_q_heads=32, n_kv_heads=8, head_dim=128))
        s.ws = torch.empty(sgc.sgc_project_fp8_workspace(case["m"], case["n"], case["k"]), dtype=torch.uint8, device=DEVICE)
        s.y = torch.empty((case["m"], case["n"]), dtype=TORCH[case["y"]], device=DEVICE)
    return s


def _weights(s, dtype):
    e = s.w_exponents.to(dtype) - 127
    w = s.w_codes.view(torch.float8_e4m3fn).to(dtype).unflatten(1, (-1, 128))
    return (w * torch.exp2(e).repeat_interleave(128, 0)[: w.shape[0], :, None]).flatten(1)


def _project_run(s):
    case = s.case
    if own:
        from paper_2505_10951_amd import sgc
        types = {"bf16": sgc.SGC_BF16, "f32": sgc.SGC_F32}
        sgc.sgc_project_fp8(s.ctx, s.x.data_ptr(), types[case["x"]], case["k"], case["m"], s.w_codes.data_ptr(), s.w_exponents.data_ptr(), case["n"],
                            case["k"], s.y.data_ptr(), types[case["y"]], case["n"], s.ws.data_ptr(), s.ws.numel(), _stream())
        return s.y
    x = _blocks(s.x.float())
    e = _exponent(x.abs().amax(dim=2, keepdim=True))
    x = torch.ldexp(torch.ldexp(x, -e).to(torch.float8_e4m3fn).float(), e).flatten(1)
    return (x @ _weights(s, torch.float32).t()).to(TORCH[case["y"]])


def _project_exact(case, seed):
    if 2.0 * case["m"] * case["n"] * case["k"] > 6e11 or case["n"] * case["k"] > 3e8:
        return None
    s = _project_inputs(case, seed)
    x = _blocks(s.x.double())
    a = x.abs().amax(dim=2, keepdim=True)
    e = torch.where(a > 0, torch.ceil(torch.log2(a / 448.0)), torch.zeros_like(a))
    e = torch.where(448.0 * torch.exp2(e - 1) >= a, e - 1, e)          # (where the logarithm came out just above a whole number)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)             # e4m3: four significant bits, 2^-9 at the bottom
    y = (torch.round(y / step) * step * torch.exp2(e)).flatten(1)
    return y @ _weights(s, torch.float64).t()


def _project_work(case):
    m, n, k = case["m"], case["n"], case["k"]
    b = {"bf16": 2, "f32": 4}
    kb = -(-k // 128)
    return {"bytes": float(n * k + -(-n // 128) * kb + m * k * b[case["x"]] + m * n * b[case["y"]]), "flops": 2.0 * m * n * k}


# ---- probs -------------------------------------------------------------------------------------------------------------------
def _logits(g, rows, vocab, dtype):
    """Logits of a few likely tokens over a bulk, a part of the vocabulary ruled out."""
    x = torch.randn((rows, vocab), generator=g, device=DEVICE) * 3.0
    x = x + 9.0 * (torch.rand((rows, vocab), generator=g, device=DEVICE) < 8.0 / vocab)
    x.masked_fill_(torch.rand((rows, vocab), generator=g, device=DEVICE) < 0.02, float("-inf"))
    return x.to(dtype)


def _probs_inputs(case, seed):
    s = State()
    s.case = case
    s.x = _logits(_generator(seed), case["rows"], case["vocab"], TORCH[case["x"]])
    if case["rows"] > 3:
        s.x[3] = float("-inf")               # a row that is ruled out whole
    return s


def _probs_prepare(case, seed):
    s = _probs_inputs(case, seed)
    if own:
        from paper_2505_10951_amd import sgc
        s.ctx = sgc.sgc_ctx_create(sgc.make_params(n_q_heads=32, n_kv_heads=8, head_dim=128))
        s.ws = torch.empty(max(1, sgc.sgc_token_probs_workspace(case["rows"], case["vocab"])), dtype=torch.uint8, device=DEVICE)
        s.p = torch.empty((case["rows"], case["vocab"]), device=DEVICE)
    return s


def _probs_run(s):
    case = s.case
    if own:
        from paper_2505_10951_amd import sgc
        sgc.sgc_token_probs(s.ctx, case["rows"], case["vocab"], s.x.data_ptr(), {"bf16": sgc.SGC_BF16, "f32": sgc.SGC_F32}[case["x"]], case["vocab"],
                            case["temperature"], s.p.data_ptr(), case["vocab"], s.ws.data_ptr(), s.ws.numel(), _stream())
        return s.p
    x = s.x.float()
    top = x.amax(dim=1, keepdim=True)
    some = top > float("-inf")
    if case["temperature"] == 0.0:
        first = (x == top).to(torch.int8).argmax(dim=1, keepdim=True)
        return ((torch.arange(case["vocab"], device=DEVICE) == first) & some).float()
    e = torch.exp((x - torch.where(some, top, torch.zeros_like(top))) * (1.0 / case["temperature"]))
    return e / torch.where(some, e.sum(dim=1, keepdim=True), torch.ones_like(top))


def _probs_exact(case, seed):
    x = _probs_inputs(case, seed).x.double()
    out = torch.zeros_like(x)
    if case["temperature"] == 0.0:
        best = torch.from_numpy(np.argmax(x.cpu().numpy(), axis=1)).to(DEVICE)
        out.scatter_(1, best[:, None], 1.0)
    else:
        out = torch.softmax(x / case["temperature"], dim=1)
    out[torch.isinf(x).all(dim=1)] = 0.0
    return out


def _probs_work(case):
    n = float(case["rows"]) * case["vocab"]
    return {"bytes": n * ({"bf16": 2, "f32": 4}[case["x"]] + 4), "flops": 4.0 * n}


# ---- verify ------------------------------------------------------------------------------------------------------------------
def _verify_prepare(case, seed):
    g, s = _generator(seed), State()
    s.case = case
    nq, R, V = case["queries"], case["rows"], case["vocab"]
    x = _logits(g, nq * R, V, torch.float32)
    s.p = torch.softmax(x, dim=1).view(nq, R, V)
    x = x.view(nq, R, V)[:, : R - 1]
    x = torch.softmax(x + torch.randn(x.shape, generator=g, device=DEVICE), dim=2)           # a smaller model's
    s.tokens = torch.zeros((nq, R), dtype=torch.int32, device=DEVICE)
    if R > 1:
        # a draft drawn from the draft's probabilities: the largest of p / (an exponential variate)
        s.tokens[:, 1:] = (x / (-torch.log1p(-torch.rand(x.shape, generator=g, device=DEVICE))).clamp(min=1e-30)).argmax(dim=2).int()
    s.q = x.contiguous() if case["draft_probs"] and R > 1 else None
    s.rows = torch.randint(1, R + 1, (nq,), generator=g, device=DEVICE, dtype=torch.int32)
    s.u = torch.rand((nq, R), generator=g, device=DEVICE)
    if own:
        from paper_2505_10951_amd import sgc
        s.ctx = sgc.sgc_ctx_create(sgc.make_params(n_q_heads=32, n_kv_heads=8, head_dim=128))
        s.ws = torch.empty(max(1, sgc.sgc_verify_workspace(nq, V)), dtype=torch.uint8, device=DEVICE)
        s.out, s.accepted = torch.empty_like(s.tokens), torch.empty_like(s.rows)
    return s


def _verify_run(s):
    case = s.case
    nq, R, V = case["queries"], case["rows"], case["vocab"]
    if own:
        from paper_2505_10951_amd import sgc
        sgc.sgc_verify_drafts(s.ctx, nq, R, V, s.p.data_ptr(), V, None if s.q is None else s.q.data_ptr(), V, s.tokens.data_ptr(), s.rows.data_ptr(),
                              s.u.data_ptr(), s.out.data_ptr(), s.accepted.data_ptr(), None, s.ws.data_ptr(), s.ws.numel(), _stream())
        return s.out, s.accepted
    # how many drafts stand: draft j + 1 is judged by row j's probabilities
    x = s.tokens[:, 1:].long()
    px = s.p[:, : R - 1].gather(2, x[:, :, None]).squeeze(2).double()
    qx = torch.ones_like(px) if s.q is None else s.q.gather(2, x[:, :, None]).squeeze(2).double()
    stands = (s.u[:, : R - 1].double() * qx < px) & (torch.arange(1, R, device=DEVICE) < s.rows[:, None])
    accepted = stands.long().cumprod(dim=1).sum(dim=1)
    # the token behind them: from what the draft's probabilities leave of the target's, or behind the last draft from the target's
    n = torch.arange(nq, device=DEVICE)
    p = s.p[n, accepted].double()
    refused = accepted + 1 < s.rows
    at = accepted.clamp(max=max(R - 2, 0))
    if R == 1:
        q = torch.zeros_like(p)
    elif s.q is None:
        q = torch.zeros_like(p).scatter_(1, x.gather(1, at[:, None]), 1.0)
    else:
        q = s.q[n, at].double()
    w = torch.where(refused[:, None], (p - q).clamp(min=0), p)
    w = torch.where((w.sum(dim=1) > 0)[:, None], w, p)
    c = w.cumsum(dim=1)
    token = (c > s.u[:, R - 1: R].double() * c[:, -1:]).to(torch.int8).argmax(dim=1)
    j = torch.arange(R, device=DEVICE)
    ahead = torch.cat([s.tokens[:, 1:], torch.zeros_like(s.tokens[:, :1])], dim=1)
    out = torch.where(j < accepted[:, None], ahead, torch.where(j == accepted[:, None], token[:, None].int(), torch.full_like(ahead, -1)))
    return out, accepted.int()


def _verify_work(case):
    nq, R, V = float(case["queries"]), case["rows"], case["vocab"]
    rows = 1.0 + (0.5 if case["draft_probs"] and R > 1 else 0.0)         # about half the queries end on a refusal
    return {"bytes": nq * (4.0 * V * rows + 16.0 * R), "flops": 3.0 * nq * V}


# ----------------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    return {"draft": _draft_prepare, "project": _project_prepare, "probs": _probs_prepare, "verify": _verify_prepare}[case["op"]](case, seed)


def run(state):
    return {"draft": _draft_run, "project": _project_run, "probs": _probs_run, "verify": _verify_run}[state.case["op"]](state)


def exact(case, seed):
    if case["op"] == "verify":
        return None                      # whole numbers
    return {"draft": _draft_exact, "project": _project_exact, "probs": _probs_exact}[case["op"]](case, seed)


def work(case):
    return {"draft": _draft_work, "project": _project_work, "probs": _probs_work, "verify": _verify_work}[case["op"]](case)
