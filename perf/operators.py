"""Timed cases of the attention operators: queries of one sequence over the keys
of another (cross attention), and attention with a relative position bias
learned by buckets, each as a training step, as a forward pass alone and for
single tokens.

A case is one call of `attn_forward`, or of it and `attn_backward`, on tensors
that a program holds at that point: projected queries, keys and values, the key
mask of a padded batch, the bias table, the gradient that comes back.

Fields of a case:
  kind    "cross" (keys of another length, no bias) or "relpos" (self attention
          with the bias; causal: one direction of buckets, else both)
  mode    "step" (forward and backward), "forward" or "token" (few queries per
          sequence against all keys held for it)
  batch, heads, kv_heads, seq_q, seq_k, dtype ("bf16" or "f32")
  len_lo, len_hi   range of the sequences' numbers of valid keys; 0, 0: all.
          relpos tokens: the position after a sequence's last query; the cache
          behind it holds what an earlier sequence left there
  causal, buckets, max_distance
"""
import math

import numpy as np
import torch

own = False
HEAD_DIM = 64


def _case(name, kind, mode, dtype, batch, heads, kv_heads, seq_q, seq_k, len_lo=0, len_hi=0,
          causal=False, buckets=0, max_distance=0):
    return {"name": name, "kind": kind, "mode": mode, "dtype": dtype, "batch": batch,
            "heads": heads, "kv_heads": kv_heads, "seq_q": seq_q, "seq_k": seq_k,
            "len_lo": len_lo, "len_hi": len_hi, "causal": causal, "buckets": buckets,
            "max_distance": max_distance}


def listed():
    return [
        # One token of one sequence over one sentence's encoder states (12
        # heads, 77 keys): the smallest call, launch and memory latency only.
        _case("cross_token_one", "cross", "token", "bf16", 1, 12, 12, 1, 77),
        # A token for each of 32 sequences over padded encoder outputs of the
        # 32 x 512 batch.
        _case("cross_token_batch", "cross", "token", "bf16", 32, 16, 16, 1, 512, 128, 512),
        # A token for each of 16 sequences over long documents: 0.5 GB of keys
        # and values, read once.
        _case("cross_token_long", "cross", "token", "bf16", 16, 16, 16, 1, 8192),
        # A token of each sequence over its own cache with the one-directional
        # bias, four query heads to a key head, every sequence at its own
        # position.
        _case("relpos_token_grouped", "relpos", "token", "bf16", 8, 16, 4, 1, 4096, 700, 4096,
              True, 32, 128),
        # The fp32 check of a training step: sentences of 32 tokens over
        # states of 45.
        _case("cross_tiny_f32_step", "cross", "step", "f32", 2, 2, 2, 32, 45, 16, 45),
        # A micro-batch with odd lengths, as a pipeline splits its batch.
        _case("cross_micro_step", "cross", "step", "bf16", 3, 12, 12, 77, 201, 20, 201),
        # Targets of 128 tokens over the padded 32 x 512 batch, one sequence
        # may be empty.
        _case("cross_large_step", "cross", "step", "bf16", 32, 16, 16, 128, 512, 0, 512),
        # fp32 self attention with the bias at the sentences' length.
        _case("relpos_f32_step", "relpos", "step", "f32", 8, 12, 12, 128, 128, 64, 128, False, 32,
              128),
        # One layer's attention of the 32 x 512 batch with uneven sentences.
        _case("relpos_base_step", "relpos", "step", "bf16", 32, 12, 12, 512, 512, 256, 512, False,
              32, 128),
        # The same with 16 heads, an odd length and one direction (a decoder's
        # self attention).
        _case("relpos_causal_step", "relpos", "step", "bf16", 13, 16, 16, 387, 387, 0, 0, True, 32,
              128),
        # Evaluation of long documents.
        _case("relpos_long_forward", "relpos", "forward", "bf16", 2, 16, 16, 4096, 4096, 0, 0,
              False, 32, 128),
        # Training on long documents, grouped heads, wider buckets.
        _case("relpos_long_step", "relpos", "step", "bf16", 1, 16, 4, 2500, 2500, 0, 0, True, 64,
              512),
    ]


def _mean_len(c):
    return (c["len_lo"] + c["len_hi"]) / 2.0 if c["len_hi"] else float(c["seq_k"])


def _pairs(c):
    """(query, key) pairs of one head and sequence."""
    if c["causal"] and c["mode"] != "token":
        return c["seq_q"] * (c["seq_q"] + 1) / 2.0
    return c["seq_q"] * _mean_len(c)


def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    B, H, G, Sq, D = c["batch"], c["heads"], c["kv_heads"], c["seq_q"], HEAD_DIM
    keys = _mean_len(c)
    qrow, krow = B * Sq * H * D * esz, B * keys * G * D * esz
    step = c["mode"] == "step"
    # q, k, v and out (step: the gradients of all four too), lse, mask, table
    nbytes = (2 * qrow + 2 * krow) * (2 if step else 1) + B * H * Sq * 4
    if step:
        nbytes += 2 * B * (c["seq_k"] - keys) * G * D * esz  # zero gradients of masked keys
    if c["len_hi"] and c["kind"] == "cross":
        nbytes += B * c["seq_k"]
    nbytes += c["buckets"] * H * 4 * (2 if step else 1)
    return {"bytes": nbytes, "flops": (14.0 if step else 4.0) * D * B * H * _pairs(c)}


def draw(rng):
    """One more case: kinds, modes, types, heads, batches and lengths over the
    ranges of the listed cases."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(work(c)["flops"] for c in listed())
    most_f32 = 16 * max(work(c)["flops"] for c in listed() if c["dtype"] == "f32")
    most_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(("cross", "relpos"))
        mode = rng.choice(("token", "token", "step", "step", "step", "forward"))
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        kv = rng.choice((1, 2, 3, 4, 8, 12, 16))
        heads = kv * rng.choice((1, 1, 1, 2, 4, 8))
        batch = spread(1, 32)
        causal, buckets, max_distance = False, 0, 0
        if kind == "relpos":
            causal = mode == "token" or rng.random() < 0.4
            buckets = rng.choice((16, 32, 32, 32, 64))
            max_distance = rng.choice((64, 128, 128, 256, 512))
        if mode == "token":
            seq_q, seq_k = rng.choice((1, 1, 1, 2, 4)), spread(24, 8192)
        elif kind == "relpos":
            seq_q = seq_k = spread(20, 4096)
        else:
            seq_q, seq_k = spread(9, 2048), spread(17, 4096)
        lo = hi = 0
        if (mode == "token" and kind == "relpos") or (rng.random() < 0.6 and not causal):
            hi = rng.randint(max(seq_k // 2, 12), seq_k)
            lo = rng.randint(max(hi // 4, 8), hi)
        c = _case("", kind, mode, dtype, batch, heads, kv, seq_q, seq_k, lo, hi, causal, buckets,
                  max_distance)
        del c["name"]
        w = work(c)
        if heads <= 32 and w["flops"] <= (most_f32 if dtype == "f32" else most) and \
                w["bytes"] <= most_bytes:
            return c


def _inputs(case, seed):
    """The tensors of a case, on the GPU, from the seed alone.  Self attention
    and the projections of encoder states come as views of one packed tensor
    where a program has them from one product."""
    c = case
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 777)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, H, G, Sq, Sk, D = (c["batch"], c["heads"], c["kv_heads"], c["seq_q"], c["seq_k"], HEAD_DIM)

    def normal(shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    if c["kind"] == "relpos" and c["mode"] != "token" and G == H:
        q, k, v = normal((B, Sq, 3, H, D)).to(dt).unbind(2)
    else:
        q = normal((B, Sq, H, D)).to(dt)
        k, v = normal((B, Sk, 2, G, D)).to(dt).unbind(2)
    lens = np.random.default_rng(seed).integers(c["len_lo"], c["len_hi"], size=B, endpoint=True)
    mask = q_pos = table = dout = None
    if c["mode"] == "token" and c["kind"] == "relpos":
        q_pos = torch.from_numpy((lens - Sq).astype(np.int32)).cuda()
    elif c["len_hi"]:
        mask = torch.from_numpy((np.arange(Sk)[None, :] < lens[:, None]).astype(np.uint8)).cuda()
    if c["buckets"]:
        table = normal((c["buckets"], H), 0.5)
    if c["mode"] == "step":
        dout = normal((B, Sq, H, D)).to(dt)
    return {"q": q, "k": k, "v": v, "mask": mask, "q_pos": q_pos, "table": table, "dout": dout}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    s["scale"] = 1.0 / math.sqrt(HEAD_DIM)
    if own:
        import paper_2202_11836_amd as P
        c = case
        q, k = s["q"], s["k"]
        B, Sq, H, D = q.shape
        Sk, G = k.shape[1], k.shape[2]
        s["relpos"] = P.RelPos(c["buckets"], c["max_distance"], not c["causal"]) \
            if c["buckets"] else None
        s["out"] = torch.empty((B, Sq, H, D), dtype=q.dtype, device="cuda")
        s["lse"] = torch.empty((B, H, Sq), dtype=torch.float32, device="cuda")
        if c["mode"] == "step":
            if c["kind"] == "relpos" and G == H:
                s["grads"] = torch.empty((B, Sq, 3, H, D), dtype=q.dtype, device="cuda").unbind(2)
            else:
                dq = torch.empty((B, Sq, H, D), dtype=q.dtype, device="cuda")
                dk, dv = torch.empty((B, Sk, 2, G, D), dtype=q.dtype, device="cuda").unbind(2)
                s["grads"] = (dq, dk, dv)
            s["dtable"] = torch.empty_like(s["table"]) if c["buckets"] else None
    return s


# ---------------------------------------------------------------------------
# Plain form, in 32 bits
# ---------------------------------------------------------------------------
def _bucket(rel, buckets, max_distance, both):
    """Bucket of a distance rel = key position - query position.  Half of a
    direction's buckets hold one distance each, the others grow with its
    logarithm up to max_distance (in 64 bits: borders that are whole numbers
    belong to the bucket that they open)."""
    base = torch.zeros_like(rel)
    if both:
        buckets //= 2
        base = (rel > 0).to(rel.dtype) * buckets
        n = rel.abs()
    else:
        n = (-rel).clamp(min=0)
    one = buckets // 2
    log = torch.log(n.clamp(min=1).double() / one) / math.log(max_distance / one)
    far = one + torch.floor(log * (buckets - one) + 1e-9).to(rel.dtype)
    return base + torch.where(n < one, n, far.clamp(max=buckets - 1))


def _visible(s):
    """(bucket of every pair or None, truth of every visible pair or None);
    shapes broadcast to [B, 1, Sq, Sk]."""
    c, q, k = s["case"], s["q"], s["k"]
    B, Sq, Sk = q.shape[0], q.shape[1], k.shape[1]
    see = None if s["mask"] is None else (s["mask"] != 0)[:, None, None, :]
    if not c["buckets"]:
        return None, see
    qi = torch.arange(Sq, device="cuda")[None, :, None]
    if s["q_pos"] is not None:
        qi = qi + s["q_pos"].long()[:, None, None]
    rel = (torch.arange(Sk, device="cuda")[None, None, :] - qi)[:, None]
    if c["causal"]:
        see = rel <= 0 if see is None else see & (rel <= 0)
    return _bucket(rel, c["buckets"], c["max_distance"], not c["causal"]), see


def _heads(t, H):
    """[B, S, G, D] -> [B, H, S, D] in 32 bits, key heads repeated."""
    t = t.float().transpose(1, 2)
    if t.shape[1] != H:
        t = t.repeat_interleave(H // t.shape[1], 1)
    return t.contiguous()


def _run_plain(s):
    c = s["case"]
    H, G, dt = c["heads"], c["kv_heads"], s["q"].dtype
    q, k, v = _heads(s["q"], H), _heads(s["k"], H), _heads(s["v"], H)
    bucket, see = _visible(s)
    sc = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]
    if bucket is not None:
        sc += s["table"][bucket[:, 0]].permute(0, 3, 1, 2)
    if see is not None:
        sc = sc.masked_fill(~see, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(top == -math.inf, torch.zeros_like(top), top))
    del sc
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    p /= torch.where(total == 0, torch.ones_like(total), total)
    out = torch.matmul(p, v).transpose(1, 2).contiguous().to(dt)
    got = {"out": out, "lse": lse}
    if c["mode"] != "step":
        return got
    do = _heads(s["dout"], H)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    del p, dp
    dq = torch.matmul(ds, k) * s["scale"]
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q) * s["scale"]

    def back(t):
        return t.transpose(1, 2).contiguous().to(dt)

    def shared(t):
        B, _, S, D = t.shape
        return back(t.reshape(B, G, H // G, S, D).sum(2))

    got.update(dq=back(dq), dk=shared(dk), dv=shared(dv))
    if bucket is not None:
        # Sum along the diagonals (one distance each): rows in reverse order and
        # one element longer than the view that reads them.
        Sq, Sk = ds.shape[2:]
        rows = torch.nn.functional.pad(ds.sum(0).flip(1), (0, Sq)).reshape(H, -1)
        by_rel = rows[:, :Sq * (Sq + Sk - 1)].reshape(H, Sq, -1).sum(1, dtype=torch.float64)
        rel = torch.arange(1 - Sq, Sk, device="cuda")
        ids = _bucket(rel, c["buckets"], c["max_distance"], not c["causal"])
        total = torch.zeros((c["buckets"], H), dtype=torch.float64, device="cuda")
        got["dtable"] = total.index_add_(0, ids, by_rel.t().contiguous()).float()
    return got


def run(state):
    if not own:
        return _run_plain(state)
    import paper_2202_11836_amd as P
    s, c = state, state["case"]
    kw = dict(key_mask=s["mask"], scale=s["scale"], causal=c["causal"], q_pos=s["q_pos"],
              relpos=s["relpos"], table=s["table"])
    out, lse = P.attn_forward(s["q"], s["k"], s["v"], out=s["out"], lse=s["lse"], **kw)
    if c["mode"] != "step":
        return {"out": out, "lse": lse}
    dq, dk, dv = s["grads"]
    P.attn_backward(s["q"], s["k"], s["v"], out, lse, s["dout"], dq=dq, dk=dk, dv=dv,
                    dtable=s["dtable"], **kw)
    got = {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    if s["dtable"] is not None:
        got["dtable"] = s["dtable"]
    return got


# ---------------------------------------------------------------------------
# From the definition in 64 bits, one sequence at a time
# ---------------------------------------------------------------------------
def _buckets64(buckets, max_distance, both, far):
    """Bucket of the distances 0 .. far of one direction, by whole numbers: the
    bucket one + j begins at the least n with (n / one)^m >= (max / one)^j."""
    nb = buckets // 2 if both else buckets
    one = nb // 2
    m = nb - one
    got, j = [], 0
    for n in range(far + 1):
        while n >= one and j + 1 < m and \
                n ** m * one ** (j + 1) >= one ** m * max_distance ** (j + 1):
            j += 1
        got.append(n if n < one else one + j)
    return np.array(got, dtype=np.int64), nb


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    H, G, Sq, Sk = c["heads"], c["kv_heads"], c["seq_q"], c["seq_k"]
    scale, step = 1.0 / math.sqrt(HEAD_DIM), c["mode"] == "step"
    table = None if s["table"] is None else s["table"].double()
    got = {n: [] for n in ("out", "lse", "dq", "dk", "dv")}
    dtable = torch.zeros((c["buckets"], H), dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        seen = torch.ones((Sq, Sk), dtype=torch.bool, device="cuda")
        if s["mask"] is not None:
            seen &= s["mask"][b].bool()[None, :]
        first = int(s["q_pos"][b]) if s["q_pos"] is not None else 0
        where = np.arange(Sk)[None, :] - (first + np.arange(Sq))[:, None]
        if c["causal"]:
            seen &= torch.from_numpy(where <= 0).cuda()
        ids = None
        if c["buckets"]:
            near, nb = _buckets64(c["buckets"], c["max_distance"], not c["causal"],
                                  c["max_distance"])
            n = np.minimum(np.abs(where) if not c["causal"] else np.maximum(-where, 0),
                           c["max_distance"])
            ids = near[n] + (nb * (where > 0) if not c["causal"] else 0)
            ids = torch.from_numpy(ids).cuda().reshape(-1)
        parts = {n: [] for n in ("out", "lse", "dq")}
        dk = torch.zeros((Sk, G, HEAD_DIM), dtype=torch.float64, device="cuda")
        dv = torch.zeros_like(dk)
        for h in range(H):
            kv = h * G // H
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :, kv].double(), s["v"][b, :, kv].double()
            z = (q @ k.t()) * scale
            if ids is not None:
                z = z + table[:, h][ids].reshape(Sq, Sk)
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            lse = torch.logsumexp(z, -1)
            w = torch.where(seen, torch.exp(z - lse[:, None]), torch.zeros_like(z))
            parts["out"].append(w @ v)
            parts["lse"].append(lse)
            if not step:
                continue
            do = s["dout"][b, :, h].double()
            dw = do @ v.t()
            dz = w * dw
            dz -= w * dz.sum(-1, keepdim=True)
            parts["dq"].append(dz @ k * scale)
            dk[:, kv] += dz.t() @ q * scale
            dv[:, kv] += w.t() @ do
            if ids is not None:
                dtable[:, h] += torch.bincount(ids, weights=dz.reshape(-1), minlength=c["buckets"])
        got["out"].append(torch.stack(parts["out"], 1))
        got["lse"].append(torch.stack(parts["lse"], 0))
        if step:
            got["dq"].append(torch.stack(parts["dq"], 1))
            got["dk"].append(dk)
            got["dv"].append(dv)
    got = {n: torch.stack(t) for n, t in got.items() if t}
    if step and c["buckets"]:
        got["dtable"] = dtable
    return got
