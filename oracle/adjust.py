"""Oracle of the confidences of adjusted logits: penalties, biases and masks as defined, in the fp32 operations of the
definition, then softmax and candidates in fp64."""

import numpy as np

F32 = np.float32


def adjust_logits(logits, rows_per_seq, history=None, history_len=None, repetition=None, frequency=None, presence=None,
                  bias_ids=None, bias=None, mask=None, mask_index=None):
    """x [rows, vocab] float32; forbidden tokens -inf.  mask [n, words] uint32."""
    R, V = logits.shape
    x = np.array(logits, dtype=F32)
    for r in range(R):
        q = r // rows_per_seq
        count, add = {}, {}
        if history is not None:
            H = history.shape[1]
            n = H if history_len is None else min(max(int(history_len[q]), 0), H)
            for v in history[q, :n].tolist():
                if 0 <= v < V:
                    count[v] = count.get(v, 0) + 1
        if bias is not None:
            for v, y in zip(bias_ids[q].tolist(), bias[q]):
                if 0 <= v < V:
                    add[v] = F32(add[v] + y) if v in add else F32(y)
        rep = F32(1 if repetition is None else repetition[q])
        f = F32(0 if frequency is None else frequency[q])
        p = F32(0 if presence is None else presence[q])
        for v in set(count) | set(add):
            y, c, a = x[r, v], count.get(v, 0), add.get(v, F32(0))
            if c > 0:
                with np.errstate(over="ignore"):
                    y = F32(y / rep) if y > 0 else F32(y * rep)
                a = F32(a - F32(F32(f * F32(c)) + p))
            with np.errstate(invalid="ignore"):
                x[r, v] = F32(y + a)
        if mask is not None:
            m = r if mask_index is None else int(mask_index[r])
            if 0 <= m < mask.shape[0]:
                v = np.arange(V)
                x[r, (mask[m, v // 32] >> (v % 32).astype(np.uint32)) & 1 == 0] = -np.inf
            elif m != -1:
                x[r] = -np.inf
    return x


def confidence_topk_adjusted(logits, k, rows_per_seq, **how):
    """(conf [rows, k] float64, idx [rows, k] int32); slots without an allowed token: 0 and -1."""
    x = adjust_logits(logits, rows_per_seq, **how).astype(np.float64)
    conf = np.zeros((x.shape[0], k))
    idx = np.full((x.shape[0], k), -1, np.int32)
    for r, row in enumerate(x):
        if not (row > -np.inf).any():
            continue
        w = np.exp(row - row.max())
        order = np.argsort(-row, kind="stable")[:k]
        order = order[row[order] > -np.inf]
        idx[r, :len(order)] = order
        conf[r, :len(order)] = w[order] / w.sum()
    return conf, idx
