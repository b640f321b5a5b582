"""CPU oracle for decode steps over drafted tokens, running attention weights and evicted contexts.  TEST INFRASTRUCTURE ONLY.

A node of a drafted tree is defined by the path to it: its output is what the last of those tokens gives when they are
decoded one after the other (oracle/decode.py's step, with the context kept per KV head so that slots can be taken out
of it; tests/test_oracle_decode_tree.py pins the two to each other).  Float64; the one rounding is K/V -> bf16.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Sequence, Tuple

import numpy as np

from oracle.cache_ops import select_slots
from oracle.reuse_prefill import Model, PromptResult, rmsnorm, rope, round_to_bf16, silu


@dataclass
class State:
    k: List[np.ndarray]          # per layer: rotated keys [slots, Hkv, hd]
    v: List[np.ndarray]
    w: List[np.ndarray]          # per layer: running weights [Hkv, slots]
    position: int                # of the next token (slots may be fewer)
    score_abs: float = 0.0       # largest sum |q k| / sqrt(hd) met: what rounding errors of a score scale with

    def copy(self) -> "State":
        return State([x.copy() for x in self.k], [x.copy() for x in self.v], [x.copy() for x in self.w], self.position, self.score_abs)


def begin(result: PromptResult) -> State:
    k = [np.array(x) for x in result.k_ctx]
    return State(k, [np.array(x) for x in result.v_ctx], [np.zeros((x.shape[1], x.shape[0])) for x in k], k[0].shape[0])


def step(model: Model, st: State, hidden: np.ndarray) -> Tuple[np.ndarray, List[np.ndarray]]:
    """One token at st.position.  Returns its final residual and, per layer, its softmax weights [Hkv, slots + 1] summed over the
    query heads of each KV head.  K and V join the context; the running weights get a zero for the new slot."""
    hq, hkv, hd = model.n_q_heads, model.n_kv_heads, model.head_dim
    pos = np.array([st.position])
    x = np.array(hidden, dtype=np.float64).reshape(1, model.d_model)
    got = []
    for l in range(model.n_layers):
        xn = rmsnorm(x, model.w(l, "attn_norm"), model.rms_eps)
        q = rope((xn @ model.w(l, "wq").T).reshape(1, hq, hd), pos, model.rope_theta)[0]
        k = rope(round_to_bf16((xn @ model.w(l, "wk").T).reshape(1, hkv, hd)), pos, model.rope_theta)
        v = round_to_bf16((xn @ model.w(l, "wv").T).reshape(1, hkv, hd))
        st.k[l] = np.concatenate([st.k[l], k], axis=0)
        st.v[l] = np.concatenate([st.v[l], v], axis=0)
        st.w[l] = np.concatenate([st.w[l], np.zeros((hkv, 1))], axis=1)
        att = np.zeros((hq, hd))
        share = np.zeros((hkv, st.k[l].shape[0]))
        for h in range(hq):
            g = h // (hq // hkv)
            s = st.k[l][:, g] @ q[h] / np.sqrt(hd)
            st.score_abs = max(st.score_abs, float((np.abs(st.k[l][:, g]) @ np.abs(q[h])).max() / np.sqrt(hd)))
            p = np.exp(s - s.max())
            p /= p.sum()
            att[h] = p @ st.v[l][:, g]
            share[g] += p
        got.append(share)
        x = x + att.reshape(1, -1) @ model.w(l, "wo").T
        yn = rmsnorm(x, model.w(l, "ffn_norm"), model.rms_eps)
        x = x + (silu(yn @ model.w(l, "w_gate").T) * (yn @ model.w(l, "w_up").T)) @ model.w(l, "w_down").T
    st.position += 1
    return x[0], got


def path_to(parents: Sequence[int], node: int) -> List[int]:
    path = []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


def tree_outputs(model: Model, st: State, parents: Sequence[int], hidden: np.ndarray) -> np.ndarray:
    """Final residual of every node: hidden [n, d]."""
    out = []
    for i in range(len(parents)):
        s = st.copy()
        for j in path_to(parents, i):
            y, _ = step(model, s, hidden[j])
        out.append(y)
    return np.stack(out)


def accept(model: Model, st: State, hidden: np.ndarray, path: Sequence[int], track: bool, decay: float) -> None:
    """The path's tokens join the context; tracked: the running weights decay once and get the path's weights."""
    shares = [step(model, st, hidden[j])[1] for j in path]
    if track and path:
        for l in range(model.n_layers):
            st.w[l] *= decay
            for s in shares:
                st.w[l][:, :s[l].shape[1]] += s[l]


def evict(st: State, budget: int, sink: int, recent: int, weights: List[np.ndarray]) -> None:
    """Keep at most `budget` slots per layer and head, chosen by `weights` (fp32, per layer [Hkv, slots])."""
    for l in range(len(st.k)):
        n = st.k[l].shape[0]
        keep = [select_slots(weights[l][g].astype(np.float32), n, budget, sink, recent) for g in range(st.k[l].shape[1])]
        st.k[l] = np.stack([st.k[l][keep[g], g] for g in range(len(keep))], axis=1)
        st.v[l] = np.stack([st.v[l][keep[g], g] for g in range(len(keep))], axis=1)
        st.w[l] = np.stack([st.w[l][g, keep[g]] for g in range(len(keep))])
