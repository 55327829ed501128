"""What the tests of the 4-bit operators share: inputs, the float64 reference, and reading the stored format."""
import numpy as np
import torch

from oracle import ctcsd_oracle as orc
from paper_2412_00061_b200 import binding

DEV = "cuda:0"
WORD_BITS = (3, 19, 7, 23, 11, 27, 31, 15)


def act_of(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def handle(dtype, B=1, H=64, V=50, T=5, k=2, nodes=2, Hq=1, Hkv=1, D=64, rows=0):
    return binding.Handle(B, H, V, T, k, 8, 4, max(2, nodes), Hq, Hkv, D, binding.DTYPE_BF16 if dtype == "bf16" else binding.DTYPE_F32,
                          max_draft_rows=rows, device=DEV)


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def stands_for(v, group, dtype):
    """v (tensor [...,n]) through the 4-bit format: float64 values, by the oracle."""
    q, s, o = orc.q4_quantize(v.float().cpu().numpy(), group)
    return torch.from_numpy(orc.q4_values(q, s, o, group, dtype == "bf16"))


def levels_of(words, n):
    """Levels [...,n] from stored bytes [...,n/2]: a word's values 0..7 at the bits of WORD_BITS (turned by a word's length)."""
    w = np.ascontiguousarray(words.cpu().numpy()).view("<u4")
    out = np.zeros(w.shape + (8,), dtype=np.int64)
    w = w.astype(np.uint64)
    for i, bit in enumerate(WORD_BITS):
        out[..., i] = ((w | (w << np.uint64(32))) >> np.uint64(bit)) & np.uint64(15)
    return out.reshape(*w.shape[:-1], -1)[..., :n]


def tree_mask(rng, B, nodes, n_live):
    W = (max(2, nodes) + 63) // 64
    m = np.zeros((B, max(2, nodes), W), dtype=np.uint64)
    for b in range(B):
        for i in range(n_live[b]):
            if i:
                m[b, i] = m[b, int(rng.integers(0, i))]
            m[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return m


def attention_reference(Q, K, V, Kt, Vt, kv_len, n_nodes, mask, scale):
    """float64: K, V the cached rows as values [B,Hkv,Lcap,D] (float64), Kt, Vt the tree's."""
    B, nodes, Hq, D = Q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    O = torch.zeros(B, nodes, Hq, D, dtype=torch.float64, device=Q.device)
    lse = torch.full((B, nodes, Hq), -np.inf, dtype=torch.float64, device=Q.device)
    for b in range(B):
        n, L = int(n_nodes[b]), int(kv_len[b])
        for i in range(n):
            seen = [j for j in range(n) if (int(mask[b, i, j // 64]) >> (j % 64)) & 1]
            if L + len(seen) == 0:
                continue
            for g in range(Hkv):
                k = torch.cat([K[b, g, :L], Kt[b, g, seen].double()])
                v = torch.cat([V[b, g, :L], Vt[b, g, seen].double()])
                x = Q[b, i, g * G:(g + 1) * G].double() @ k.t() * scale
                O[b, i, g * G:(g + 1) * G] = torch.softmax(x, -1) @ v
                lse[b, i, g * G:(g + 1) * G] = torch.logsumexp(x, -1)
    return O, lse
