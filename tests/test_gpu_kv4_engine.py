"""KOALA_F_KV4: the target's keys and values in the paged 4-bit cache, call by call against the oracle.

A key that differs in its last bits may fall on the other side of a code's boundary, so the oracle goes on from what the cache holds: every
key and value that it computes is compared with the cache's number - half a step of the vector's scale, on top of what the bf16 paths are
compared with - and replaced by it.  Hidden states, logits and tokens then follow from the same numbers on both sides."""
import numpy as np
import pytest
import torch

from oracle.koala_oracle import KoalaOracle, round_to_bf16
from paper_2408_08146_b200 import KOALA_F_KV4, Koala, KoalaError, PagedKV4
from tests.harness import static_tree_for, tok_list
from tests.helpers import HostWeights
from tests.kv4_reference import tree_masks
from tests.parity import TOL, assert_close, check_argmax
from workloads import T13_EAGLE, T7_EAGLE, T7_MEDUSA, TINY_EAGLE, reduced
from workloads.generate import WeightStore

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Pair:
    def __init__(self, cfg, page, flags=0, seed=0):
        self.cfg, self.rng = cfg, np.random.default_rng(seed)
        per = -(-cfg.S_max // page)
        self.cache = PagedKV4(cfg.L, cfg.n_heads, cfg.head_dim, page, cfg.B * per + 3, device=DEV)
        self.cache.pages.fill_(0xFF)
        order = self.rng.permutation(cfg.B * per + 3)[:cfg.B * per].reshape(cfg.B, per)
        self.table = torch.tensor(order, dtype=torch.int32, device=DEV)
        torch.cuda.synchronize()
        store, st = WeightStore(cfg, DEV), static_tree_for(cfg)
        self.eng = Koala(cfg, store.tensors, static_tree=st, flags=flags, kv4=(self.cache, self.table))
        self.orc = KoalaOracle(cfg, HostWeights(store, np.float32), dtype=np.float32, static_tree=st, kv_round=self.kv_round)
        self.now, self.plain = None, self.orc.target_forward
        self.orc.target_forward = self.target_forward

    def held(self, b, first, n):
        """fp32 [layers][n][heads][head_dim], keys and values."""
        torch.cuda.synchronize()
        one = lambda v: torch.tensor([v], dtype=torch.int32, device=DEV)
        k, v = self.cache.read(self.cache.rows(self.table[b:b + 1].contiguous(), one(first), max_rows=n), dtype=torch.float32)
        return k.cpu().numpy(), v.cpu().numpy()

    def target_forward(self, b, tok, parent):
        self.now = [self.held(b, self.orc.seq_len[b], len(tok)), 0]
        out = self.plain(b, tok, parent)
        assert self.now[1] == 2 * self.cfg.L
        self.now = None
        return out

    def kv_round(self, x):
        if self.now is None:
            return round_to_bf16(x)                      # the head's own cache
        layer, which = divmod(self.now[1], 2)
        self.now[1] += 1
        got = self.now[0][which][layer]
        atol, rtol = TOL[1]
        slack = np.maximum(atol, rtol * np.abs(x))
        # a step: the range over 15, each end moved by the slack, the lower one and the step rounded outwards to bf16
        ends = np.abs(x).max(-1, keepdims=True)
        step = (x.max(-1, keepdims=True) - x.min(-1, keepdims=True) + 2 * slack.max(-1, keepdims=True) + 2.0 ** -7 * ends) / 15 * (1 + 2.0 ** -7)
        assert np.isfinite(got).all()
        worst = (np.abs(got - x) / (step / 2 + slack)).max()
        assert worst <= 1.0, f"layer {layer} {'value' if which else 'key'}: {worst:.3g} of the bound"
        return got

    def verify(self, trees):
        cfg, eng, orc = self.cfg, self.eng, self.orc
        n_max = max(len(t) for t, _ in trees)
        pad = lambda i: torch.tensor(np.stack([np.pad(t[i], (0, n_max - len(t[i]))) for t in trees]).astype(np.int32), device=DEV)
        eng.koala_verify((pad(0), pad(1), torch.tensor([len(t) for t, _ in trees], dtype=torch.int32, device=DEV), n_max))
        orc.verify(trees)
        bufs = eng.buffers()
        tgt = bufs["verify_tgt"].cpu().numpy()
        for b, (t, _) in enumerate(trees):
            rows = slice(b * cfg.N, b * cfg.N + len(t))
            assert_close(bufs["verify_hid"][rows].cpu().numpy(), orc.verify_hid[b], 1, f"hidden states of {b}")
            assert_close(bufs["verify_logits"][rows].cpu().numpy(), orc.verify_logits[b], 1, f"logits of {b}")
            check_argmax(tgt[rows], orc.verify_logits[b], f"tokens of {b}")
            tgt[rows] = orc.verify_tgt[b]
        bufs["verify_tgt"].copy_(torch.from_numpy(tgt))

    def accept(self, forced):
        S = list(self.orc.seq_len)
        got = tok_list(*self.eng.koala_accept(torch.tensor(forced, dtype=torch.int32, device=DEV)))
        tokens, lens = self.orc.accept(forced)
        assert [list(map(int, x)) for x in tokens] == got[0] and list(lens) == got[1]
        assert self.eng.seq_len.cpu().tolist() == self.orc.seq_len
        for b, n in enumerate(got[1]):
            k, v = self.held(b, 0, S[b] + n)
            for l in range(self.cfg.L):                  # the oracle holds the cache's own numbers: bit for bit, what lay before too
                assert np.array_equal(k[l], self.orc.target_k[l][b][:S[b] + n]) and np.array_equal(v[l], self.orc.target_v[l][b][:S[b] + n])

    def tree(self, n):
        sees, _ = tree_masks(n, self.rng)
        parent = [-1] + [int(np.flatnonzero(sees[u, :u])[-1]) for u in range(1, n)]
        return self.rng.integers(0, self.cfg.V, n), np.array(parent)

    def finish(self):
        assert self.eng.device_status() == 0
        assert self.eng.check_guards()[1] == 0
        self.eng.close()


CASES = {
    "medusa": (reduced(T7_MEDUSA, 2, S_max=256), [90], 16, 64, 0),
    "eagle_batch2": (reduced(T7_EAGLE, 2, K=1, B=2, S_max=320), [130, 61], 64, 60, 0),
    "narrow_heads": (reduced(T7_EAGLE, 2, K=1, n_heads=64, head_dim=64, S_max=256), [70], 32, 60, 0),
    "batch4_ragged": (reduced(T13_EAGLE, 1, K=1, S_max=384), [200, 17, 64, 150], 128, 64, 0),
    "whole_trees_of_128": (reduced(T7_EAGLE, 1, K=1, N=128, S_max=384), [140], 32, 128, 0),
    "few_rows": (reduced(T7_EAGLE, 2, K=1, B=2, N=4, D=3, topk=1, S_max=192), [21, 9], 16, 4, 0),
    "cuda_cores": (reduced(T7_EAGLE, 1, K=1, S_max=192), [40], 16, 33, 1),
    "layer_kernel_flag": (reduced(T7_EAGLE, 2, K=1, S_max=192), [40], 16, 60, 4),
}


@pytest.mark.parametrize("name", CASES)
def test_prompt_trees_and_acceptance(name):
    cfg, lens, page, n, flags = CASES[name]
    p = Pair(cfg.with_(prompt_len=max(lens)), page, flags, seed=len(name))
    prompts = [p.rng.integers(0, cfg.V, m) for m in lens]
    p.eng.prefill(prompts, cfg.N)
    p.orc.prefill(prompts, cfg.N)
    assert p.eng.seq_len.cpu().tolist() == lens
    for b in range(cfg.B):                               # hand over: the last chunk's tokens may differ by a near tie
        p.eng.buffers()["root_tok"][b] = p.orc.root_tok[b]
    for step in range(3):
        # a whole tree, one with a node less for every other sequence, a single node each
        sizes = [max(1, n - b % 2) if step < 2 else 1 for b in range(cfg.B)]
        trees = [p.tree(m) for m in sizes]
        for (tok, _), root in zip(trees, p.orc.root_tok):
            tok[0] = root
        p.verify(trees)
        p.accept([1 + (3 * b + 2 * step + 1) % 5 for b in range(cfg.B)])
    p.finish()


def test_iterations_do_not_depend_on_the_pages():
    """Free-running iterations over pages of 16 and of 128 slots, and once more: the same tokens, the same numbers in the cache."""
    cfg = reduced(T7_MEDUSA, 2, S_max=256, prompt_len=50)
    prompt = [np.random.default_rng(3).integers(0, cfg.V, 50)]
    forced = torch.tensor([2], dtype=torch.int32, device=DEV)
    seen = []
    for page in (16, 128, 16):
        p = Pair(cfg, page, seed=page)
        p.eng.prefill(prompt, cfg.N)
        toks = [tok_list(*p.eng.step(forced)) for _ in range(4)]
        S = int(p.eng.seq_len[0])
        seen.append((toks, S, p.held(0, 0, S)))
        p.finish()
    assert seen[0][1] >= 58
    for other in seen[1:]:
        assert other[:2] == seen[0][:2]
        for a, b in zip(seen[0][2], other[2]):
            assert np.array_equal(a, b)


def test_moved_pages_and_a_new_table():
    """koala_set_kv4 again, between two steps: the same numbers from pages in another order."""
    cfg = reduced(T7_MEDUSA, 1, S_max=192, prompt_len=40)
    p = Pair(cfg, 16, seed=9)
    prompt = [p.rng.integers(0, cfg.V, 40)]
    p.eng.prefill(prompt, cfg.N)
    p.orc.prefill(prompt, cfg.N)
    n = p.cache.n_pages
    pages = p.cache.pages.view(cfg.L, n, -1)
    order = torch.randperm(n, device=DEV)
    moved = PagedKV4(cfg.L, cfg.n_heads, cfg.head_dim, 16, n, device=DEV)
    moved.pages.view(cfg.L, n, -1)[:, order] = pages
    table = order[p.table.long()].to(torch.int32).contiguous()
    torch.cuda.synchronize()
    p.cache.pages.fill_(0xFF)
    p.cache, p.table = moved, table
    p.eng.set_kv4(moved, table)
    tok, parent = p.tree(30)
    tok[0] = p.orc.root_tok[0]
    p.verify([(tok, parent)])
    with pytest.raises(KoalaError):                      # the tree lies in these pages
        p.eng.set_kv4(moved, table)
    p.accept([3])
    p.eng.set_kv4(moved, table)
    p.finish()


def test_refusals():
    cfg = reduced(T7_EAGLE, 1, K=1, V=256, S_max=128, prompt_len=16)
    store = WeightStore(cfg, DEV)
    cache = PagedKV4(1, cfg.n_heads, cfg.head_dim, 16, 16, device=DEV)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(1, 8)
    eng = Koala(cfg, store.tensors)
    with pytest.raises(KoalaError):                      # a context without the flag
        eng.set_kv4(cache, table)
    eng.close()
    for wrong in (PagedKV4(2, cfg.n_heads, cfg.head_dim, 16, 16, device=DEV), PagedKV4(1, cfg.n_heads - 1, cfg.head_dim, 16, 16, device=DEV),
                  PagedKV4(1, cfg.n_heads, 64, 16, 16, device=DEV)):
        with pytest.raises(KoalaError):
            Koala(cfg, store.tensors, kv4=(wrong, table))
    with pytest.raises(KoalaError):                      # 112 of 128 slots
        Koala(cfg, store.tensors, kv4=(cache, table[:, :7].contiguous()))
    with pytest.raises(ValueError):
        Koala(cfg, store.tensors, kv4=(cache, table.long()))
    with pytest.raises(KoalaError):                      # fp32
        Koala(TINY_EAGLE, WeightStore(TINY_EAGLE, DEV).tensors, flags=KOALA_F_KV4)
    eng = Koala(cfg, store.tensors, flags=KOALA_F_KV4)   # no cache yet
    one = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    with pytest.raises(KoalaError):
        eng.koala_verify((one, one - 1, one[0] + 1, 1))
    with pytest.raises(KoalaError):
        eng.prefill([[1, 2, 3]], 8)
    eng.set_kv4(cache, table)
    eng.prefill([[1, 2, 3]], 8)
    assert eng.device_status() == 0
    eng.close()


def test_a_slot_without_a_page_is_reported():
    cfg = reduced(T7_EAGLE, 1, K=1, V=256, S_max=128, prompt_len=16)
    cache = PagedKV4(1, cfg.n_heads, cfg.head_dim, 16, 16, device=DEV)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(1, 8)
    table[0, 1] = -1
    eng = Koala(cfg, WeightStore(cfg, DEV).tensors, kv4=(cache, table))
    with pytest.raises(KoalaError):
        eng.prefill([np.arange(20)], 60)
        if eng.device_status() != 0:
            raise KoalaError(eng.device_status(), "reported")
    eng.close()


def test_a_tree_that_does_not_fit_moves_nothing():
    """100 + 60 nodes in 128 slots: reported, and no page changes, whatever the table says about slots that are not reached."""
    cfg = reduced(T7_EAGLE, 1, K=1, V=256, S_max=128, prompt_len=16)
    cache = PagedKV4(1, cfg.n_heads, cfg.head_dim, 16, 16, device=DEV)
    cache.pages.zero_()
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(1, 8)
    table[0, 7] = 0                                      # slots 112 .. : the first page once more
    eng = Koala(cfg, WeightStore(cfg, DEV).tensors, kv4=(cache, table))
    eng.prefill([np.arange(100)], 60)
    assert eng.device_status() == 0
    before = cache.pages.clone()
    tok = torch.zeros(1, 60, dtype=torch.int32, device=DEV)
    parent = torch.zeros(1, 60, dtype=torch.int32, device=DEV)
    parent[0, 0], parent[0, 20], parent[0, 21:] = -1, 1, torch.arange(20, 59, device=DEV)      # the walk: 0, 1, 20, 21, which would lie at slots 100 ..
    n = torch.full((1,), 60, dtype=torch.int32, device=DEV)
    eng.koala_verify((tok, parent, n, 60))
    eng.koala_accept(torch.tensor([4], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(cache.pages, before)
    assert eng.device_status() == 3                      # KOALA_E_CAPACITY
    eng.close()
