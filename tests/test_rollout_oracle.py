"""Pins of the rollout oracle, and the host entry point rlk_tree_ends against it (no GPU)."""
import numpy as np
import pytest

import paper_2608_16798_amd as rlk
from oracle import rollout as RO

from test_tree_pack import random_calls


def packed(seed, rollouts=5):
    rng = np.random.default_rng(seed)
    return rlk.tree_pack([random_calls(rng, n_calls=int(rng.integers(1, 9))) for _ in range(rollouts)])


@pytest.mark.parametrize("seed", range(6))
def test_tree_ends_of_packed_calls(seed):
    t = packed(seed)
    end = rlk.tree_ends(t["pos_off"], t["parent"])
    np.testing.assert_array_equal(end, RO.tree_ends(t["pos_off"], t["parent"]))
    # j <= i < end[j] is "j on the root path of i"
    for o, e in zip(t["pos_off"][:-1], t["pos_off"][1:]):
        for i in range(o, e):
            path, j = set(), i
            while j >= 0:
                path.add(j)
                j = t["parent"][j]
            assert path == {j for j in range(o, i + 1) if i - o < end[j]}
            assert t["depth"][i] == len(path) - 1


def test_tree_ends_sizes_and_refusals():
    assert rlk.tree_ends([0], []).size == 0
    np.testing.assert_array_equal(rlk.tree_ends([0, 0, 1], [-1]), [1])
    np.testing.assert_array_equal(rlk.tree_ends([0, 3], [-1, -1, -1]), [1, 2, 3])        # three trees of one position
    np.testing.assert_array_equal(rlk.tree_ends([0, 4], [-1, 0, 0, 2]), [4, 2, 4, 4])
    np.testing.assert_array_equal(rlk.tree_ends([0, 2, 4], [-1, 0, -1, 2]), [2, 2, 2, 2])  # counted per rollout
    for off, par in (([0, 2], [-1, 1]), ([0, 2], [-1, 5]), ([0, 2], [-2, 0]), ([0, 1, 3], [-1, 0, 1]),
                     ([0, 4], [-1, 0, 0, 1]), ([1, 2], [-1, 0]), ([0, 2, 1, 2], [-1, 0])):
        with pytest.raises(rlk.RlkError) as e:
            rlk.tree_ends(off, par)
        assert e.value.code == rlk.RLK_EINVAL, (off, par)
    with pytest.raises(ValueError, match="parent has"):
        rlk.tree_ends([0, 3], [-1, 0])
    lib = rlk.load_library()
    assert lib.rlk_tree_ends(-1, None, None, None) == rlk.RLK_ESHAPE
    assert lib.rlk_tree_ends(0, None, None, None) == rlk.RLK_OK
    assert lib.rlk_tree_ends(1, None, None, None) == rlk.RLK_EINVAL


def paged(rng, lens, K, ps, D, extra=3):
    """Dense [len, K, D] keys and values of each sequence, and the pools that hold them."""
    used = [-(-n // ps) for n in lens]
    pages = rng.permutation(sum(used) + extra)
    table = np.zeros((len(lens), max(1, max(used))), np.int64)
    kp, vp = (rng.standard_normal((sum(used) + extra, K, ps, D)) for _ in range(2))
    dense, at = [], 0
    for b, n in enumerate(lens):
        table[b, :used[b]] = pages[at:at + used[b]]
        at += used[b]
        j = np.arange(n)
        dense.append((kp[table[b, j // ps], :, j % ps], vp[table[b, j // ps], :, j % ps]))
    return kp, vp, table, dense


def test_attention_of_a_tree_is_that_of_its_paths():
    """Along a root path the tree's attention is plain causal attention over the path's own keys."""
    rng = np.random.default_rng(3)
    t = packed(1, 2)
    lens = np.diff(t["pos_off"])
    kp, vp, table, dense = paged(rng, lens, 2, 4, 8)
    ends = np.zeros((2, lens.max()), np.int64)
    e = rlk.tree_ends(t["pos_off"], t["parent"])
    for b in range(2):
        ends[b, :lens[b]] = e[t["pos_off"][b]:t["pos_off"][b + 1]]
    q = rng.standard_normal((lens.sum(), 4, 8))
    got = RO.kv_attention(q, kp, vp, table, lens, t["pos_off"], 0.3, ends)["out"]
    for i in range(lens.sum()):
        b = int(i >= t["pos_off"][1])
        path, j = [], i
        while j >= 0:
            path.append(j - t["pos_off"][b])
            j = t["parent"][j]
        k, v = dense[b][0][path[::-1]], dense[b][1][path[::-1]]
        for h in range(4):
            x = np.exp(0.3 * k[:, h // 2] @ q[i, h])
            np.testing.assert_allclose(got[i, h], x @ v[:, h // 2] / x.sum(), rtol=1e-12, atol=1e-14)


def test_append_then_read_back():
    """Rotations by positions p and p' leave q . k a function of p - p'; norms leave the mean square at 1."""
    rng = np.random.default_rng(4)
    T, H, D, ps = 9, 2, 16, 4
    freq = 10.0 ** -np.arange(8)
    q, k, v = (rng.standard_normal((T, H, D)) for _ in range(3))
    z = np.zeros((3, H, ps, D))
    args = dict(page_table=np.array([[2, 0, 1]]), kv_len=np.array([T]), cu_new=np.array([0, T]), freq=freq)
    for style in ("half", "pairs"):
        a = RO.kv_append(z, z, q=q, k=k, v=v, rot_style=style, **args)
        b = RO.kv_append(z, z, q=q, k=k, v=v, rot_style=style, positions=np.arange(T) + 77, **args)
        j = np.arange(T)
        pages = args["page_table"][0, j // ps]
        ka, kb = a["k_pages"][pages, :, j % ps], b["k_pages"][pages, :, j % ps]
        for s in range(T):
            np.testing.assert_allclose(np.einsum("hd,thd->th", a["q"][s], ka), np.einsum("hd,thd->th", b["q"][s], kb), atol=1e-12)
        np.testing.assert_array_equal(a["v_pages"][pages, :, j % ps], v)
        np.testing.assert_allclose((a["q"] ** 2).sum(-1), (q ** 2).sum(-1))
    n = RO.kv_append(z, z, q=q, k=k, v=v, q_norm=np.full(D, 2.0), norm_eps=0.0, **args)
    np.testing.assert_allclose((n["q"] ** 2).mean(-1), 4.0)


@pytest.mark.parametrize("dist", [True, False])
def test_verified_tokens_follow_the_target(dist):
    """Drafts drawn from q and verified against p: the first token's distribution is p (drafts without
    probabilities: for every draft).  A grid of both random numbers in place of chance."""
    rng = np.random.default_rng(5)
    V, G = 6, 400
    z, zq = rng.standard_normal((2, V)), rng.standard_normal((1, V))
    p = np.exp(RO._log_softmax(z[0], 0.7))
    q = np.exp(RO._log_softmax(zq[0], 0.7))
    seen = np.zeros(V)
    grid = (np.arange(G) + 0.5) / G
    for y in range(V):
        for ua in grid[::8]:
            for us in grid[::8]:
                r = RO.draft_verify(z, np.array([y]), np.array([0, 1]), np.array([ua]), np.array([us]),
                                    zq if dist else None, 0.7)
                seen[r["tokens"][0]] += q[y] if dist else 1.0 / V
                assert r["tokens"][1] == -1 or r["n_accepted"][0] == 1
                np.testing.assert_allclose(r["logp"][0], np.log(p[r["tokens"][0]]), rtol=1e-12)
    seen /= seen.sum()
    np.testing.assert_allclose(seen, p, atol=0.03)  # a grid of 50 per random number: steps of 0.02
