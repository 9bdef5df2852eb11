"""How far the weights of tree attention may be off, form by form: 4 to 256 rows (nodes times query heads of a KV head), which one, two, four and eight
waves share.  Scores here are a_h * c_t: queries have a_h in their first column, keys c_t, all else is zero, and the scale is ln 2, so that a token's weight
is 2^(a_h c_t)."""
import math

import numpy as np
import pytest
import torch

import tree_reference as ref
from paper_2508_07101_amd import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"
# (sequences, query heads, KV heads, nodes): rows of one KV head's group, and enough workgroups for the form of 256 rows
FORMS = [(1, 8, 2, 1), (2, 8, 2, 8), (2, 8, 2, 16), (2, 8, 2, 32), (20, 64, 16, 64)]


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _tokens(B, H, G, nodes, a, c, v):
    """Tree attention of B equal sequences of scalar keys c [tokens] and values v [tokens, 128], the last `nodes` of them drafted in a chain."""
    k = torch.zeros((B, G, len(c), 128), dtype=torch.bfloat16, device=DEV)
    k[..., 0] = torch.as_tensor(c, dtype=torch.float32).to(device=DEV, dtype=torch.bfloat16)
    vv = v.to(device=DEV, dtype=torch.bfloat16).expand(B, G, len(c), 128).contiguous()
    q = torch.zeros((B * nodes, H, 128), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = torch.as_tensor(a, dtype=torch.float32).to(device=DEV, dtype=torch.bfloat16)
    words = cb.mask_words(nodes)
    bits = ref.masks([j - 1 for j in range(nodes)], words)[0]
    tree = cb.Tree(_i32(np.arange(B + 1) * nodes), torch.from_numpy(np.tile(bits, (B, 1)).view(np.int64)).to(DEV), nodes)
    params = cb.make_params(B, H, G, 1, 0, sm_scale=math.log(2.0))
    out = torch.full((B * nodes, H, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = cb.alloc_tree_workspace(params, len(c), B * nodes, nodes)
    print("weights", B, H, G, nodes, len(c), flush=True)
    cb.tree_attn(params, q, cb.KvCache(k, vv, _i32([len(c)] * B), len(c)), tree, out, ws)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("B,H,G,nodes", FORMS)
def test_a_mean_of_equal_values_is_that_value(B, H, G, nodes):
    """Every token has the same value, so every mean is that value, whatever the weights: they are rounded alike above and below the line.  A weight that
    is rounded above only is off by up to 2^-8, and the values' next neighbours in bf16 are 2^-8 away (2^-9 to the border): one token outweighs the others,
    at a weight that is no power of two.  It stands behind the first tiles of 32 of all teams of waves that share the tokens, since a row's reference is taken from there."""
    teams = min(8, 64 // nodes)
    c = torch.full((32 * teams + 32 + nodes,), -16.0)
    c[0: 32 * teams: 32] = 0.0
    c[32 * teams + 16] = 1.0
    a = 3.0 + 4.5 * torch.rand((B * nodes, H), generator=torch.Generator().manual_seed(nodes))
    value = 1.9921875 * 2.0 ** torch.arange(-4, 4).repeat(16) * torch.tensor([1.0, -1.0]).repeat(64)
    out = _tokens(B, H, G, nodes, a, c, value.expand(len(c), 128))
    assert torch.equal(out.float().cpu(), value.expand_as(out))


@pytest.mark.parametrize("nodes", [1, 8, 16])
def test_few_rows_have_weights_of_fifteen_bits(nodes):
    """Up to 64 rows: a weight is off by 2^-15 of itself, and 2^-17 more by its exponent (128 products added in 32 bits: 2^-17 of the sum of their sizes, about
    10 here), above the line and below: 2^-12 of the weighted mean of sizes at most.  The output's own rounding is 2^-8 of it.  A few tokens weigh more
    than all others."""
    rng = np.random.default_rng(nodes)
    H, G, n = 8, 2, 700
    gen = torch.Generator(device=DEV)
    gen.manual_seed(nodes)
    k, v = (torch.randn((1, G, n, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((nodes, H, 128), generator=gen, device=DEV).to(torch.bfloat16)
    for t in rng.integers(0, n - nodes, size=6).tolist():
        k[0, :, t] = (q[0].float().view(G, -1, 128).sum(1) * 0.4).to(torch.bfloat16)
    bits = ref.masks([j - 1 for j in range(nodes)], 1)[0]
    tree = cb.Tree(_i32([0, nodes]), torch.from_numpy(bits.view(np.int64).copy()).to(DEV), nodes)
    params = cb.make_params(1, H, G, 1, 0)
    out = torch.empty((nodes, H, 128), dtype=torch.bfloat16, device=DEV)
    cb.tree_attn(params, q, cb.KvCache(k, v, _i32([n]), n), tree, out, cb.alloc_tree_workspace(params, n, nodes, nodes))
    torch.cuda.synchronize()
    want, mass = ref.attention(q, k[0].double(), v[0].double(), n - nodes, nodes, ref.allowed(bits, nodes), 128 ** -0.5)
    err, tol = (out.double() - want).abs(), 2.0 ** -12 * mass + 2.0 ** -8 * want.abs()
    assert (err <= tol).all(), f"{int((err > tol).sum())} of {err.numel()}, worst {float((err / tol).max()):.3g} of the bound"


@pytest.mark.parametrize("below", [126, 127, 130, 132])
@pytest.mark.parametrize("B,H,G,nodes", FORMS)
def test_weights_below_the_normal_range_count(B, H, G, nodes, below):
    """One token has all the weight and the value 0, another a weight of 2^-below beside it and the value 2^120: the whole output.  In the first one's
    tile, in a later one of the same team, in another team's, and (1100 tokens) in another piece."""
    for n, heavy, light in ((40 + nodes, 3, 30), (300 + nodes, 3, 270), (300 + nodes, 3, 40), (300 + nodes, 270, 3), (1100 + nodes, 3, 1090), (1100 + nodes, 900, 3)):
        c = torch.full((n,), -200.0)
        c[heavy], c[light] = 0.0, -float(below)
        v = torch.zeros((n, 128))
        v[light] = 2.0 ** 120
        out = _tokens(B, H, G, nodes, torch.ones((B * nodes, H)), c, v)
        assert (out.float() == 2.0 ** (120 - below)).all(), (n, heavy, light, out.float().amin().item(), out.float().amax().item())


@pytest.mark.parametrize("before", [40, 300, 1100, 5000])
@pytest.mark.parametrize("B,H,G,nodes", FORMS)
def test_infinite_values_of_nodes_whatever_their_piece_weighs(B, H, G, nodes, before):
    """A token of the prefix outweighs the nodes by 2^200, more than 32 bits hold: an infinite value of the last node is the output of the last node all the
    same, in one piece (up to 300 tokens) as in several, and reaches no other node."""
    c = torch.full((before + nodes,), -200.0)
    c[3] = 0.0
    v = torch.ones((len(c), 128))
    v[-1, 5:90:3], v[-1, 6:90:3] = float("inf"), -float("inf")
    out = _tokens(B, H, G, nodes, torch.ones((B * nodes, H)), c, v).float().view(B, nodes, H, 128)
    want = torch.ones((nodes, 128), device=DEV)
    want[-1] = torch.where(v[-1].isinf(), v[-1], torch.ones(128)).to(DEV)
    assert torch.equal(out, want[None, :, None].expand_as(out))
