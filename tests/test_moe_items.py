"""Experts whose work-groups go from item to item, against 64 bits: more items than twice the work-groups, last rounds that are not full, parts of
K among them, items of a single stage, every width of an item.  That the shapes do this is asserted on the CPU, from the launches and the ids."""
import pytest
import torch

from paper_2607_07862_amd import binding as B
from tests._mx import NAMES
from tests._mx_gpu import assert_near, experts_and_tol, held
from tests._mx_launches import experts, program, work

BF = torch.bfloat16
ID, GELU, SWIGLU = B.ACT_IDENTITY, B.ACT_GELU_TANH, B.ACT_SWIGLU
# T, H, F, E, k, activation, weights: of either product the rows of an item, items, work-groups and parts of K
CASES = [
    (40, 2880, 3008, 24, 4, SWIGLU, "bf16", (64, 1152, 512, 2), (32, 1104, 512, 2)),
    (40, 3008, 2880, 24, 4, GELU, "bf16", (64, 1104, 512, 2), (32, 1728, 512, 3)),
    (307, 3648, 704, 52, 1, GELU, "bf16", (64, 936, 512, 3), (32, 1508, 512, 1)),
    (10, 256, 4032, 48, 6, SWIGLU, "bf16", (16, 1056, 768, 1), (16, 462, 714, 7)),
    (10, 4032, 1088, 17, 6, SWIGLU, "bf16", (64, 459, 512, 3), (32, 1088, 512, 2)),
    (68, 1344, 2560, 43, 1, ID, "bf16", (16, 640, 768, 1), (16, 704, 768, 2)),
    (20, 2112, 1344, 90, 8, SWIGLU, "bf16", (16, 1628, 768, 2), (16, 1258, 768, 1)),
    (40, 2880, 3008, 24, 4, SWIGLU, "mxfp4", (16, 1128, 512, 1), (16, 1104, 512, 2)),
    (40, 192, 4032, 24, 4, SWIGLU, "mxfp4", (16, 1512, 512, 1), (16, 384, 512, 8)),
    (10, 256, 4032, 48, 6, SWIGLU, "mxfp4", (16, 2079, 512, 1), (16, 396, 512, 6)),
    (10, 4096, 256, 48, 6, ID, "mxfp4", (16, 264, 512, 4), (16, 1056, 512, 1)),
    (150, 8256, 1088, 44, 3, SWIGLU, "mxfp4", (32, 1496, 512, 2), (16, 2860, 512, 1)),
    (30, 8256, 1088, 46, 3, SWIGLU, "mxfp4", (16, 1836, 512, 3), (16, 2340, 512, 1)),
    (200, 1088, 1088, 40, 9, SWIGLU, "mxfp4", (32, 1292, 512, 1), (16, 1071, 512, 1)),
    (300, 832, 1088, 16, 8, GELU, "mxfp4", (32, 693, 512, 1), (16, 994, 512, 1)),
    (139, 832, 3584, 47, 6, GELU, "mxfp4", (32, 1316, 512, 1), (16, 469, 512, 1)),
    (32, 2368, 2112, 27, 3, ID, "mxfp4", (16, 442, 512, 1), (16, 494, 512, 1)),
]


def names(c):
    return "x".join(str(v) for v in c[:5]) + f"-{NAMES[c[5]]}-{c[6]}"


def choice(T, E, k):
    """Different experts for each token, with every ninth slot empty."""
    gen = torch.Generator().manual_seed(T + E + k)
    ids = torch.rand((T, E), generator=gen).argsort(1)[:, :k].to(torch.int32)
    ids.view(-1)[5::9] = -1
    return ids.contiguous()


@pytest.mark.skipif(program() is None, reason="hipcc not available")
def test_work_groups_have_several_items():
    found = experts(*[(T, H, F, E, k, act, B.DTYPE_MXFP4 if w == "mxfp4" else B.DTYPE_BF16, T) for T, H, F, E, k, act, w, *_ in CASES])
    seen = set()
    for (T, H, F, E, k, act, w, *wanted), launches in zip(CASES, found):
        for second, (p, want) in enumerate(zip(launches, wanted)):
            q = work(p, choice(T, E, k).numpy(), E)
            assert (p.rows, q.items, p.groups, q.parts) == want, (T, H, F, E, k, w, second)
            assert (q.parts - 1) * q.per < p.steps <= q.parts * q.per
            if q.items > p.groups and q.items % p.groups:
                seen.add((w, second, p.rows, q.parts > 1))
                if q.items > 2 * p.groups:
                    seen.add((w, second, "two rounds", T * k <= 64))
                if q.per == 1:
                    seen.add((w, second, "single stages"))
    for w, rows in (("bf16", ((16, 64), (16, 32))), ("mxfp4", ((16, 32), (16,)))):
        for second in range(2):
            for r in rows[second]:
                assert (w, second, r, False) in seen or (w, second, r, True) in seen, (w, second, r)
            assert any((w, second, r, True) in seen for r in rows[second]), (w, second, "parts of K")
            assert (w, second, "two rounds", False) in seen
    assert ("mxfp4", 0, "single stages") in seen and ("mxfp4", 1, "single stages") in seen
    assert ("mxfp4", 0, "two rounds", True) in seen and ("bf16", 1, "two rounds", True) in seen


def weights(gen, E, H, F, act, w):
    """The experts' weights as the plan takes them, and functions expert -> fp64 ([W1 ...], W2)."""
    nb = 2 if act == SWIGLU else 1
    W1 = torch.randn((E, nb, H, F), generator=gen, device="cuda", dtype=BF) * H**-0.5
    W2 = torch.randn((E, F, H), generator=gen, device="cuda", dtype=BF) * F**-0.5
    if w == "bf16":
        return W1, W2, lambda e: ([m.double() for m in W1[e]], W2[e].double())
    a, b = B.MxMatrix(F, H, E * nb), B.MxMatrix(H, F, E)
    B.mx_quantize(W1.view(E * nb, H, F), a, down=True)
    B.mx_quantize(W2, b, down=True)
    return a, b, lambda e: ([held(a, e * nb + i).t().contiguous() for i in range(nb)], held(b, e).t().contiguous())


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,F,E,k,act,w,first,second", CASES, ids=map(names, CASES))
def test_experts(lib, T, H, F, E, k, act, w, first, second):
    gen = torch.Generator(device="cuda").manual_seed(T + H)
    W1, W2, of = weights(gen, E, H, F, act, w)
    X = torch.randn((T, H), generator=gen, device="cuda", dtype=BF)
    ids, gates = choice(T, E, k).cuda(), torch.rand((T, k), generator=gen, device="cuda") + 0.1
    Y = torch.full((T, H), float("nan"), dtype=BF, device="cuda")
    plan = B.MoePlan(T, H, F, E, k, act, BF if w == "bf16" else w)
    plan.experts(X, ids, gates, W1, W2, Y)
    ref, tol = experts_and_tol(X, ids, gates, of, E, NAMES[act])
    assert_near(Y, ref, tol, "Y")
    # the same bits again, and other inputs in the same plan
    again = torch.zeros_like(Y)
    plan.experts(X, ids, gates, W1, W2, again)
    assert torch.equal(again, Y)
    X.normal_()
    ids = ids.flip(0).contiguous()
    plan.experts(X, ids, gates, W1, W2, again)
    ref, tol = experts_and_tol(X, ids, gates, of, E, NAMES[act])
    assert_near(again, ref, tol, "Y of new inputs")


# 4-bit weights, then bf16: tokens, experts and tokens of each, so that a work-group of the second product completes more blocks of columns
# of tokens than it has room to note (2112 in 4 bits, 4224 in bf16) and adds up the others at once.
NOTED = [("mxfp4", 8191, 1, 8191, 2112), ("bf16", 8184, 248, 33, 4224)]


def many(T, E, each):
    return torch.arange(T, dtype=torch.int32).div(each, rounding_mode="floor").view(T, 1)


@pytest.mark.skipif(program() is None, reason="hipcc not available")
@pytest.mark.parametrize("w,T,E,each,room", NOTED)
def test_more_tokens_than_a_work_group_can_note(w, T, E, each, room):
    H, ids = 32768, many(T, E, each).numpy()
    p = experts((T, H, 64, E, 1, ID, B.DTYPE_MXFP4 if w == "mxfp4" else B.DTYPE_BF16, T))[0][1]
    q = work(p, ids, E)
    assert q.parts == 1 and p.blocks == 256
    # one slot to a token and whole K: who ends an item completes its rows.  Items: blocks of columns, then chunks of rows, then experts
    rows = [min(p.rows, each - first) for _ in range(E) for first in range(0, each, p.rows)]
    assert len(rows) * p.blocks == q.items
    mine = [sum(rows[n // p.blocks] for n in range(g, q.items, p.groups)) for g in range(p.groups)]
    assert max(mine) > room, max(mine)


@pytest.mark.gpu
@pytest.mark.parametrize("w,T,E,each,room", NOTED)
def test_tokens_past_the_room_to_note_them(lib, w, T, E, each, room):
    H, F = 32768, 64
    gen = torch.Generator(device="cuda").manual_seed(E)
    W1, W2, of = weights(gen, E, H, F, ID, w)
    X = torch.randn((T, H), generator=gen, device="cuda", dtype=BF)
    ids, gates = many(T, E, each).cuda(), torch.rand((T, 1), generator=gen, device="cuda") + 0.1
    Y = torch.full((T, H), float("nan"), dtype=BF, device="cuda")
    B.MoePlan(T, H, F, E, 1, ID, BF if w == "bf16" else w).experts(X, ids, gates, W1, W2, Y)
    for t0 in range(0, T, 1024):
        t = slice(t0, min(T, t0 + 1024))
        ref, tol = experts_and_tol(X[t], ids[t], gates[t], of, E, "identity")
        assert_near(Y[t], ref, tol, f"Y from token {t0} on")
