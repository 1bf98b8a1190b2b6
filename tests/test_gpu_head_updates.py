"""AdamW's updates at the ends of the float range, bit for bit against the float32
form of the definition."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from paper_2307_14490_amd import binding as B  # noqa: E402
from oracle import head as ref  # noqa: E402
from gpu_common import say  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# what rounds to infinity in the type of the parameters: half a step above the largest
LARGEST = {"f32": np.float32(np.inf), "bf16": np.float32(float.fromhex("0x1.ffp127"))}


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("states", ["f32", "q8"])
@pytest.mark.parametrize("ptype", ["f32", "bf16"])
def test_updates_that_are_not_finite(ptype, states):
    """Quotients that overflow, parameters that leave the range or were not numbers: such
    elements keep parameter and moments, the others move; check() reports.  The first
    4096 elements go four at a time, the rest one by one."""
    say(f"adamw updates that are not finite, {ptype} {states}")
    rng = np.random.default_rng(41)
    f = np.float32
    size = 4096 + 700
    p, g = rng.normal(size=size).astype(f), (rng.normal(size=size) * 1e-2).astype(f)
    m, v = np.zeros(size, f), np.zeros(size, f)
    held = []
    for at in (0, 4096):
        # a large first moment over nothing: 9e35 / 1e-8 is beyond the range
        m[at + 3], g[at + 3] = 1e36, 0
        # -3.3e38 - 9e37, where the quotient is finite
        p[at + 300], m[at + 300], g[at + 300] = -3.3e38, 1e33, 0
        p[at + 520], p[at + 521], p[at + 522] = np.nan, np.inf, -np.inf
        held += [at + k for k in (3, 300, 520, 521, 522)]
    t = torch.from_numpy(p).to(TYPES[ptype]).cuda()
    opt = P.AdamW([t], lr=1e-3, weight_decay=0.0, states=states)
    opt.load([torch.from_numpy(m).cuda()], [torch.from_numpy(v).cuda()], 100_000)
    p0 = t.float().cpu().numpy()
    m0, v0 = (x[0].cpu().numpy() for x in opt.values())
    opt.step([torch.from_numpy(g).cuda()])
    pn, mn, vn, ok = ref.adamw_f32(p0, g, m0, v0, 100_001, 1e-3, 0.9, 0.999, 1e-8, 0.0,
                                   largest=LARGEST[ptype])
    assert np.flatnonzero(~ok).tolist() == held
    if states == "q8":
        mn, vn = ref.q8_f32(mn, vn)
    gm, gv = (x[0].cpu().numpy() for x in opt.values())
    np.testing.assert_array_equal(gm, mn)
    np.testing.assert_array_equal(gv, vn)
    np.testing.assert_array_equal(t.float().cpu().numpy(),
                                  torch.from_numpy(pn).to(TYPES[ptype]).float().numpy())
    with pytest.raises(P.HugeError) as e:
        opt.check()
    assert e.value.status == B.HUGE_ERR_NOT_FINITE


@pytest.mark.parametrize("size", [256, 4096])
def test_bf16_parameters_that_round_to_infinity(size):
    """A parameter of the largest bf16 moves by less than half a step, then by more: that
    is finite in 32 bits, but not in the parameter's type."""
    f = np.float32
    top = f(float.fromhex("0x1.fep127"))
    move = f(float.fromhex("0x1p119"))  # half a step
    p = torch.full((size,), float(top)).bfloat16().cuda()
    opt = P.AdamW([p], lr=1.0, betas=(0.0, 0.0), eps=1e-5, weight_decay=0.0)
    # with both betas 0 the update is lr g / (|g| + eps)
    g = np.zeros(size, f)
    g[:3] = -1.0
    z = torch.zeros(size, device="cuda")
    opt.load([z], [z], 5)
    for lr, moves in ((0.9 * float(move), True), (1.01 * float(move), False)):
        was = p.clone()
        opt.step([torch.from_numpy(g).cuda()], lr=lr)
        assert torch.equal(p, was) and p.isfinite().all()
        if moves:
            opt.check()
        else:
            with pytest.raises(P.HugeError):
                opt.check()
