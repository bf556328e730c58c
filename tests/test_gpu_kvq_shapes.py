"""The 4-bit attention where there is work for many steps per CTA: several heads per CTA, teams of CTAs, places without a head."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_kvq import Layer, api  # noqa: F401  (api is a fixture)

pytestmark = pytest.mark.gpu


def _shape(lens, nodes, gamma, H):
    """Heads per CTA and CTAs per team (log2), as the kernels choose them on this GPU."""
    rows = nodes * (1 + gamma)
    tile = 0 if rows <= 16 else 32 if rows <= 32 else 64
    block, chunk = tile or (8 if rows <= 8 else 16), 128 if tile else 32
    warps = 0 if tile else 2
    grid = torch.cuda.get_device_properties(0).multi_processor_count * (1 if tile else 3 if block == 8 else 2)
    streams = 0 if gamma == 0 else min((block + gamma - 2) // gamma + 1, nodes) * gamma
    extra = -(-(nodes + streams) // chunk)
    blocks = -(-rows // block) * len(lens)
    chunks = sum((-(-n // chunk) + extra) * -(-rows // block) for n in lens)
    if chunks * H < (6 << warps) * grid:
        return 0, 0
    fits = lambda lg: 8 * (-(-H // (1 << lg)) << lg) <= 9 * H
    heads = team = 0
    while heads < warps and fits(heads + 1) and 10 * blocks * (H >> (heads + 1)) >= grid:
        heads += 1
    while team < 3 and fits(heads + team + 1):
        team += 1
    return heads, team


# heads, head_dim, sequences, nodes, streams; heads per CTA and CTAs per team (log2)
CASES = [(32, 64, 8, 1, 0, (2, 3)), (13, 80, 16, 5, 0, (1, 0)), (15, 128, 16, 4, 1, (2, 2)), (31, 64, 10, 16, 0, (2, 3)), (14, 80, 16, 4, 3, (1, 0)),
         (32, 128, 9, 12, 0, (2, 3)), (13, 128, 10, 20, 0, (0, 1)), (15, 64, 10, 64, 0, (0, 3)), (31, 80, 9, 27, 2, (0, 3)), (32, 64, 8, 8, 3, (0, 3)),
         (7, 128, 24, 30, 0, (0, 0))]


@pytest.mark.parametrize("H,d,B,nodes,gamma,shape", CASES)
@pytest.mark.parametrize("order", ["slots", "heads"])
def test_attention_of_batches_with_many_steps(api, H, d, B, nodes, gamma, shape, order):
    rng = np.random.default_rng(H + nodes)
    lens = [int(n) for n in rng.integers(1400, 2600, B)]
    lens[1], lens[B - 2] = 3, 0                                # (units of one step between the long ones)
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        assert _shape(lens, nodes, gamma, H) == shape
    counts = [nodes if b % 3 else max(1, nodes - b) for b in range(B)]
    x = Layer(api, B, H, d, lens, counts, gamma, seed=H + d, order=order)
    rooms = []
    for name in ("o_main", "o_spec", "lse_main", "lse_spec"):  # what lies around the outputs
        t = getattr(x, name)
        if t is not None:
            rooms.append(torch.full((t.numel() + 4096,), 77.0, dtype=t.dtype, device="cuda"))
            setattr(x, name, rooms[-1][2048:-2048].view(t.shape))
    ws = x.run()
    x.check([0, 1, 2, B // 2, B - 2, B - 1])
    first = [t.clone() for t in rooms]
    for t in rooms:
        assert (t[:2048] == 77.0).all() and (t[-2048:] == 77.0).all()
        t.fill_(77.0)
    x.run(ws)                                                  # the same results, whatever the order of arrival
    assert all(torch.equal(t, f) for t, f in zip(rooms, first))
