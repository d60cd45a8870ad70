"""Block tables and slots on the GPU against the slot-by-slot reference: all
outputs equal."""
import numpy as np
import pytest

from tests import decode_ref as ref

pytestmark = pytest.mark.gpu


def _state(rng, B, max_blocks, S, spare, done_share=0.2, grow_hi=20, empty_share=0.2):
    """Slots with some blocks held, a ring that wraps, lengths that may end anywhere in the last block (or below it,
    where drafts were rejected)."""
    held = rng.randint(0, max_blocks + 1, B)
    held[rng.rand(B) < empty_share] = 0
    lens = np.array([rng.randint(max(0, h * S - 2 * S), h * S + 1) for h in held])
    total = int(held.sum())
    N = total + spare
    ids = rng.permutation(N).astype(np.int32)
    table = rng.randint(-5, N, (B, max_blocks)).astype(np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    head = int(rng.randint(0, N)) if N else 0
    ring = rng.randint(0, max(N, 1), N).astype(np.int32)
    ring[(head + np.arange(spare)) % N] = ids[total:]
    done = (rng.rand(B) < done_share).astype(np.uint8)
    grow = rng.randint(0, grow_hi + 1, B)
    return dict(grow=grow.astype(np.int32), table=table, held=held.astype(np.int32), lens=lens.astype(np.int32),
                ring=ring, ring_pos=np.array([head, spare], np.int32), done=done)


def _run(s, S, T, with_done=True):
    import torch

    import paper_2609_15359_amd as maps
    d = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in s.items()}
    r = maps.block_step(d["grow"], d["table"], d["held"], d["lens"], d["ring"], d["ring_pos"], S, T,
                        done=d["done"] if with_done else None)
    torch.cuda.synchronize()
    got = dict(table=d["table"], ring=d["ring"], slots=r.slots, tok_off=r.tok_off, lens=r.lens, held=r.held,
               ring_pos=r.ring_pos, granted=r.granted)
    return {k: v.cpu().numpy() for k, v in got.items()}, maps.error_names(int(r.dev_err.item()))


def _same(got, want, held_rows=None):
    for k in want:
        assert np.array_equal(got[k].astype(np.int64), np.asarray(want[k], np.int64)), k


@pytest.mark.parametrize("B,max_blocks,S,spare,grow_hi", [
    (1, 4, 16, 8, 40), (7, 5, 16, 30, 33), (64, 12, 16, 400, 1), (64, 12, 16, 20, 60), (300, 9, 7, 500, 31),
    (1000, 3, 64, 700, 200), (33, 40, 1, 300, 9), (8192, 3, 32, 9000, 64)])
def test_step_matches_the_reference(B, max_blocks, S, spare, grow_hi):
    rng = np.random.RandomState(B + S)
    for with_done in (True, False):
        s = _state(rng, B, max_blocks, S, spare, grow_hi=grow_hi)
        s["grow"] = np.minimum(s["grow"], max_blocks * S - np.where(with_done * s["done"], 0, s["lens"])).astype(np.int32)
        T = int(s["grow"].sum()) + 5                        # five entries past the last token
        got, err = _run(s, S, T, with_done)
        assert err == []
        _same(got, ref.block_step(s["grow"], s["table"], s["held"], s["lens"], s["ring"], s["ring_pos"], S, T,
                                  s["done"] if with_done else None))


def test_a_slot_is_refilled_in_the_call_that_ends_its_request():
    """Its old blocks go back, its new ones come from the ring: a row is read before it is rewritten."""
    rng = np.random.RandomState(3)
    s = _state(rng, 200, 30, 16, 7000, done_share=1.0, grow_hi=480, empty_share=0.0)
    T = int(s["grow"].sum())
    got, err = _run(s, 16, T)
    assert err == []
    _same(got, ref.block_step(s["grow"], s["table"], s["held"], s["lens"], s["ring"], s["ring_pos"], 16, T, s["done"]))


def test_prompts_of_long_requests():
    rng = np.random.RandomState(5)
    B, S = 96, 16
    lens = np.rint(np.exp(rng.uniform(0, 9.7, B))).astype(np.int32)
    need = -(-lens // S)
    N = int(need.sum()) - 100                               # the last ones are refused
    s = dict(grow=lens, table=np.full((B, int(need.max())), -1, np.int32), held=np.zeros(B, np.int32),
             lens=np.zeros(B, np.int32), ring=rng.permutation(N).astype(np.int32),
             ring_pos=np.array([N - 3, N], np.int32), done=np.zeros(B, np.uint8))
    T = int(lens.sum())
    got, err = _run(s, S, T)
    assert err == [] and not got["granted"].all()
    _same(got, ref.block_step(s["grow"], s["table"], s["held"], s["lens"], s["ring"], s["ring_pos"], S, T, s["done"]))


def test_value_errors():
    """Each raises its bit and stays in its arrays."""
    rng = np.random.RandomState(9)
    base = _state(rng, 20, 6, 16, 60, grow_hi=3)
    for name, change, bit in (
            ("negative growth", lambda s: s["grow"].__setitem__(3, -1), "NEG_LEN"),
            ("negative length", lambda s: s["lens"].__setitem__(3, -7), "NEG_LEN"),
            ("more blocks than a row has", lambda s: s["held"].__setitem__(3, 7), "BLOCK_TABLE"),
            ("a request that outgrows its row", lambda s: s["grow"].__setitem__(3, 97), "BLOCK_TABLE"),
            ("a front outside the ring", lambda s: s["ring_pos"].__setitem__(0, len(s["ring"])), "BLOCK_TABLE"),
            ("more free blocks than there are", lambda s: s["ring_pos"].__setitem__(1, len(s["ring"]) + 1), "BLOCK_TABLE"),
            ("blocks given back twice", lambda s: (s["done"].fill(1), s["ring_pos"].__setitem__(1, len(s["ring"]))), "BLOCK_TABLE"),
            ("a free block that does not exist", lambda s: (s["ring"].fill(len(s["ring"])), s["grow"].fill(16)), "BLOCK_TABLE")):
        s = {k: v.copy() for k, v in base.items()}
        change(s)
        T = int(np.maximum(s["grow"], 0).sum())
        got, err = _run(s, 16, T)
        assert bit in err, (name, err)
        assert got["slots"].max(initial=-1) < 16 * len(s["ring"]), name
    got, err = _run(base, 16, int(base["grow"].sum()) - 1)
    assert err == ["SEG_OFFSETS"]


@pytest.mark.parametrize("B,short", [(20, 1), (20, 30), (300, 1), (300, 500)])
def test_a_total_that_is_too_small_takes_no_block(B, short):
    """No slot is granted, blocks of finished requests come back all the same, and every block is in a row or in the ring
    once."""
    rng = np.random.RandomState(B + short)
    s = _state(rng, B, 6, 16, 200 * B // 20, grow_hi=40)
    s["grow"] = np.minimum(s["grow"], 6 * 16 - np.where(s["done"], 0, s["lens"])).astype(np.int32)
    N, T = len(s["ring"]), int(s["grow"].sum()) - short
    got, err = _run(s, 16, T)
    assert err == ["SEG_OFFSETS"]
    zero = {**s, "grow": np.zeros_like(s["grow"])}
    want = ref.block_step(zero["grow"], s["table"], s["held"], s["lens"], s["ring"], s["ring_pos"], 16, T, s["done"])
    for k in ("table", "ring", "lens", "held", "ring_pos"):
        assert np.array_equal(got[k].astype(np.int64), np.asarray(want[k], np.int64)), k
    assert not got["granted"].any() and (got["slots"] == -1).all()
    assert np.array_equal(got["tok_off"], np.concatenate([[0], np.cumsum(s["grow"].astype(np.int64))]))
    used = np.concatenate([got["table"][b, :got["held"][b]] for b in range(B)])
    free = got["ring"][(got["ring_pos"][0] + np.arange(got["ring_pos"][1])) % N]
    assert sorted(np.concatenate([used, free]).tolist()) == list(range(N))


def test_arrays_to_write_into():
    """A result of an earlier call takes the next one's values; whatever else could be written past or while it is read
    is refused before anything is launched."""
    import dataclasses

    import torch

    import paper_2609_15359_amd as maps
    rng = np.random.RandomState(13)
    s = _state(rng, 30, 5, 16, 60, done_share=0.0, grow_hi=9)
    s["grow"] = np.minimum(s["grow"], 5 * 16 - s["lens"]).astype(np.int32)
    T, B = int(s["grow"].sum()), 30
    d = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in s.items() if k != "done"}
    first = maps.block_step(block_size=16, total=T, **d)
    def empty(n, dtype=torch.int32):
        return torch.empty(n, dtype=dtype, device="cuda")
    blank = maps.BlockStep(slots=empty(T, torch.int64), tok_off=empty(B + 1, torch.int64), lens=empty(B), held=empty(B),
                           ring_pos=empty(2), granted=empty(B, torch.uint8), dev_err=first.dev_err)
    again = maps.block_step(block_size=16, total=T, out=blank, **d)
    assert again is blank
    for name in ("slots", "tok_off", "lens", "held", "ring_pos", "granted"):
        assert torch.equal(getattr(again, name), getattr(first, name)), name
    before = {k: v.clone() for k, v in d.items()}
    both = empty(2 * B - 1)
    for wrong, error, what in (
            (dict(slots=empty(T + 1, torch.int64)), maps.MapsError, "slots"), (dict(tok_off=empty(B, torch.int64)), maps.MapsError, "tok_off"),
            (dict(lens=empty(B - 1)), maps.MapsError, "lens"), (dict(held=empty(B + 1)), maps.MapsError, "held"),
            (dict(ring_pos=empty(1)), maps.MapsError, "ring_pos"), (dict(granted=empty(B - 1, torch.uint8)), maps.MapsError, "granted"),
            (dict(tok_off=empty(B + 1)), TypeError, "tok_off"), (dict(lens=empty(B, torch.int64)), TypeError, "lens"),
            (dict(held=empty(B, torch.uint8)), TypeError, "held"), (dict(ring_pos=empty(2, torch.int64)), TypeError, "ring_pos"),
            (dict(granted=empty(B)), TypeError, "granted"), (dict(held=empty(2 * B)[::2]), maps.MapsError, "contiguous"),
            (dict(granted=torch.empty(B, dtype=torch.uint8)), maps.MapsError, "device tensor"),
            (dict(held=d["lens"]), maps.MapsError, "overlap"), (dict(lens=d["grow"]), maps.MapsError, "overlap"),
            (dict(lens=d["lens"]), maps.MapsError, "overlap"), (dict(held=d["ring"][5:5 + B]), maps.MapsError, "overlap"),
            (dict(lens=d["table"].flatten()[-B:]), maps.MapsError, "overlap"),
            (dict(ring_pos=d["ring_pos"]), maps.MapsError, "overlap"),
            (dict(lens=both[:B], held=both[B - 1:]), maps.MapsError, "overlap")):
        with pytest.raises(error, match=what):
            maps.block_step(block_size=16, total=T, out=dataclasses.replace(blank, **wrong), **d)
    torch.cuda.synchronize()
    assert all(torch.equal(d[k], before[k]) for k in d)


def test_tables_from_step_to_step():
    """BlockTables over 30 steps of requests that come, grow, shrink and end, against the reference on the host."""
    import torch

    import paper_2609_15359_amd as maps
    rng = np.random.RandomState(11)
    B, max_blocks, N, S = 40, 8, 150, 16
    t = maps.BlockTables(B, max_blocks, N, S)
    want = dict(table=np.full((B, max_blocks), -1, np.int32), held=np.zeros(B, np.int64), lens=np.zeros(B, np.int64),
                ring=np.arange(N, dtype=np.int32), ring_pos=np.array([0, N]))
    for step in range(30):
        done = ((rng.rand(B) < 0.15) & (want["lens"] > 0)).astype(np.uint8)
        base = np.where(done, 0, want["lens"])
        grow = np.where(base == 0, rng.randint(1, 60, B) * (rng.rand(B) < 0.5), rng.randint(0, 5, B))
        grow = np.minimum(grow, max_blocks * S - base).astype(np.int32)
        T = int(grow.sum())
        r = t.step(torch.from_numpy(grow).cuda(), T, torch.from_numpy(done).cuda())
        want = ref.block_step(grow, want["table"], want["held"], want["lens"], want["ring"], want["ring_pos"], S, T, done)
        got = dict(table=t.table, ring=t.ring, slots=r.slots, tok_off=r.tok_off, lens=t.lens, held=t.held,
                   ring_pos=t.ring_pos, granted=r.granted)
        _same({k: v.cpu().numpy() for k, v in got.items()}, want)
        back = np.minimum(rng.randint(0, 3, B), want["lens"]).astype(np.int32)      # rejected drafts
        t.lens -= torch.from_numpy(back).cuda()
        want["lens"] = want["lens"] - back
        used = np.concatenate([want["table"][b, :want["held"][b]] for b in range(B)])
        free = want["ring"][(want["ring_pos"][0] + np.arange(want["ring_pos"][1])) % N]
        assert sorted(np.concatenate([used, free]).tolist()) == list(range(N))      # no block lost or held twice
    assert int(t.dev_err.item()) == 0
