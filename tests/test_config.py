"""CPU tests of the binding's Config: what it keeps for the calls follows its fields."""
import copy
import pickle

from paper_2606_24033_amd import blockgtq as bg


def cfg_of(**kw):
    return bg.Config(**{**dict(n_layers=2, batch=3, n_kv_heads=2, group=4, capacity=128, k_budget=128, v_bits=2), **kw})


def test_a_field_set_while_another_thread_makes_the_struct(monkeypatch):
    """Whether it is set before or after the struct holds the old value: the next call has the new one."""
    real, cfg = bg._Config, cfg_of()

    def between(*fields):
        monkeypatch.setattr(bg, "_Config", real)
        made = real(*fields)
        cfg.batch = 99  # (the other thread, behind this one's reads)
        return made
    monkeypatch.setattr(bg, "_Config", between)
    cfg.c()
    assert cfg.c().batch == 99
    assert bg.Config.c(cfg).batch == 99 and cfg._make()[1][3] == (2, 99, 2, 128)


def test_copies_follow_their_own_fields():
    cfg = cfg_of()
    cfg.c()
    for other in (copy.copy(cfg), copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg))):
        assert other == cfg
        other.v_bits = 5
        assert (other.c().v_bits, cfg.c().v_bits) == (5, 2)
