"""The package's names are the binding's."""


def test_a_name_is_what_the_binding_has_now(monkeypatch):
    import paper_2404_16109_amd as zk
    first = zk.zkmi_version
    assert first is zk.binding.zkmi_version
    monkeypatch.setattr(zk.binding, "zkmi_version", lambda: "another")
    assert zk.zkmi_version() == "another"
    monkeypatch.undo()
    assert zk.zkmi_version is first
    monkeypatch.setattr(zk.binding, "a_new_name", 5, raising=False)
    assert zk.a_new_name == 5
    monkeypatch.undo()
    assert not hasattr(zk, "a_new_name")


def test_names_that_are_not_there():
    import paper_2404_16109_amd as zk
    for name in ("no_such_entry_point", "__no_such_attribute__"):
        assert not hasattr(zk, name)
